// Beam search's selection over beams and vocabulary.
//
// Within a row the order of the scores, score + ((logit - max) - log(sum)), is
// the order of the logits.  The vocabulary is read once, for the row's maximum,
// its sum of exponentials and the maxima of groups of 128 logits (256 of 16
// bits).  A value that k = 2 beams of those maxima reach bounds the k largest
// logits from below, so a second kernel reads only the groups that reach it
// again, turns the k largest logits of each of a request's rows into scores
// and ranks them.
#include <algorithm>
#include <cfloat>

#include "wf_device.cuh"
#include "wf_kv4.cuh"

namespace wf {

struct SelectParams {
  const void *logits;
  long long ld;
  const float *scores;
  const uint8_t *suppress;
  int n_req, W, V, eos;
  int tiles, segments, groups;  // tiles of a warp's segment; segments and groups of a row
  int32_t *token, *parent;
  float *score;
  int32_t *fin_parent;
  float *fin_score;
  // scratch
  unsigned long long *sum;  // [rows][segments] in units of 2^-40, relative to
  float *max;               // [rows][segments]
  float *group_max;         // [rows][groups]
};
constexpr int kSelThreads = 256;
constexpr int kSelWarps = kSelThreads / 32;
constexpr int kSelBlocks = 3;  // CTAs of an SM
constexpr int kSelPer = 32;             // logits of a lane and tile
constexpr int kSelTile = 32 * kSelPer;  // of a warp's step
constexpr int kSelTiles = 8;            // of a segment, at most
constexpr int kSelKeep = 128;           // candidates of a row that the join holds

// (value descending, index ascending) as one descending unsigned key; 0 is
// below every key of a value above -inf.
__device__ __forceinline__ uint32_t order_bits(float v) {
  const uint32_t b = __float_as_uint(v + 0.f);  // -0 as 0
  return (b & 0x80000000u) ? ~b : (b | 0x80000000u);
}
__device__ __forceinline__ unsigned long long order_key(float v, uint32_t idx) {
  return static_cast<unsigned long long>(order_bits(v)) << 32 | (0xffffffffu - idx);
}
__device__ __forceinline__ float order_value(uint32_t o) {
  return __uint_as_float((o & 0x80000000u) ? (o & 0x7fffffffu) : ~o);
}
__device__ __forceinline__ float key_value(unsigned long long k) { return order_value(static_cast<uint32_t>(k >> 32)); }
__device__ __forceinline__ uint32_t key_index(unsigned long long k) { return 0xffffffffu - static_cast<uint32_t>(k); }
// The largest key of a warp: its upper word, then the largest lower word under it (if there are several).
__device__ __forceinline__ unsigned long long warp_max(unsigned long long k) {
  const uint32_t hi = __reduce_max_sync(0xffffffffu, static_cast<uint32_t>(k >> 32));
  const unsigned have = __ballot_sync(0xffffffffu, static_cast<uint32_t>(k >> 32) == hi);
  const uint32_t lo = (have & (have - 1)) ? __reduce_max_sync(0xffffffffu, static_cast<uint32_t>(k >> 32) == hi ? static_cast<uint32_t>(k) : 0u)
                                          : __shfl_sync(0xffffffffu, static_cast<uint32_t>(k), __ffs(have) - 1);
  return static_cast<unsigned long long>(hi) << 32 | lo;
}
// floor(x 2^k) of x in [0, 2^(63 - k)), by shifts: the FP64 pipe takes a warp's
// instruction in tens of clocks, and its conversions with it.
__device__ __forceinline__ unsigned long long fixed_point(float x, int k) {
  const uint32_t b = __float_as_uint(x), e = b >> 23;
  const unsigned long long mant = (b & 0x7fffffu) | (e ? 0x800000u : 0u);
  const int up = static_cast<int>(e ? e : 1u) - 150 + k;
  return up >= 0 ? mant << up : up > -24 ? mant >> -up : 0;
}
// Sorts a warp's values, largest in lane 0: a bitonic network.
__device__ __forceinline__ float warp_sort(float v, int lane) {
#pragma unroll
  for (int size = 2; size <= 32; size <<= 1)
#pragma unroll
    for (int off = size >> 1; off; off >>= 1) {
      const float w = __shfl_xor_sync(0xffffffffu, v, off);
      v = ((lane & off) == 0) == ((lane & size) == 0) ? fmaxf(v, w) : fminf(v, w);
    }
  return v;
}

template <typename T>
struct Logits;
template <>
struct Logits<float> {
  static constexpr int kVec = 4;
  static __device__ __forceinline__ float one(const uint4 *v, int i) { return reinterpret_cast<const float *>(v)[i]; }
  static __device__ __forceinline__ void unpack(uint4 v, float *x) {
    x[0] = __uint_as_float(v.x), x[1] = __uint_as_float(v.y), x[2] = __uint_as_float(v.z), x[3] = __uint_as_float(v.w);
  }
};
template <typename T>
struct Logits16 {
  static constexpr int kVec = 8;
  static __device__ __forceinline__ float one(const uint4 *v, int i) { return Kv4Type<T>::lo(reinterpret_cast<const uint16_t *>(v)[i]); }
  static __device__ __forceinline__ void unpack(uint4 v, float *x) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) x[2 * i] = Kv4Type<T>::lo(w[i]), x[2 * i + 1] = Kv4Type<T>::hi(w[i]);
  }
};
template <>
struct Logits<__nv_bfloat16> : Logits16<__nv_bfloat16> {};
template <>
struct Logits<__half> : Logits16<__half> {};

// kVec logits from id on, those outside [0, V) as -inf.
template <typename T>
__device__ __noinline__ uint4 edge_vector(const T *src, int id, int V) {
  constexpr int kVec = Logits<T>::kVec, kBits = 128 / kVec;
  uint32_t w[4];
  uint32_t none = 0xff800000u;  // -inf in fp32
  if constexpr (kBits == 16) none = Kv4Type<T>::pack(-INFINITY, -INFINITY) & 0xffffu;
  for (int i = 0; i < 4; ++i) {
    w[i] = 0;
    for (int e = 0; e < kVec / 4; ++e) {
      const int at = id + i * (kVec / 4) + e;
      uint32_t bits = none;
      if (at >= 0 && at < V) bits = kBits == 32 ? reinterpret_cast<const uint32_t *>(src)[at] : reinterpret_cast<const uint16_t *>(src)[at];
      w[i] |= bits << (kBits * e & 31);
    }
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}

__device__ __noinline__ uint4 edge_bytes(const uint8_t *src, int id, int V) {
  uint32_t w[4] = {};
  for (int i = 0; i < 16; ++i)
    if (id + i >= 0 && id + i < V) w[i >> 2] |= static_cast<uint32_t>(src[id + i]) << (8 * (i & 3));
  return make_uint4(w[0], w[1], w[2], w[3]);
}

// Logits of a row by 16-byte vectors from the multiple of 16 bytes at or before
// its first one, whatever its alignment.
template <typename T>
struct RowOf {
  const T *src;
  int V, skew;
  __device__ __forceinline__ RowOf(const SelectParams &p, long long row)
      : src(static_cast<const T *>(p.logits) + row * p.ld), V(p.V), skew(static_cast<int>((reinterpret_cast<uintptr_t>(src) & 15) / sizeof(T))) {}
  __device__ __forceinline__ uint4 vector(int id) const {
    return id >= 0 && id + Logits<T>::kVec <= V ? *reinterpret_cast<const uint4 *>(src + id) : edge_vector<T>(src, id, V);
  }
};

__device__ __forceinline__ void copy16_async(void *smem_dst, const void *src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_u32(smem_dst)), "l"(src) : "memory");
}

// A CTA has a segment of up to 8 tiles of 1024 logits of eight rows, a warp
// each; its suppressed ids are read once for the eight.  A tile's logits go to
// shared memory and from there to registers, which frees their place for the
// next tile's while this one is worked on: bound by HBM, and by the ends of the
// one wave of CTAs.  With the joining kernel after it 96 requests x 5 beams x
// 51866 fp32 take 28.8 us, 3.5 TB/s (tiles straight to registers and a mask per
// warp 30.8; four CTAs an SM, which spill, 31.3).  The sum adds a tile's 32
// terms a lane in fp32 and the tiles with the rounding carried along; lanes and
// segments add in fixed point (2^-40), without order.  A NaN is never the
// larger of a comparison, which keeps it out of the maxima and the candidates;
// only the sum has to look for it.
template <typename T>
__global__ void __launch_bounds__(kSelThreads, kSelBlocks) beam_segment_kernel(const SelectParams p) {
  using L = Logits<T>;
  constexpr int kVec = L::kVec, kVecs = kSelPer / kVec;
  constexpr int kMask = kSelTiles * kSelTile + 48;         // 16 bytes before a segment, for skew, and to the next multiple of 16
  __shared__ uint4 ahead[kSelWarps][kVecs][32];            // the next tile: a lane's own vectors, which no other lane reads
  __shared__ __align__(16) unsigned char mask[kMask + 16]; // the segment's suppressed ids, for all the CTA's rows
  __shared__ uint32_t flags[kMask / 512 + 4];              // bit i of word k: some id of mask's 16 from 512 k + 16 i on
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int segment = blockIdx.x % p.segments;
  const long long row = static_cast<long long>(blockIdx.x / p.segments) * kSelWarps + warp, unit = row * p.segments + segment;
  const bool live = row < static_cast<long long>(p.n_req) * p.W;
  pdl_wait();
  const RowOf<T> in(p, live ? row : 0);
  const int base = segment * p.tiles * kSelTile, start = base - in.skew, end = live ? min(start + p.tiles * kSelTile, p.V) : start;
  float *group = p.group_max + row * p.groups + segment * p.tiles * kVecs;
  float m = -INFINITY, sum = 0.f, carry = 0.f;
  uint4 *next = &ahead[warp][0][lane];
  const auto request = [&](int first) {
    if (first >= 0 && first + kSelTile <= p.V) {
#pragma unroll
      for (int v = 0; v < kVecs; ++v) copy16_async(next + v * 32, in.src + first + (v * 32 + lane) * kVec);
    } else {
#pragma unroll 1
      for (int v = 0; v < kVecs; ++v) {
        const int id = first + (v * 32 + lane) * kVec;
        if (id >= 0 && id + kVec <= p.V)
          copy16_async(next + v * 32, in.src + id);
        else
          next[v * 32] = edge_vector<T>(in.src, id, p.V);
      }
    }
  };
  if (start < end) request(start);
  int mask_from = 0;  // id of mask's first byte; the id's address is a multiple of 16
  if (p.suppress) {
    mask_from = base - 16 - static_cast<int>((reinterpret_cast<uintptr_t>(p.suppress) + base) & 15);
    for (int i = threadIdx.x; i < (kMask / 512 + 1) * 32; i += kSelThreads) {  // whole warps: their ballots are the flags
      const int id = mask_from + i * 16;
      uint4 w = {};
      if (i * 16 < p.tiles * kSelTile + 48) {
        if (id >= 0 && id + 16 <= p.V)
          w = *reinterpret_cast<const uint4 *>(p.suppress + id);
        else if (id + 16 > 0 && id < p.V)
          w = edge_bytes(p.suppress, id, p.V);
        *reinterpret_cast<uint4 *>(mask + i * 16) = w;
      }
      const uint32_t some = __ballot_sync(0xffffffffu, (w.x | w.y | w.z | w.w) != 0);
      if (lane == 0) flags[i >> 5] = some;
    }
    __syncthreads();
  }
  for (int first = start; first < end; first += kSelTile, group += kVecs) {
    float x[kSelPer];
    asm volatile("cp.async.wait_all;" ::: "memory");
#pragma unroll
    for (int v = 0; v < kVecs; ++v) L::unpack(next[v * 32], x + v * kVec);
    if (first + kSelTile < end) request(first + kSelTile);
    if (p.suppress) {
      const int from = first - mask_from;
      if (flags[from >> 9] | flags[(from >> 9) + 1] | flags[(from >> 9) + 2]) {
#pragma unroll
        for (int q = 0; q < kSelPer / 4; ++q) {
          const int at = from + ((q * 4 / kVec) * 32 + lane) * kVec + q * 4 % kVec;
          const uint32_t *word = reinterpret_cast<const uint32_t *>(mask) + (at >> 2);
          const uint32_t b = __funnelshift_r(word[0], word[1], (at & 3) * 8);
          if (!b) continue;
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (b & (0xffu << (8 * e))) x[q * 4 + e] = -INFINITY;
        }
      }
    }
    // the groups' maxima, lane v that of vector v
    float tops = 0.f, tile_top = -INFINITY;
#pragma unroll
    for (int v = 0; v < kVecs; ++v) {
      float t = max3(-INFINITY, x[v * kVec], x[v * kVec + 1]);  // -inf where all are NaN: the join orders these
#pragma unroll
      for (int e = 2; e < kVec; e += 2) t = max3(t, x[v * kVec + e], x[v * kVec + e + 1]);
      const float g = warp_max(t);
      tops = lane == v ? g : tops;
      tile_top = fmaxf(tile_top, g);
    }
    if (lane < kVecs) group[lane] = tops;
    if (tile_top == -INFINITY) continue;
    if (tile_top > m) {
      const float f = expf(m - tile_top);
      sum *= f, carry *= f;
      m = tile_top;
    }
    float2 part2 = {0.f, 0.f};
#pragma unroll
    for (int i = 0; i < kSelPer; i += 2) {  // the difference first: its rounding does not grow with the logits
      const float2 y = mul2(add2(make_float2(x[i], x[i + 1]), make_float2(-m, -m)), make_float2(1.4426950408889634f, 1.4426950408889634f));
      part2 = add2(part2, make_float2(ex2(y.x), ex2(y.y)));
    }
    float part = part2.x + part2.y;
    if (part != part) {  // a NaN; or a +inf, whose row the join knows by its maximum
      part = 0.f;
#pragma unroll
      for (int i = 0; i < kSelPer; ++i) {
        const float e = ex2((x[i] - m) * 1.4426950408889634f);
        part += e == e ? e : 0.f;
      }
    }
    const float y = part - carry, t = sum + y;
    carry = (t - sum) - y;
    sum = t;
  }
  pdl_launch_dependents();  // not before: the join's CTAs would take the room of this kernel's
  if (!live) return;
  // tiles of the last segment that lie past the row
  for (int i = static_cast<int>(group - p.group_max - row * p.groups) + lane; i < min((segment + 1) * p.tiles * kVecs, p.groups); i += 32)
    p.group_max[row * p.groups + i] = -INFINITY;
  unsigned long long fixed = fixed_point(sum, 40);
#pragma unroll
  for (int off = 16; off; off >>= 1) fixed += __shfl_xor_sync(0xffffffffu, fixed, off);
  if (lane == 0) p.sum[unit] = fixed, p.max[unit] = m;
}

// 512 groups' maxima, 16 a lane, all loads in flight; -inf past the last.
__device__ __forceinline__ void load_groups(const float *tops, int base, int groups, int lane, float (&t)[16]) {
#pragma unroll
  for (int u = 0; u < 16; ++u) {
    const int i = base + u * 32 + lane;
    t[u] = i < groups ? tops[i] : -INFINITY;
  }
}

// One CTA per request, two warps per beam: one picks the row's best logits,
// one takes its maximum and sum meanwhile; the logarithms (in 64 bits) are one
// warp's for all rows.  Most of
// its time is the latency of a few dependent reads, so each is issued at once:
// the maxima into registers, the groups into shared memory.  About 5 us of one
// request's 9.5 and 7 of 96 requests' 28.5 with 5 beams each; one request's 16
// beams take 20 in all, by issue on one SM.
constexpr int kJoinGroups = 64;  // groups of a row that are looked through
constexpr int kJoinAhead = 8;    // of them in shared memory at a time
template <typename T>
__global__ void __launch_bounds__(2 * WF_MAX_BEAMS * 32, 1) beam_join_kernel(const SelectParams p) {
  using L = Logits<T>;
  constexpr int kVec = L::kVec;
  const int W = p.W, K = 2 * W, req = blockIdx.x, lane = threadIdx.x & 31, beam = threadIdx.x >> 5;
  __shared__ unsigned long long keeps[WF_MAX_BEAMS][kSelKeep], best_key[WF_MAX_BEAMS * 2 * WF_MAX_BEAMS], cand[WF_MAX_BEAMS * 2 * WF_MAX_BEAMS];
  __shared__ unsigned long long ranked[2 * WF_MAX_BEAMS], row_sum[WF_MAX_BEAMS];
  __shared__ float row_max[WF_MAX_BEAMS], row_log[WF_MAX_BEAMS], row_score[WF_MAX_BEAMS];
  __shared__ int counts[WF_MAX_BEAMS], chosen[WF_MAX_BEAMS][kJoinGroups];
  extern __shared__ uint4 vectors[];  // [W][kJoinAhead][32]
  pdl_wait();
  pdl_launch_dependents();
  const long long row0 = static_cast<long long>(req) * W;
  if (beam >= W) {
    const int w = beam - W;
    const float *sm = p.max + (row0 + w) * p.segments;
    const unsigned long long *ss = p.sum + (row0 + w) * p.segments;
    const float m0 = lane < p.segments ? sm[lane] : -INFINITY;
    const unsigned long long s0 = lane < p.segments ? ss[lane] : 0;
    if (lane == 0) row_score[w] = p.scores[row0 + w];
    if (w == 0 && lane < K) ranked[lane] = 0;
    float m = m0;
    for (int c = lane + 32; c < p.segments; c += 32) m = fmaxf(m, sm[c]);
    m = warp_max(m);
    const auto scaled = [&](unsigned long long v, float at) -> unsigned long long {
      if (at == m) return v;
      const float f = expf(at - m);
      return f < 1.f ? __umul64hi(v, fixed_point(f, 64)) : f == 1.f ? v : 0;
    };
    unsigned long long s = scaled(s0, m0);
    for (int c = lane + 32; c < p.segments; c += 32) s += scaled(ss[c], sm[c]);
#pragma unroll
    for (int off = 16; off; off >>= 1) s += __shfl_xor_sync(0xffffffffu, s, off);
    if (lane == 0) row_max[w] = m, row_sum[w] = s;
    asm volatile("bar.sync 1, %0;" ::"r"(W * 32) : "memory");  // these warps; one takes the logarithms of all rows
    if (w == 0 && lane < W) row_log[lane] = static_cast<float>(log(static_cast<double>(row_sum[lane]) * 0x1p-40));
  } else {
    const long long row = row0 + beam;
    float *tops = p.group_max + row * p.groups;
    float lane_top = -INFINITY, lane_next = -INFINITY;  // the largest and the next of this lane's groups
    if (lane == 0) counts[beam] = 0;
    for (int i = lane; i < K; i += 32) best_key[beam * K + i] = 0;
    for (int base = 0; base < p.groups; base += 512) {
      float t[16];
      load_groups(tops, base, p.groups, lane, t);
#pragma unroll
      for (int u = 0; u < 16; ++u) lane_next = fmaxf(lane_next, fminf(lane_top, t[u])), lane_top = fmaxf(lane_top, t[u]);
    }
    __syncwarp();
    // Of 32 maxima over the lanes' groups the K-th is reached by K groups and
    // few more (all, below K finite ones); for K above 16, of the lanes' two
    // largest.  More groups than can be held: K groups one by one.
    float order = warp_sort(lane_top, lane);
    if (K > 16) order = warp_sort(fmaxf(order, __shfl_sync(0xffffffffu, warp_sort(lane_next, lane), 31 - lane)), lane);
    float floor_v = __shfl_sync(0xffffffffu, order, K - 1);
    if (floor_v == -INFINITY) floor_v = -FLT_MAX;
    for (int base = 0; base < p.groups; base += 512) {
      float t[16];
      load_groups(tops, base, p.groups, lane, t);
      uint32_t hits = 0;
#pragma unroll
      for (int u = 0; u < 16; ++u) hits |= t[u] >= floor_v ? 1u << u : 0u;
      for (; hits; hits &= hits - 1) {
        const int at = atomicAdd(&counts[beam], 1);
        if (at < kJoinGroups) chosen[beam][at] = base + (__ffs(hits) - 1) * 32 + lane;
      }
    }
    __syncwarp();
    int n_groups = counts[beam];
    if (n_groups > kJoinGroups) {
      unsigned long long last = 0, mine = 0;
      const auto look = [&]() {
        float v = -INFINITY;
        int g = -1;
        for (int i = lane; i < p.groups; i += 32) {
          const float t = tops[i];
          if (t > v) v = t, g = i;
        }
        mine = g < 0 ? 0 : order_key(v, g);
      };
      look();
      for (n_groups = 0; n_groups < K; ++n_groups) {  // ties: the first groups, whose ids are lower
        const unsigned long long best = warp_max(mine);
        if (!best) break;
        last = best;
        if (lane == 0) chosen[beam][n_groups] = static_cast<int>(key_index(best));
        if (mine == best) {
          tops[key_index(best)] = -INFINITY;
          look();
        }
      }
      floor_v = n_groups == K ? key_value(last) : -FLT_MAX;
    }
    __syncwarp();
    // every logit of theirs that reaches the bound
    const RowOf<T> in(p, row);
    const auto id_of = [&](int k) { return chosen[beam][k] * (32 * kVec) - in.skew + lane * kVec; };
    unsigned long long *keep = keeps[beam];
    uint4 *mine = vectors + beam * (kJoinAhead * 32) + lane;
    int n = 0;
    for (bool again = floor_v == -FLT_MAX;; again = true) {
      // fewer groups than places, or a bound that too many reach: that of the lanes'
      // two largest logits (20 x 8 beams x 1000: 14 us, by rounds as below 56)
      if (again) {
        float top = -INFINITY, next = -INFINITY;
#pragma unroll 2
        for (int g = 0; g < n_groups; ++g) {
          const int id = id_of(g);
          float y[kVec];
          L::unpack(in.vector(id), y);
#pragma unroll
          for (int e = 0; e < kVec; ++e) {
            if (!(y[e] > next) || (p.suppress && p.suppress[id + e])) continue;  // (outside the row -inf)
            next = fmaxf(next, fminf(top, y[e])), top = fmaxf(top, y[e]);
          }
        }
        order = warp_sort(top, lane);
        order = warp_sort(fmaxf(order, __shfl_sync(0xffffffffu, warp_sort(next, lane), 31 - lane)), lane);
        floor_v = fmaxf(floor_v, __shfl_sync(0xffffffffu, order, K - 1));
        n = 0;
        __syncwarp();
      }
      for (int k0 = 0; k0 < n_groups; k0 += kJoinAhead) {
        const int here = min(kJoinAhead, n_groups - k0);
        for (int u = 0; u < here; ++u) {
          const int id = id_of(k0 + u);
          if (id >= 0 && id + kVec <= p.V)
            copy16_async(mine + u * 32, in.src + id);
          else
            mine[u * 32] = edge_vector<T>(in.src, id, p.V);
        }
        asm volatile("cp.async.wait_all;" ::: "memory");
        // a bit for each of a lane's values, 32 at a time; the lanes' hits one after another
        constexpr int kBatch = 32 / kVec;
#pragma unroll
        for (int u0 = 0; u0 < kJoinAhead; u0 += kBatch) {
          uint32_t hits = 0;
#pragma unroll
          for (int u = 0; u < kBatch; ++u) {
            if (u0 + u >= here) continue;
            float y[kVec];
            L::unpack(mine[(u0 + u) * 32], y);
#pragma unroll
            for (int e = 0; e < kVec; ++e) hits |= y[e] >= floor_v ? 1u << (u * kVec + e) : 0u;
          }
          int upto = __popc(hits);
#pragma unroll
          for (int off = 1; off < 32; off <<= 1) {
            const int v = __shfl_up_sync(0xffffffffu, upto, off);
            if (lane >= off) upto += v;
          }
          int at = n + upto - __popc(hits);
          n += __shfl_sync(0xffffffffu, upto, 31);
          for (; hits && at < kSelKeep; hits &= hits - 1, ++at) {
            const int bit = __ffs(hits) - 1, u = u0 + bit / kVec, e = bit % kVec;
            keep[at] = order_key(L::one(mine + u * 32, e), id_of(k0 + u) + e);
          }
        }
      }
      if (n <= kSelKeep || again) break;
    }
    __syncwarp();
    if (n <= kSelKeep) {  // each one's rank is the number of larger ones
      if (p.suppress)
        for (int i = lane; i < n; i += 32)
          if (p.suppress[key_index(keep[i])]) keep[i] = 0;
      __syncwarp();
      for (int i = lane; i < n; i += 32) {
        const unsigned long long key = keep[i];
        if (!key) continue;
        int rank = 0;
#pragma unroll 4
        for (int j = 0; j < n; ++j) rank += keep[j] > key;
        if (rank < K) best_key[beam * K + rank] = key;
      }
    } else {  // many equal ones: round by round over the groups
      unsigned long long below = ~0ull;
      for (int k = 0; k < K; ++k) {
        unsigned long long best = 0;
#pragma unroll 1
        for (int g = 0; g < n_groups; ++g) {
          const int id = id_of(g);
          float y[kVec];
          L::unpack(in.vector(id), y);
#pragma unroll
          for (int e = 0; e < kVec; ++e) {
            const unsigned long long key = y[e] >= floor_v && !(p.suppress && p.suppress[id + e]) ? order_key(y[e], id + e) : 0;
            if (key < below && key > best) best = key;
          }
        }
        below = warp_max(best);
        if (lane == 0) best_key[beam * K + k] = below;
      }
    }
  }
  __syncthreads();
  for (int i = threadIdx.x; i < W * K; i += blockDim.x) {
    const int w = i / K;
    const unsigned long long k = best_key[i];
    // a row whose maximum is infinite has no scores but NaN, which is no candidate
    const float m = row_max[w], total = k && m < INFINITY ? row_score[w] + ((key_value(k) - m) - row_log[w]) : -INFINITY;
    cand[i] = total > -INFINITY ? order_key(total, i) : 0;
  }
  __syncthreads();
  for (int i = threadIdx.x; i < W * K; i += blockDim.x) {
    const unsigned long long k = cand[i];
    if (!k) continue;
    int rank = 0;  // of every row, whose candidates descend, those above
#pragma unroll 4
    for (int w = 0; w < W; ++w) {
      const unsigned long long *of = cand + w * K;
      int above = 0;
      for (int step = 1 << (31 - __clz(K)); step; step >>= 1)
        if (above + step <= K && of[above + step - 1] > k) above += step;
      rank += above;
    }
    if (rank < K) ranked[rank] = k;
  }
  __syncthreads();
  if (beam != 0) return;
  // lane r has rank r
  const unsigned long long k = lane < K ? ranked[lane] : 0;
  const int place = k ? static_cast<int>(key_index(k)) : 0, b = place / K, t = k ? static_cast<int>(key_index(best_key[place])) : -1;
  const bool ends = k && t == p.eos;
  const unsigned going = __ballot_sync(0xffffffffu, k && !ends), ending = __ballot_sync(0xffffffffu, ends && lane < W);
  const unsigned below = (1u << lane) - 1;
  const size_t o = static_cast<size_t>(req) * W;
  const int at = __popc(going & below), fin = __popc(ending & below);
  if (k && !ends && at < W) p.token[o + at] = t, p.parent[o + at] = b, p.score[o + at] = key_value(k);
  if (ends && lane < W) p.fin_parent[o + fin] = b, p.fin_score[o + fin] = key_value(k);
  if (lane < W) {
    if (lane >= __popc(going)) p.token[o + lane] = -1, p.parent[o + lane] = lane, p.score[o + lane] = -INFINITY;
    if (lane >= __popc(ending)) p.fin_parent[o + lane] = -1, p.fin_score[o + lane] = -INFINITY;
  }
}

}  // namespace wf

using namespace wf;

// The kernels of a call, with one carveout: an SM drains before it changes it.
constexpr int kSelCarve = 60;  // percent: three of the first kernel's CTAs
template <typename T>
static bool select_ready(const void **segment, const void **join) {
  *segment = reinterpret_cast<const void *>(beam_segment_kernel<T>), *join = reinterpret_cast<const void *>(beam_join_kernel<T>);
  static PerDevice ready;
  return ready.get(current_device(), [&]() -> int {
    return cudaFuncSetAttribute(*join, cudaFuncAttributeMaxDynamicSharedMemorySize, WF_MAX_BEAMS * kJoinAhead * 512) == cudaSuccess &&
           cudaFuncSetAttribute(*segment, cudaFuncAttributePreferredSharedMemoryCarveout, kSelCarve) == cudaSuccess &&
           cudaFuncSetAttribute(*join, cudaFuncAttributePreferredSharedMemoryCarveout, kSelCarve) == cudaSuccess;
  });
}
constexpr int kSelMaxVocab = 1 << 22;  // its terms in units of 2^-40 stay below 2^63
// Segments of a row: as many as make one wave of CTAs, or more of at most 8 tiles.
struct SelectPlan {
  int tiles, segments, groups;
};
static SelectPlan select_plan(long long rows, int V, bool wide) {
  const int all = (V + 7 + kSelTile - 1) / kSelTile;  // 15 bytes of skew may push a row's end into another tile
  SelectPlan a;
  const long long most = std::min<long long>(all, std::max<long long>(1, kSms * kSelBlocks / ((rows + kSelWarps - 1) / kSelWarps)));
  a.tiles = static_cast<int>(std::min<long long>(kSelTiles, (all + most - 1) / most));
  a.segments = (all + a.tiles - 1) / a.tiles;
  a.groups = all * (wide ? 8 : 4);
  return a;
}

extern "C" {

size_t wf_beam_select_scratch_bytes(int32_t n_req, int32_t beams, int32_t vocab) {
  if (n_req <= 0 || beams <= 0 || beams > WF_MAX_BEAMS || vocab < 2 * beams || vocab > kSelMaxVocab) return 0;
  const SelectPlan a = select_plan(static_cast<long long>(n_req) * beams, vocab, true);
  return static_cast<size_t>(n_req) * beams * (a.segments * 12 + a.groups * 4);
}

wf_status wf_beam_select(const void *d_logits, int32_t dtype, int64_t ld, const float *d_scores, const uint8_t *d_suppress,
                         int32_t n_req, int32_t beams, int32_t vocab, int32_t eos, int32_t *d_token, int32_t *d_parent,
                         float *d_score, int32_t *d_fin_parent, float *d_fin_score, void *d_scratch, size_t scratch_bytes,
                         void *stream) {
  if (!d_logits || !d_scores || !d_token || !d_parent || !d_score || !d_fin_parent || !d_fin_score || !d_scratch || n_req <= 0 ||
      beams <= 0 || vocab <= 0 || ld < vocab || (reinterpret_cast<uintptr_t>(d_scratch) & 7) ||
      (reinterpret_cast<uintptr_t>(d_logits) & (dtype == WF_F32 ? 3 : 1)))
    return WF_ERR_INVALID;
  if (dtype < WF_BF16 || dtype > WF_F32 || beams > WF_MAX_BEAMS || vocab < 2 * beams || vocab > kSelMaxVocab)
    return WF_ERR_UNSUPPORTED;
  const long long rows = static_cast<long long>(n_req) * beams;
  if (rows > INT32_MAX) return WF_ERR_INVALID;
  if (scratch_bytes < wf_beam_select_scratch_bytes(n_req, beams, vocab)) return WF_ERR_CAPACITY;
  SelectParams p = {};
  p.logits = d_logits, p.ld = ld, p.scores = d_scores, p.suppress = d_suppress;
  p.n_req = n_req, p.W = beams, p.V = vocab, p.eos = eos < 0 ? -2 : eos;
  const SelectPlan plan = select_plan(rows, vocab, dtype == WF_F32);
  p.tiles = plan.tiles, p.segments = plan.segments, p.groups = plan.groups;
  p.token = d_token, p.parent = d_parent, p.score = d_score, p.fin_parent = d_fin_parent, p.fin_score = d_fin_score;
  p.sum = static_cast<unsigned long long *>(d_scratch);
  p.max = reinterpret_cast<float *>(p.sum + rows * p.segments);
  p.group_max = p.max + rows * p.segments;
  const void *fn, *join;
  if (!(dtype == WF_F32 ? select_ready<float>(&fn, &join) : dtype == WF_F16 ? select_ready<__half>(&fn, &join) : select_ready<__nv_bfloat16>(&fn, &join)))
    return WF_ERR_CUDA;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  void *args[] = {&p};
  const long long grid = (rows + kSelWarps - 1) / kSelWarps * p.segments;
  if (grid > INT32_MAX) return WF_ERR_UNSUPPORTED;
  if (launch_pdl(fn, static_cast<unsigned>(grid), kSelThreads, 0, args, s) != cudaSuccess ||
      launch_pdl(join, n_req, beams * 64, static_cast<size_t>(beams) * kJoinAhead * 512, args, s) != cudaSuccess)
    return WF_ERR_CUDA;
  return WF_OK;
}

}  // extern "C"
