// Beam search's selection over beams and vocabulary.
//
// Within a row the order of the scores, score + ((logit - max) - log(sum)), is
// the order of the logits,
// so the vocabulary is read once: each CTA takes a chunk of a row, keeps the
// chunk's running maximum and sum of exponentials and its 2 beams largest
// logits.  A second kernel joins the chunks of a request's rows, turns the
// survivors into scores and ranks them.
#include <algorithm>

#include "wf_device.cuh"
#include "wf_kv4.cuh"

namespace wf {

struct SelectParams {
  const void *logits;
  long long ld;
  const float *scores;
  const uint8_t *suppress;
  int n_req, W, V, eos, chunks;
  int32_t *token, *parent;
  float *score;
  int32_t *fin_parent;
  float *fin_score;
  // scratch: per (row, chunk) the maximum and the sum, and 2W keys
  unsigned long long *keys;  // [rows][chunks][2W]
  unsigned long long *sum;   // [rows][chunks] in units of 2^-40
  float *max;                // [rows][chunks]
};
constexpr int kSelThreads = 256;
constexpr int kSelPer = 32;                       // logits of a thread
constexpr int kSelChunk = kSelThreads * kSelPer;  // of a CTA
constexpr int kSelKeep = 512;                     // candidates of a chunk that are held

// (value descending, index ascending) as one descending unsigned key; 0 is
// below every key of a value above -inf.
__device__ __forceinline__ uint32_t order_bits(float v) {
  const uint32_t b = __float_as_uint(v + 0.f);  // -0 as 0
  return (b & 0x80000000u) ? ~b : (b | 0x80000000u);
}
__device__ __forceinline__ unsigned long long order_key(float v, uint32_t idx) {
  return static_cast<unsigned long long>(order_bits(v)) << 32 | (0xffffffffu - idx);
}
__device__ __forceinline__ float key_value(unsigned long long k) {
  const uint32_t o = static_cast<uint32_t>(k >> 32);
  return __uint_as_float((o & 0x80000000u) ? (o & 0x7fffffffu) : ~o);
}
__device__ __forceinline__ uint32_t key_index(unsigned long long k) { return 0xffffffffu - static_cast<uint32_t>(k); }
// The largest key of a warp: its upper word, then the largest lower word under it (if there are several).
__device__ __forceinline__ unsigned long long warp_max(unsigned long long k) {
  const uint32_t hi = __reduce_max_sync(0xffffffffu, static_cast<uint32_t>(k >> 32));
  const unsigned have = __ballot_sync(0xffffffffu, static_cast<uint32_t>(k >> 32) == hi);
  const uint32_t lo = (have & (have - 1)) ? __reduce_max_sync(0xffffffffu, static_cast<uint32_t>(k >> 32) == hi ? static_cast<uint32_t>(k) : 0u)
                                          : __shfl_sync(0xffffffffu, static_cast<uint32_t>(k), __ffs(have) - 1);
  return static_cast<unsigned long long>(hi) << 32 | lo;
}
// Sorts a warp's values (keys), largest in lane 0: a bitonic network.
template <typename K>
__device__ __forceinline__ K warp_sort(K v, int lane) {
#pragma unroll
  for (int size = 2; size <= 32; size <<= 1)
#pragma unroll
    for (int off = size >> 1; off; off >>= 1) {
      const K w = __shfl_xor_sync(0xffffffffu, v, off);
      const bool keep_max = ((lane & off) == 0) == ((lane & size) == 0);
      v = keep_max ? (w > v ? w : v) : (w > v ? v : w);
    }
  return v;
}

template <typename T>
struct Logits;
template <>
struct Logits<float> {
  static constexpr int kVec = 4;
  static __device__ __forceinline__ void unpack(uint4 v, float *x) {
    x[0] = __uint_as_float(v.x), x[1] = __uint_as_float(v.y), x[2] = __uint_as_float(v.z), x[3] = __uint_as_float(v.w);
  }
  static __device__ __forceinline__ float one(float v) { return v; }
};
template <typename T>
struct Logits16 {
  static constexpr int kVec = 8;
  static __device__ __forceinline__ void unpack(uint4 v, float *x) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) x[2 * i] = Kv4Type<T>::lo(w[i]), x[2 * i + 1] = Kv4Type<T>::hi(w[i]);
  }
};
template <>
struct Logits<__nv_bfloat16> : Logits16<__nv_bfloat16> {
  static __device__ __forceinline__ float one(__nv_bfloat16 v) { return __bfloat162float(v); }
};
template <>
struct Logits<__half> : Logits16<__half> {
  static __device__ __forceinline__ float one(__half v) { return __half2float(v); }
};

// One CTA: 8192 logits of a row, 32 a thread in registers, by 16-byte loads
// whatever the row's alignment (a chunk starts up to 15 bytes before a
// multiple of 8192 logits; what lies outside the row is -inf).
//
// The k = 2 beams largest: of the 32 maxima over 256 logits each, the k-th is
// a value that at least k logits reach and few more do; those are collected
// and ranked by one warp.  Where many reach it (equal logits), k rounds over
// the CTA pick them one by one.  The sum of exponentials adds 32 terms a
// thread in fp32, the threads' in fixed point (2^-40), so it has no order.
// A NaN is never the larger of a comparison, which keeps it out of the maxima
// and the candidates; only the sum has to look for it.
template <typename T>
__global__ void __launch_bounds__(kSelThreads, 4) beam_chunk_kernel(const SelectParams p) {
  using L = Logits<T>;
  constexpr int kVec = L::kVec, kVecs = kSelPer / kVec;
  __shared__ float sm_g[32], sm_floor;
  __shared__ unsigned long long sm_sum[kSelThreads / 32], sm_k[2][kSelThreads / 32], keep[kSelKeep];
  __shared__ int kept;
  __shared__ __align__(16) unsigned char mask[kSelChunk + 32];
  const int chunk = blockIdx.x, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, K = 2 * p.W;
  const long long row = blockIdx.y + static_cast<long long>(blockIdx.z) * 65535;
  if (row >= static_cast<long long>(p.n_req) * p.W) return;
  if (tid == 0) kept = 0;
  pdl_wait();
  pdl_launch_dependents();
  const T *src = static_cast<const T *>(p.logits) + row * p.ld;
  const int skew = static_cast<int>((reinterpret_cast<uintptr_t>(src) & 15) / sizeof(T));
  const int first = chunk * kSelChunk - skew;  // a multiple of 16 bytes from address 0
  const auto id_of = [&](int i) { return first + ((i / kVec) * kSelThreads + tid) * kVec + i % kVec; };
  float x[kSelPer];
  const bool inside = first >= 0 && first + kSelChunk <= p.V;
  if (inside) {
    const uint4 *at = reinterpret_cast<const uint4 *>(src + first) + tid;
    uint4 raw[kVecs];
#pragma unroll
    for (int v = 0; v < kVecs; ++v) raw[v] = at[v * kSelThreads];
#pragma unroll
    for (int v = 0; v < kVecs; ++v) L::unpack(raw[v], x + v * kVec);
  } else {
#pragma unroll
    for (int i = 0; i < kSelPer; ++i) {
      const int id = id_of(i);
      const float v = L::one(src[min(max(id, 0), p.V - 1)]);
      x[i] = id >= 0 && id < p.V ? v : -INFINITY;
    }
  }
  // a logit again, from memory, for the rare paths that would keep registers from the others
  const auto again = [&](int i) {
    const int id = id_of(i);
    if (id < 0 || id >= p.V || (p.suppress && p.suppress[id])) return -INFINITY;
    return L::one(src[id]);
  };
  if (p.suppress) {  // its bytes by 16, from the multiple of 16 before the chunk; read back at the skew between the two
    const int lead = static_cast<int>((reinterpret_cast<uintptr_t>(p.suppress) + first) & 15);
    for (int i = tid; i < kSelChunk / 16 + 1; i += kSelThreads) {
      const int id = first - lead + i * 16;
      if (id >= 0 && id + 16 <= p.V) {
        *reinterpret_cast<uint4 *>(mask + i * 16) = *reinterpret_cast<const uint4 *>(p.suppress + id);
      } else {
        for (int e = 0; e < 16; ++e) mask[i * 16 + e] = id + e >= 0 && id + e < p.V ? p.suppress[id + e] : 0;
      }
    }
    __syncthreads();
#pragma unroll
    for (int v = 0; v < kSelPer / 4; ++v) {
      const int at = lead + ((v * 4 / kVec) * kSelThreads + tid) * kVec + v * 4 % kVec;
      const uint32_t *word = reinterpret_cast<const uint32_t *>(mask) + (at >> 2);
      const uint32_t w = __funnelshift_r(word[0], word[1], (at & 3) * 8);
      if (!w) continue;
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (w & (0xffu << (8 * e))) x[v * 4 + e] = -INFINITY;
    }
  }
  float top = -INFINITY;
#pragma unroll
  for (int i = 0; i < kSelPer; ++i) top = fmaxf(top, x[i]);
  float g = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
  g = fmaxf(g, __shfl_xor_sync(0xffffffffu, g, 2));
  g = fmaxf(g, __shfl_xor_sync(0xffffffffu, g, 4));
  if ((lane & 7) == 0) sm_g[warp * 4 + (lane >> 3)] = g;
  __syncthreads();
  g = sm_g[lane];
  const float m = key_value(static_cast<unsigned long long>(__reduce_max_sync(0xffffffffu, order_bits(g))) << 32);
  if (warp == 0) {
    const float kth = __shfl_sync(0xffffffffu, warp_sort(g, lane), K - 1);
    if (lane == 0) sm_floor = kth;
  }
  float2 part2 = {0.f, 0.f};
#pragma unroll
  for (int i = 0; i < kSelPer; i += 2) {  // the difference first: its rounding does not grow with the logits
    const float2 y = mul2(add2(make_float2(x[i], x[i + 1]), make_float2(-m, -m)), make_float2(1.4426950408889634f, 1.4426950408889634f));
    part2 = add2(part2, make_float2(ex2(y.x), ex2(y.y)));
  }
  float part = part2.x + part2.y;
  if (part != part) {  // a NaN; or all -inf, or a +inf: the join knows those rows by their maximum
    part = 0.f;
#pragma unroll 1
    for (int i = 0; i < kSelPer; ++i) {
      const float e = ex2((again(i) - m) * 1.4426950408889634f);
      part += e == e ? e : 0.f;
    }
  }
  {
    const unsigned long long fixed = static_cast<unsigned long long>(part * 1099511627776.f);  // at most 2^45
    const unsigned lo = __reduce_add_sync(0xffffffffu, static_cast<unsigned>(fixed & 0x3fffff));
    const unsigned hi = __reduce_add_sync(0xffffffffu, static_cast<unsigned>(fixed >> 22));
    if (lane == 0) sm_sum[warp] = (static_cast<unsigned long long>(hi) << 22) + lo;
  }
  __syncthreads();
  const float floor_v = sm_floor;
  if (top >= floor_v && top > -INFINITY) {
    uint32_t hits = 0;
#pragma unroll
    for (int i = 0; i < kSelPer; ++i) hits |= x[i] >= floor_v ? 1u << i : 0u;
    for (; hits; hits &= hits - 1) {
      const int i = __ffs(hits) - 1;
      const float v = again(i);
      if (!(v > -INFINITY)) continue;
      const int at = atomicAdd(&kept, 1);
      if (at < kSelKeep) keep[at] = order_key(v, id_of(i));
    }
  }
  __syncthreads();
  const int n = kept;
  unsigned long long *out = p.keys + (row * p.chunks + chunk) * K;
  if (n <= kSelKeep) {
    if (warp == 0) {  // each key's rank is the number of larger ones
      for (int i = lane; i < n; i += 32) {
        const unsigned long long k = keep[i];
        int rank = 0;
#pragma unroll 8
        for (int j = 0; j < n; ++j) rank += keep[j] > k;
        if (rank < K) out[rank] = k;
      }
      if (lane >= n && lane < K) out[lane] = 0;
    }
  } else {
    unsigned long long below = ~0ull;
    for (int k = 0; k < K; ++k) {
      unsigned long long best = 0;
#pragma unroll 1
      for (int i = 0; i < kSelPer; ++i) {
        const float v = again(i);
        const unsigned long long q = v > -INFINITY ? order_key(v, id_of(i)) : 0;
        if (q < below && q > best) best = q;
      }
      best = warp_max(best);
      if (lane == 0) sm_k[k & 1][warp] = best;
      __syncthreads();
      below = 0;
      for (int w = 0; w < kSelThreads / 32; ++w) below = sm_k[k & 1][w] > below ? sm_k[k & 1][w] : below;
      if (tid == 0) out[k] = below;
    }
  }
  if (tid == 0) {
    unsigned long long total = 0;
    for (int w = 0; w < kSelThreads / 32; ++w) total += sm_sum[w];
    p.sum[row * p.chunks + chunk] = total;
    p.max[row * p.chunks + chunk] = m;
  }
}

// One CTA per request, one warp per beam and one more, which takes the rows'
// logarithms in 64 bits while the others pick their rows' best keys.
constexpr int kJoinStage = 40 << 10;  // shared memory for the rows' keys; past it they are read where they lie
__global__ void __launch_bounds__((WF_MAX_BEAMS + 1) * 32) beam_join_kernel(const SelectParams p, int staged) {
  const int W = p.W, K = 2 * W, req = blockIdx.x, lane = threadIdx.x & 31, beam = threadIdx.x >> 5, C = p.chunks;
  __shared__ unsigned long long best_key[WF_MAX_BEAMS * 2 * WF_MAX_BEAMS], cand[WF_MAX_BEAMS * 2 * WF_MAX_BEAMS];
  __shared__ unsigned long long ranked[2 * WF_MAX_BEAMS], row_sum[WF_MAX_BEAMS];
  __shared__ float row_max[WF_MAX_BEAMS], row_log[WF_MAX_BEAMS];
  extern __shared__ unsigned long long dyn[];
  unsigned char *next = reinterpret_cast<unsigned char *>(dyn + (staged ? W * C * K : 0));  // [W][C] keys taken of each list
  pdl_wait();
  pdl_launch_dependents();
  const long long row0 = static_cast<long long>(req) * W;
  const unsigned long long *keys = p.keys + row0 * C * K;
  if (staged)
    for (int i = threadIdx.x; i < W * C * K; i += blockDim.x) dyn[i] = keys[i];
  if (C > 32)
    for (int i = threadIdx.x; i < W * C; i += blockDim.x) next[i] = 0;
  if (threadIdx.x < K) ranked[threadIdx.x] = 0;
  if (beam < W) {  // the row's maximum and sum
    const float *cm = p.max + (row0 + beam) * C;
    const unsigned long long *cs = p.sum + (row0 + beam) * C;
    const float m0 = lane < C ? cm[lane] : -INFINITY;
    const unsigned long long s0 = lane < C ? cs[lane] : 0;
    float m = m0;
    for (int c = lane + 32; c < C; c += 32) m = fmaxf(m, cm[c]);
    m = key_value(static_cast<unsigned long long>(__reduce_max_sync(0xffffffffu, order_bits(m))) << 32);
    const auto scaled = [&](unsigned long long v, float at) -> unsigned long long {
      const float f = expf(at - m);
      return f == f ? static_cast<unsigned long long>(static_cast<double>(v) * static_cast<double>(f)) : 0;
    };
    unsigned long long s = scaled(s0, m0);
    for (int c = lane + 32; c < C; c += 32) s += scaled(cs[c], cm[c]);
#pragma unroll
    for (int off = 16; off; off >>= 1) s += __shfl_xor_sync(0xffffffffu, s, off);
    if (lane == 0) row_max[beam] = m, row_sum[beam] = s;
  }
  __syncthreads();
  if (beam == W) {
    if (lane < W) row_log[lane] = static_cast<float>(log(static_cast<double>(row_sum[lane]) * 0x1p-40));
  } else {
    // each lane offers the largest key that its sorted lists have left
    const unsigned long long *mine = (staged ? dyn : keys) + static_cast<size_t>(beam) * C * K;
    if (C <= 32) {  // one list a lane, whose next key is at hand
      const unsigned long long *list = mine + lane * K;
      unsigned long long head = lane < C ? list[0] : 0, after = lane < C ? list[1] : 0;
      int at = 1;
      for (int k = 0; k < K; ++k) {
        const unsigned long long best = warp_max(head);
        if (lane == 0) best_key[beam * K + k] = best;
        if (best && best == head) {
          head = after;
          after = ++at < K ? list[at] : 0;
        }
      }
    } else {
      unsigned long long head = 0;
      int from = -1;
      const auto look = [&]() {
        head = 0;
        for (int c = lane; c < C; c += 32) {
          const int at = next[beam * C + c];
          const unsigned long long v = at < K ? mine[c * K + at] : 0;
          if (v > head) head = v, from = c;
        }
      };
      look();
      for (int k = 0; k < K; ++k) {
        const unsigned long long best = warp_max(head);
        if (lane == 0) best_key[beam * K + k] = best;
        if (best && best == head) {
          ++next[beam * C + from];
          look();
        }
      }
    }
  }
  __syncthreads();
  for (int i = threadIdx.x; i < W * K; i += blockDim.x) {
    const int w = i / K;
    const unsigned long long k = best_key[i];
    // a row whose maximum is infinite has no scores but NaN, which is no candidate
    const float m = row_max[w], total = k && m < INFINITY ? p.scores[row0 + w] + ((key_value(k) - m) - row_log[w]) : -INFINITY;
    cand[i] = total > -INFINITY ? order_key(total, i) : 0;
  }
  __syncthreads();
  for (int i = threadIdx.x; i < W * K; i += blockDim.x) {
    const unsigned long long k = cand[i];
    int rank = 0;
#pragma unroll 10
    for (int j = 0; j < W * K; ++j) rank += cand[j] > k;
    if (k && rank < K) ranked[rank] = k;
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

// 15 bytes of skew may push a row's end into another chunk.
static int select_chunks(int V) { return (V + 7 + kSelChunk - 1) / kSelChunk; }
constexpr int kSelMaxVocab = 1 << 22;  // the join keeps a byte for each of a request's chunks in shared memory

extern "C" {

size_t wf_beam_select_scratch_bytes(int32_t n_req, int32_t beams, int32_t vocab) {
  if (n_req <= 0 || beams <= 0 || beams > WF_MAX_BEAMS || vocab < 2 * beams || vocab > kSelMaxVocab) return 0;
  return static_cast<size_t>(n_req) * beams * select_chunks(vocab) * (2 * beams * 8 + 16);
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
  p.n_req = n_req, p.W = beams, p.V = vocab, p.eos = eos < 0 ? -2 : eos, p.chunks = select_chunks(vocab);
  p.token = d_token, p.parent = d_parent, p.score = d_score, p.fin_parent = d_fin_parent, p.fin_score = d_fin_score;
  p.keys = static_cast<unsigned long long *>(d_scratch);
  p.sum = reinterpret_cast<unsigned long long *>(p.keys + rows * p.chunks * 2 * beams);
  p.max = reinterpret_cast<float *>(p.sum + rows * p.chunks);
  const void *fn = dtype == WF_F32 ? reinterpret_cast<const void *>(beam_chunk_kernel<float>)
                   : dtype == WF_F16 ? reinterpret_cast<const void *>(beam_chunk_kernel<__half>)
                                     : reinterpret_cast<const void *>(beam_chunk_kernel<__nv_bfloat16>);
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const size_t lists = static_cast<size_t>(beams) * p.chunks;
  int staged = lists * 2 * beams * 8 <= kJoinStage;
  void *args[] = {&p}, *join_args[] = {&p, &staged};
  const dim3 grid(p.chunks, static_cast<unsigned>(std::min<long long>(rows, 65535)), static_cast<unsigned>((rows + 65534) / 65535));
  if (launch_pdl(fn, grid, kSelThreads, 0, args, s) != cudaSuccess ||
      launch_pdl(reinterpret_cast<const void *>(beam_join_kernel), n_req, (beams + 1) * 32, lists + (staged ? lists * 2 * beams * 8 : 0),
                 join_args, s) != cudaSuccess)
    return WF_ERR_CUDA;
  return WF_OK;
}

}  // extern "C"
