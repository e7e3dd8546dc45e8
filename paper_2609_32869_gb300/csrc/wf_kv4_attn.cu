// Attention over the paged 4-bit cache (softmax(scale q K^T) V).
//
// A cached value is s (c - 8) + z with one (s, z) per position and group of 64
// dims, so both products split into exact small-integer tensor products and
// rank-one terms in fp32:
//   q . k_j        = sum_g  s_jg (q_g . (c_jg - 8)) + z_jg sum(q_g)
//   sum_j p_j v_jg = sum_j (p_j s_jg) (c_jg - 8)    + sum_j p_j z_jg
// The codes enter mma.sync (m16n8k16, fp32 sums) as exact small integers in the
// cache's 16-bit type.
//   bf16: a nibble in the low mantissa bits of 128.  Keys keep the 128 + 8, which
//   go into z (a few dozen units on a sum of 64 products in fp32); p_j s_jg is
//   rounded to bf16, whose range holds any scale.
//   fp16: a nibble where it lies, in bits 0 to 3 under 1024 or 4 to 7 under 64, so
//   that a word of eight takes one shift.  Odd nibbles of keys keep their 64 + 8,
//   which the sums start without.  p_j s_jg is rounded to fp16 after a scaling by
//   a power of two (kept per group, moved with the scales) that holds every s of
//   32 positions between 1 and 2^7: 11 bits of weights down to 2^-14 of the
//   running reference, and at most 2^-25 of its s off below.  Steps whose scales
//   span more than that, and steps with positions that are not seen, round to
//   the sum of two bf16, 16 bits of any size.
// (Keys and weights in fp16 for bf16 caches too, rows of queries scaled into its
// range: 96 requests x 9 rows took 78 us instead of 71, the row scaling and its
// registers costing more than the shifts.)
//
// The positions are the M side of both products (A operand: 16 positions of
// keys, then 16 dims of values), the query rows the N side in tiles of 8, so
// one dequantisation serves every query row of a key/value head.  K Q^T
// leaves lane (r, t) with positions r, r + 8 and rows 2t, 2t + 1; an 8x8
// transpose per tile turns the weights into the B operand of V^T P^T.
#include <climits>
#include <type_traits>

#include "wf_kv4.cuh"
#include "wf_paged_attn.cuh"

namespace wf {

constexpr int kAtTile = 64;  // positions of a warp's step

__device__ __forceinline__ uint32_t sub_f16x2(uint32_t u, uint32_t v) {
  const __half2 d = __hsub2(*reinterpret_cast<const __half2 *>(&u), *reinterpret_cast<const __half2 *>(&v));
  return *reinterpret_cast<const uint32_t *>(&d);
}
// Nibble I of each half of w as a pair of fp16 c - 8.
template <int I>
__device__ __forceinline__ uint32_t codes_f16(uint32_t w) {
  const uint32_t u = I < 2 ? w : w >> 8;
  return I % 2 ? sub_f16x2(and_or(u, 0x00f000f0u, 0x54005400u), 0x54805480u)   // 64 + c, 72
               : sub_f16x2(and_or(u, 0x000f000fu, 0x64006400u), 0x64086408u);  // 1024 + c, 1032
}
template <int I>
__device__ __forceinline__ uint32_t key_codes(uint32_t w, __half) {
  return I % 2 ? and_or(I < 2 ? w : w >> 8, 0x00f000f0u, 0x54005400u) : codes_f16<I>(w);
}
template <int I>
__device__ __forceinline__ uint32_t key_codes(uint32_t w, __nv_bfloat16) {
  return and_or(w >> (4 * I), 0x000f000fu, 0x43004300u);
}
template <int I>
__device__ __forceinline__ uint32_t codes_bf16(uint32_t w) {
  const uint32_t u = and_or(w >> (4 * I), 0x000f000fu, 0x43004300u), eight = 0x43084308u;  // 128 + c, 136
  const __nv_bfloat162 v = __hsub2(*reinterpret_cast<const __nv_bfloat162 *>(&u), *reinterpret_cast<const __nv_bfloat162 *>(&eight));
  return *reinterpret_cast<const uint32_t *>(&v);
}
template <int G, int NT>
struct AtShape {
  static constexpr int kRows = NT * 8;
  static constexpr int kStages = 2;
  static constexpr int kSub = 2;                          // tiles of 16 positions between two looks at the maximum
  static constexpr int kBlocks = G == 1 ? 6 - NT : 4 - NT;  // CTAs of an SM that the registers allow
  static constexpr int kStageBytes = 4 * G * kKv4Rec;  // 64 positions of a head
  static constexpr int kRingBytes = kAtWarps * kStages * kStageBytes;
  static constexpr int kMergeBytes = kAtWarps * kRows * (G * 64 + 4 + 2) * 4 + kRows * (G * 64 + 2) * 4;
  static constexpr int kBarOff = ((kRingBytes > kMergeBytes ? kRingBytes : kMergeBytes) + 15) / 16 * 16;
  static constexpr int kSmem = kBarOff + kAtWarps * kStages * 8;
};

// A unit is (sequence, key/value head, NT * 8 query rows).  Each warp takes
// steps of 64 positions of a unit through a ring of its own in shared memory
// (one bulk copy per record, an mbarrier per stage; no other warp is waited
// for) and keeps a running maximum, sum and weighted values.  A CTA's warps
// take a unit, or a chunk of one, in turns and join in order; up to 8 chunks
// join over a cluster, more by a second kernel.
//   96 sequences x 9 rows x 20 heads, 1500 positions, bf16: 70 us, 3.0 TB/s,
//     by instructions and their latencies (58% of the slots at 15 warps an SM;
//     half of the loop's instructions unpack nibbles) and a last, sixth-full
//     round of CTAs
//   80 sequences of 4 to 448 positions, 20 heads, bf16: 13.7 us, by the
//     instructions before and after the loop
//   6 sequences of 5000 to 65001 positions, 32 heads on 8, 128 wide, fp16: 38 us,
//     3.3 TB/s, likewise (52% of the slots at 9 warps an SM)
//   5 rows of one sequence, 1500 positions, 20 heads, bf16: 6 us, by the launch
//     and one chain of reads
// One wave of CTAs that go on to their next unit, its first records on their way
// while one is joined, took 77 and 15.8 us for the first two; warps with equal
// shares of all steps and a kernel that joins their pieces 84 and 22.
template <typename T, int G, int NT>
__global__ void __launch_bounds__(kAtThreads, AtShape<G, NT>::kBlocks) kv4_attention_kernel(const PagedAttnParams<Kv4Pool> p) {
  using X = Kv4Type<T>;
  using S = AtShape<G, NT>;
  constexpr int kRows = S::kRows, kStages = S::kStages, kSub = S::kSub;
  constexpr bool kF16 = std::is_same<T, __half>::value;
  extern __shared__ __align__(16) unsigned char smem[];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, r = lane >> 2, t = lane & 3;
  uint64_t *bars = reinterpret_cast<uint64_t *>(smem + S::kBarOff) + warp * kStages;
  unsigned char *ring = smem + warp * kStages * S::kStageBytes;
  if (lane == 0) {
    for (int i = 0; i < kStages; ++i) mbar_init(&bars[i], 1);
    fence_barrier_init();
  }
  __syncwarp();
  pdl_wait();
  pdl_launch_dependents();
  const int head = blockIdx.x % p.pool.heads, seq = blockIdx.x / p.pool.heads;
  const int row0 = blockIdx.z * kRows, rows = p.rps * p.group;  // rows of this key/value head: j * group + query head
  const int32_t *table = p.table + static_cast<long long>(seq) * p.table_stride;
  const int raw_len = p.len[seq], len = clamp_len(p, raw_len);
  if (raw_len != len && threadIdx.x == 0) set_error(p.err, raw_len < 0 ? WF_DEV_ERR_PAGE : WF_DEV_ERR_CAPACITY);
  // positions that any row of this unit sees, and this CTA's share of them
  const int seen = row_limit(p, min(row0 + kRows, rows) - 1, len);
  const int begin = blockIdx.y * p.chunk, end = begin + min(seen - begin, p.chunk);
  if (begin >= end && blockIdx.y > 0 && !p.cluster) return;

  // The ring: step i of this warp is positions begin + (warp + i kAtWarps) 64.
  // Lane 4 g + k < 4 G loads tile k of group g; a step is whole blocks, so its
  // place in a block never changes and its table entry moves by whole blocks.
  const int first = begin + warp * kAtTile;
  constexpr int stride = kAtWarps * kAtTile;
  const int steps = first < end ? (end - first + stride - 1) / stride : 0;
  const int my_pos = first + (lane & 3) * 16, table_step = stride >> p.pool.bs_shift;
  const int32_t *entry = table + (my_pos >> p.pool.bs_shift);
  const unsigned char *my_base = kv4_record(p.pool, 0, head, lane >> 2, (my_pos & (p.pool.bs - 1)) >> 4);
  // steps in which this lane's tile has positions to load
  const int my_steps = lane < 4 * G && my_pos < end ? (end - my_pos + stride - 1) / stride : 0;
  int next_block = my_steps > 0 ? *entry : -1;
  int to_issue = 0, issue_stage = 0;
  uint32_t there_bits = 0;  // 4 bits a stage: tiles that were loaded
  auto issue = [&]() {
    const bool mine = to_issue < my_steps, ok = mine && static_cast<uint32_t>(next_block) < static_cast<uint32_t>(p.pool.n_blocks);
    if (mine && !ok) set_error(p.err, WF_DEV_ERR_PAGE);
    const uint32_t oks = __ballot_sync(0xffffffffu, ok);
    there_bits = (there_bits & ~(15u << (4 * issue_stage))) | (oks & 15u) << (4 * issue_stage);
    if (lane == 0) mbar_arrive_expect_tx(&bars[issue_stage], __popc(oks) * kKv4Rec);
    __syncwarp();
    if (ok)
      bulk_load(ring + issue_stage * S::kStageBytes + lane * kKv4Rec, my_base + static_cast<long long>(next_block) * p.block_bytes, kKv4Rec,
                &bars[issue_stage]);
    ++to_issue;
    issue_stage = issue_stage + 1 == kStages ? 0 : issue_stage + 1;
    entry += table_step;
    next_block = to_issue < my_steps ? *entry : -1;
  };
#pragma unroll 1
  for (int i = 0; i < kStages && i < steps; ++i) issue();

  // Queries as B operands.  Of rows 2t and 2t + 1: sums over a group and what the
  // odd codes' bias adds (fp16).
  uint32_t qb[NT][G][4][2];
  float2 qs[NT][G], start[NT][G];
  int lim[NT][2], least = INT_MAX;
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    const int row = row0 + n * 8 + r;
    const int j = p.row_of(row), h = head * p.group + row - j * p.group;
#pragma unroll
    for (int g = 0; g < G; ++g) {
      uint32_t w[8] = {};
      if (row < rows) {
        const uint4 *src = reinterpret_cast<const uint4 *>(static_cast<const T *>(p.q) + (static_cast<long long>(seq) * p.rps + j) * p.q_stride +
                                                           h * (G * 64) + g * 64 + t * 16);
        const uint4 a = src[0], b = src[1];
        w[0] = a.x, w[1] = a.y, w[2] = a.z, w[3] = a.w, w[4] = b.x, w[5] = b.y, w[6] = b.z, w[7] = b.w;
      }
      float even = 0.f, odd = 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) even += X::lo(w[i]), odd += X::hi(w[i]);
      even += odd, odd *= -72.f;
#pragma unroll
      for (int off = 1; off < 4; off <<= 1) {
        even += __shfl_xor_sync(0xffffffffu, even, off);
        if (kF16) odd += __shfl_xor_sync(0xffffffffu, odd, off);
      }
      qs[n][g] = make_float2(__shfl_sync(0xffffffffu, even, t * 8), __shfl_sync(0xffffffffu, even, t * 8 + 4));
      start[n][g] = make_float2(0.f, 0.f);
      if (kF16) start[n][g] = make_float2(__shfl_sync(0xffffffffu, odd, t * 8), __shfl_sync(0xffffffffu, odd, t * 8 + 4));
#pragma unroll
      for (int k = 0; k < 4; ++k)
#pragma unroll
        for (int u = 0; u < 2; ++u)  // dims 16t + 8u + k and + 4: the pairing of a code word's nibbles
          qb[n][g][k][u] = __byte_perm(w[u * 4 + k / 2], w[u * 4 + 2 + k / 2], k % 2 ? 0x7632 : 0x5410);
    }
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int rr = row0 + n * 8 + 2 * t + e;
      // a row past the last sees what the last does: its results are not written
      lim[n][e] = row_limit(p, min(rr, rows - 1), len);
      least = min(least, lim[n][e]);
    }
  }
  least = min(least, __shfl_xor_sync(0xffffffffu, least, 1));
  least = min(least, __shfl_xor_sync(0xffffffffu, least, 2));

  float o[NT][G][4][4] = {};  // of group g in units of 1 / so[g]
  float so[G];                // 1; fp16: a power of two that holds s so of the values in [1, 2^7]
#pragma unroll
  for (int g = 0; g < G; ++g) so[g] = 1.f;
  const float c = p.scale * 1.4426950408889634f;  // base-2 softmax
  float2 zacc[NT][G] = {}, l[NT], m[NT];  // of rows 2t and 2t + 1; m: the power of two that the weights are relative to
#pragma unroll
  for (int n = 0; n < NT; ++n) l[n] = make_float2(0.f, 0.f), m[n] = make_float2(-INFINITY, -INFINITY);

  // kSub tiles of 16 positions from k0; `edge`: some are not seen by some row, or are not there.
  // False, with nothing added: their scales need the two terms that an edge's weights have.
  auto step = [&](const unsigned char *buf, int k0, uint32_t there, auto edge_c) {
    constexpr bool edge = decltype(edge_c)::value;
    float2 x[kSub][NT][2];  // [16 positions][rows][position r, r + 8] (row 2t, row 2t + 1)
    uint2 szv[kSub][G];
    float mx[NT][2];
    bool wide = false;  // fp16: some scales are too far apart for one power of two (0 is none of them)
#pragma unroll
    for (int n = 0; n < NT; ++n) mx[n][0] = mx[n][1] = -INFINITY;
#pragma unroll
    for (int g = 0; g < G; ++g) {
      uint2 w0[kSub], w1[kSub];
      float acc[kSub][NT][4];
#pragma unroll
      for (int i = 0; i < kSub; ++i) {
        const unsigned char *rg = buf + (g * 4 + i) * kKv4Rec;
        w0[i] = *reinterpret_cast<const uint2 *>(rg + r * 32 + t * 8);
        w1[i] = *reinterpret_cast<const uint2 *>(rg + (r + 8) * 32 + t * 8);
#pragma unroll
        for (int n = 0; n < NT; ++n) acc[i][n][0] = acc[i][n][2] = start[n][g].x, acc[i][n][1] = acc[i][n][3] = start[n][g].y;
      }
      // tile by tile within a step of 16 dims: the chains of sums interleave
#define WF_KSTEP(K)                                                                                              \
  _Pragma("unroll") for (int i = 0; i < kSub; ++i) {                                                             \
    const uint32_t a[4] = {key_codes<K>(w0[i].x, T()), key_codes<K>(w1[i].x, T()), key_codes<K>(w0[i].y, T()),                    \
                           key_codes<K>(w1[i].y, T())};                                                            \
    _Pragma("unroll") for (int n = 0; n < NT; ++n) mma16(acc[i][n], a, qb[n][g][K][0], qb[n][g][K][1], T());  \
  }
      WF_KSTEP(0) WF_KSTEP(1) WF_KSTEP(2) WF_KSTEP(3)
#undef WF_KSTEP
#pragma unroll
      for (int i = 0; i < kSub; ++i) {
        const uint4 sz = *reinterpret_cast<const uint4 *>(buf + (g * 4 + i) * kKv4Rec + kKv4ScaleOff + r * 16);
        const float s0 = X::lo(sz.x) * c, s1 = X::lo(sz.y) * c;
        float z0 = X::hi(sz.x) * c, z1 = X::hi(sz.y) * c;
        if (!kF16) z0 = fmaf(-136.f, s0, z0), z1 = fmaf(-136.f, s1, z1);
        szv[i][g] = make_uint2(sz.z, sz.w);
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          const float2 a = make_float2(fmaf(s0, acc[i][n][0], z0 * qs[n][g].x), fmaf(s0, acc[i][n][1], z0 * qs[n][g].y));
          const float2 b = make_float2(fmaf(s1, acc[i][n][2], z1 * qs[n][g].x), fmaf(s1, acc[i][n][3], z1 * qs[n][g].y));
          x[i][n][0] = g == 0 ? a : add2(x[i][n][0], a);
          x[i][n][1] = g == 0 ? b : add2(x[i][n][1], b);
        }
      }
    }
#pragma unroll
    for (int i = 0; i < kSub; ++i) {
      const int pos = k0 + i * 16 + r;
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        if (edge) {
          const bool here = there >> i & 1;
          if (!here || pos >= lim[n][0]) x[i][n][0].x = -INFINITY;
          if (!here || pos >= lim[n][1]) x[i][n][0].y = -INFINITY;
          if (!here || pos + 8 >= lim[n][0]) x[i][n][1].x = -INFINITY;
          if (!here || pos + 8 >= lim[n][1]) x[i][n][1].y = -INFINITY;
        }
        mx[n][0] = max3(mx[n][0], x[i][n][0].x, x[i][n][1].x);
        mx[n][1] = max3(mx[n][1], x[i][n][0].y, x[i][n][1].y);
      }
    }
    // The reference of the weights moves only when some row's maximum passes
    // it by 2^8, that of the sums when a scale leaves its range (or is 0, which
    // changes nothing): the products stay below 2^15, which fp16 holds, and most
    // steps rescale nothing.
    constexpr float kLowS = 1.f, kHighS = 0x1p7f;
    bool moved = false;
    if (kF16 && !edge) {
#pragma unroll
      for (int g = 0; g < G; ++g) {
        const float a = X::lo(szv[0][g].x), b = X::lo(szv[0][g].y), e = X::lo(szv[1][g].x), f = X::lo(szv[1][g].y);
        moved |= fminf(fminf(a, b), fminf(e, f)) * so[g] < kLowS || fmaxf(max3(a, b, e), f) * so[g] > kHighS;
      }
    }
#pragma unroll
    for (int n = 0; n < NT; ++n) moved |= mx[n][0] > m[n].x + 8.f || mx[n][1] > m[n].y + 8.f;
    if (__any_sync(0xffffffffu, moved)) {
      float change[G];
#pragma unroll
      for (int g = 0; g < G; ++g) {
        change[g] = 1.f;
        if (!kF16 || edge) continue;
        float top = 0.f, low = INFINITY;  // the largest scale and the smallest above 0
#pragma unroll
        for (int i = 0; i < kSub; ++i)
#pragma unroll
          for (int u = 0; u < 2; ++u) {
            const float v = X::lo(u ? szv[i][g].y : szv[i][g].x);
            top = fmaxf(top, v);
            if (v > 0.f) low = fminf(low, v);
          }
        top = warp_max(top), low = -warp_max(-low);
        if (top > 0.f && (low * so[g] < kLowS || top * so[g] > kHighS)) {
          const float next_so = __uint_as_float((259u << 23) - (__float_as_uint(top) & 0x7f800000u));  // top in [2^5, 2^6)
          change[g] = next_so / so[g];                                                                 // (of powers of two)
          so[g] = next_so;
          wide |= low * next_so < kLowS;
        }
      }
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        float next[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          next[e] = e ? fmaxf(mx[n][1], m[n].y) : fmaxf(mx[n][0], m[n].x);
#pragma unroll
          for (int off = 4; off < 32; off <<= 1) next[e] = fmaxf(next[e], __shfl_xor_sync(0xffffffffu, next[e], off));
        }
        // nothing seen yet: sums are zero, whatever they are scaled by
        const float c0 = m[n].x == -INFINITY ? 0.f : ex2(m[n].x - next[0]), c1 = m[n].y == -INFINITY ? 0.f : ex2(m[n].y - next[1]);
        l[n].x *= c0, l[n].y *= c1;
#pragma unroll
        for (int g = 0; g < G; ++g) {
          zacc[n][g].x *= c0, zacc[n][g].y *= c1;
#pragma unroll
          for (int q = 0; q < 4; ++q)
            o[n][g][q][0] *= c0 * change[g], o[n][g][q][1] *= c1 * change[g], o[n][g][q][2] *= c0 * change[g], o[n][g][q][3] *= c1 * change[g];
        }
        m[n] = make_float2(next[0], next[1]);
      }
      if (kF16 && wide) return false;
    }
#pragma unroll
    for (int i = 0; i < kSub; ++i) {
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const float2 y = add2(x[i][n][u], make_float2(-m[n].x, -m[n].y));
          float2 w = make_float2(ex2(y.x), ex2(y.y));
          if (edge) {
            if (x[i][n][u].x == -INFINITY) w.x = 0.f;
            if (x[i][n][u].y == -INFINITY) w.y = 0.f;
          }
          x[i][n][u] = w;
          l[n] = add2(l[n], w);
        }
#pragma unroll
      for (int g = 0; g < G; ++g) {
        const uint4 v = *reinterpret_cast<const uint4 *>(buf + (g * 4 + i) * kKv4Rec + kKv4ValOff + lane * 16);
        if (kF16 && !edge) {
          uint32_t ph[NT][2];
#pragma unroll
          for (int u = 0; u < 2; ++u) {
            const uint32_t sz = u ? szv[i][g].y : szv[i][g].x;
            const float sv = X::lo(sz) * so[g], zv = X::hi(sz);
#pragma unroll
            for (int n = 0; n < NT; ++n) {
              ph[n][u] = transpose8x8(pack_f16(mul2(x[i][n][u], make_float2(sv, sv))));
              zacc[n][g] = fma2(x[i][n][u], make_float2(zv, zv), zacc[n][g]);
            }
          }
#define WF_VSTEP(Q)                                                                                           \
  {                                                                                                           \
    const uint32_t a[4] = {codes_f16<Q>(v.x), codes_f16<Q>(v.y), codes_f16<Q>(v.z), codes_f16<Q>(v.w)};       \
    _Pragma("unroll") for (int n = 0; n < NT; ++n) mma16(o[n][g][Q], a, ph[n][0], ph[n][1], __half());        \
  }
          WF_VSTEP(0) WF_VSTEP(1) WF_VSTEP(2) WF_VSTEP(3)
#undef WF_VSTEP
        } else {
          uint32_t ph[NT][2], pl[NT][2];
#pragma unroll
          for (int u = 0; u < 2; ++u) {
            const uint32_t sz = u ? szv[i][g].y : szv[i][g].x;
            const float sv = kF16 ? X::lo(sz) * so[g] : X::lo(sz), zv = X::hi(sz);
#pragma unroll
            for (int n = 0; n < NT; ++n) {
              const float2 w = x[i][n][u];
              float a = w.x * sv, b = w.y * sv;
              if (edge) {  // a weight of 0 stays 0 whatever the position holds
                a = w.x == 0.f ? 0.f : a, b = w.y == 0.f ? 0.f : b;
                zacc[n][g].x += w.x == 0.f ? 0.f : w.x * zv;
                zacc[n][g].y += w.y == 0.f ? 0.f : w.y * zv;
              } else {
                zacc[n][g].x = fmaf(w.x, zv, zacc[n][g].x);
                zacc[n][g].y = fmaf(w.y, zv, zacc[n][g].y);
              }
              const uint32_t h = pack_bf16(a, b);
              ph[n][u] = transpose8x8(h);
              if (kF16) pl[n][u] = transpose8x8(pack_bf16(a - __uint_as_float(h << 16), b - __uint_as_float(h & 0xffff0000u)));
            }
          }
#define WF_VSTEP(Q)                                                                                           \
  {                                                                                                           \
    const uint32_t a[4] = {codes_bf16<Q>(v.x), codes_bf16<Q>(v.y), codes_bf16<Q>(v.z), codes_bf16<Q>(v.w)};   \
    _Pragma("unroll") for (int n = 0; n < NT; ++n) {                                                          \
      mma16(o[n][g][Q], a, ph[n][0], ph[n][1], __nv_bfloat16());                                              \
      if (kF16) mma16(o[n][g][Q], a, pl[n][0], pl[n][1], __nv_bfloat16());                                    \
    }                                                                                                         \
  }
          WF_VSTEP(0) WF_VSTEP(1) WF_VSTEP(2) WF_VSTEP(3)
#undef WF_VSTEP
        }
      }
    }
    return true;
  };

  int stage = 0, k0 = first;
  uint32_t phase = 0;
#pragma unroll 1
  for (int i = 0; i < steps; ++i) {
    const bool landed = mbar_wait(&bars[stage], phase, p.err, kSpinLimitCycles);
    if (!__all_sync(0xffffffffu, landed)) {  // the copies in flight still have to land before the CTA ends
      for (int j = i; j < to_issue; ++j) mbar_drain(&bars[j % kStages], (j / kStages) & 1);
      break;
    }
    const uint32_t there = there_bits >> (4 * stage) & 15u;
    const unsigned char *buf = ring + stage * S::kStageBytes;
#pragma unroll 1
    for (int h = 0; h < 4; h += kSub) {
      const bool all = k0 + (h + kSub) * 16 <= least && there == 15u;
      if (!all || !step(buf + h * kKv4Rec, k0 + h * 16, there >> h, std::false_type()))
        step(buf + h * kKv4Rec, k0 + h * 16, there >> h, std::true_type());
    }
    __syncwarp();
    if (to_issue < steps) issue();
    k0 += stride;
    if (++stage == kStages) stage = 0, phase ^= 1;
  }

  // the warp's results: sums over its 8 position lanes, rows 2t and 2t + 1
#pragma unroll
  for (int n = 0; n < NT; ++n) {
#pragma unroll
    for (int off = 4; off < 32; off <<= 1) {
      l[n].x += __shfl_xor_sync(0xffffffffu, l[n].x, off), l[n].y += __shfl_xor_sync(0xffffffffu, l[n].y, off);
#pragma unroll
      for (int g = 0; g < G; ++g) {
        zacc[n][g].x += __shfl_xor_sync(0xffffffffu, zacc[n][g].x, off);
        zacc[n][g].y += __shfl_xor_sync(0xffffffffu, zacc[n][g].y, off);
      }
    }
  }
  __syncthreads();  // the ring is done with
  constexpr int kLd = kAtLd<G>;
  float *sm_m = reinterpret_cast<float *>(smem), *sm_l = sm_m + kAtWarps * kRows, *sm_o = sm_l + kAtWarps * kRows;
#pragma unroll
  for (int n = 0; n < NT; ++n) {
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int row = warp * kRows + n * 8 + 2 * t + e;
      if (r == 0) sm_m[row] = e ? m[n].y : m[n].x, sm_l[row] = e ? l[n].y : l[n].x;
#pragma unroll
      for (int g = 0; g < G; ++g)
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const float z = e ? zacc[n][g].y : zacc[n][g].x, os = 1.f / so[g];
          *reinterpret_cast<float4 *>(sm_o + row * kLd + g * 64 + r * 8 + u * 4) =
              make_float4(fmaf(o[n][g][0][e + 2 * u], os, z), fmaf(o[n][g][1][e + 2 * u], os, z), fmaf(o[n][g][2][e + 2 * u], os, z),
                          fmaf(o[n][g][3][e + 2 * u], os, z));
        }
    }
  }
  __syncthreads();
  paged_finish<T, G, NT>(p, sm_m, sm_l, sm_o, seen, row0, rows, head, seq);
}

}  // namespace wf

using namespace wf;

template <typename T, int G, int NT>
static cudaError_t launch(const PagedAttnParams<Kv4Pool> &p, cudaStream_t s) {
  static PerDevice ready;
  return paged_launch<T, G, NT>(reinterpret_cast<const void *>(kv4_attention_kernel<T, G, NT>), AtShape<G, NT>::kSmem, ready, p, s);
}

extern "C" {

size_t wf_kv4_attention_scratch_bytes(int32_t n_seq, int32_t rps, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim,
                                      int32_t max_len) {
  return paged_scratch_bytes(n_seq, rps, n_heads, n_kv_heads, head_dim, max_len);
}

wf_status wf_kv4_attention(const wf_kv4_pool *pool, int32_t layer, const void *d_q, int64_t q_stride, const int32_t *d_table,
                           int32_t table_stride, const int32_t *d_len, int32_t n_seq, int32_t rps, int32_t n_heads,
                           int32_t causal, float scale, int32_t max_len, void *d_out, int64_t out_stride, void *d_scratch,
                           size_t scratch_bytes, uint32_t *d_err, void *stream) {
  PagedAttnParams<Kv4Pool> p = {};
  wf_status st = kv4_pool_check(pool, layer, &p.pool, nullptr);
  if (st != WF_OK) return st;
  p.block_bytes = static_cast<uint32_t>(kv4_block_bytes(pool->block_size, pool->n_kv_heads, pool->head_dim));
  st = paged_args(*pool, d_q, q_stride, d_table, table_stride, d_len, n_seq, rps, n_heads, causal, scale, max_len, d_out, out_stride,
                  d_scratch, scratch_bytes, d_err, &p);
  if (st != WF_OK) return st;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  using B = __nv_bfloat16;
  const bool f16 = pool->dtype == WF_F16, wide = pool->head_dim == 128, two = p.tiles == 2;
  cudaError_t e;
  if (f16)
    e = wide ? (two ? launch<__half, 2, 2>(p, s) : launch<__half, 2, 1>(p, s)) : (two ? launch<__half, 1, 2>(p, s) : launch<__half, 1, 1>(p, s));
  else
    e = wide ? (two ? launch<B, 2, 2>(p, s) : launch<B, 2, 1>(p, s)) : (two ? launch<B, 1, 2>(p, s) : launch<B, 1, 1>(p, s));
  return e == cudaSuccess ? WF_OK : WF_ERR_CUDA;
}

}  // extern "C"
