// Attention over the paged 8-bit cache (softmax(scale q K^T) V).
//
// A cached value is c 2^e, c an e4m3 code and e shared by 16 positions of a
// head; fp16 holds every c, so both products run on mma.sync m16n8k16 in fp16
// with fp32 sums, and the powers of two stay outside:
//   x_j   = (q . c_j) 2^ek scale log2(e)
//   sum_j 2^x_j v_j = sum_j 2^(x_j + ev) c_j
// The weights are taken with their values' ev in the exponent, under a
// reference that follows the largest x + ev of a row: what fp16 loses is small
// beside the row's largest term, however far apart the scales are.  The sum of
// the 2^x alone takes each weight times 2^-ev (ev lies in -60 .. 36, so that a
// weight that counts there is above 2^-126 here).
//
// The positions are the M side of both products, the query rows the N side in
// tiles of 8, so one conversion of the codes serves every query row of a
// key/value head.  K Q^T leaves lane (r, t) with positions r, r + 8 and rows
// 2t, 2t + 1; an 8x8 transpose per tile turns the weights into the B operand of V^T P^T.
#include <climits>
#include <type_traits>

#include "wf_kv8.cuh"
#include "wf_paged_attn.cuh"

namespace wf {

template <int G, int NT>
struct K8Shape {
  static constexpr int kRows = NT * 8;
  static constexpr int kStages = G == 1 ? 3 : 2;  // (of 64 dims a third one takes 69.4 us to 68.0)
  static constexpr int kSub = 2;  // records of a warp's step
  static constexpr int kTile = kSub * 16;
  static constexpr int kBlocks = G == 1 ? 6 - NT : 4 - NT;  // CTAs of an SM that the registers allow
  static constexpr int kRec = G * kKv8Group + 16;
  static constexpr int kStageBytes = kSub * kRec;
  static constexpr int kRingBytes = kAtWarps * kStages * kStageBytes;
  static constexpr int kMergeBytes = kAtWarps * kRows * (kAtLd<G> + 2) * 4 + kRows * (G * 64 + 2) * 4;
  static constexpr int kBarOff = ((kRingBytes > kMergeBytes ? kRingBytes : kMergeBytes) + 15) / 16 * 16;
  static constexpr int kSmem = kBarOff + kAtWarps * kStages * 8;
};

// fp16 weights are up to 2^15, 2^8 over what the reference stands for.
constexpr float kK8Bias = 7.f;

// Bytes of w that are NaN, as 0x80 of each.
__device__ __forceinline__ uint32_t nan_bytes(uint32_t w) { return ((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u; }
// 1 in fp16 for each of the two low bytes that has its top bit set.
__device__ __forceinline__ uint32_t flags_f16(uint32_t two) { return (two & 0x80 ? 0x3c00u : 0u) | (two & 0x8000 ? 0x3c000000u : 0u); }

// A unit is (sequence, key/value head, NT * 8 query rows).  Each warp takes
// steps of 32 positions of a unit through a ring of its own in shared memory
// (one bulk copy per record, an mbarrier per stage; no other warp is waited for)
// and keeps a running reference, sum and weighted values.
//   96 sequences x 9 rows x 20 heads, 1500 positions, bf16: 68 us, 5.5 TB/s, by HBM
//     and 3.2 rounds of CTAs that take four (cut in two, the halves joined over a
//     cluster, 92; at three CTAs an SM 74, at five, which spill at length, 110; at four 8 bytes)
//   6 sequences of 5000 to 65001 positions, 32 heads on 8, 128 wide, fp16: 39.6 us,
//     5.7 TB/s, by HBM; of that the join 2 us (with a third stage, two CTAs an SM, 47)
//   5 rows of one sequence, 1500 positions, 20 heads, bf16: 5.9 us, by the launch
//     and one chain of reads
template <typename T, int G, int NT>
__global__ void __launch_bounds__(kAtThreads, K8Shape<G, NT>::kBlocks) kv8_attention_kernel(const PagedAttnParams<Kv8Pool> p) {
  using X = Type16<T>;
  using S = K8Shape<G, NT>;
  constexpr int kRows = S::kRows, kStages = S::kStages, kSub = S::kSub, kTile = S::kTile;
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

  // The ring: step i of this warp is positions begin + (warp + i kAtWarps) 32.
  // Lane k < 2 loads record k; four steps are whole blocks, so its place in a
  // block never changes and its table entry moves by whole blocks.
  const int first = begin + warp * kTile;
  constexpr int stride = kAtWarps * kTile;
  const int steps = first < end ? (end - first + stride - 1) / stride : 0;
  const int my_pos = first + (lane & (kSub - 1)) * 16, table_step = stride >> p.pool.bs_shift;
  const int32_t *entry = table + (my_pos >> p.pool.bs_shift);
  const unsigned char *my_base = kv8_record(p.pool, 0, head, (my_pos & (p.pool.bs - 1)) >> 4);
  // steps in which this lane's record has positions to load
  const int my_steps = lane < kSub && my_pos < end ? (end - my_pos + stride - 1) / stride : 0;
  int next_block = my_steps > 0 ? *entry : -1;
  int to_issue = 0, issue_stage = 0;
  uint32_t there_bits = 0;  // kSub bits a stage: records that were loaded
  auto issue = [&]() {
    const bool mine = to_issue < my_steps, ok = mine && static_cast<uint32_t>(next_block) < static_cast<uint32_t>(p.pool.n_blocks);
    if (mine && !ok) set_error(p.err, WF_DEV_ERR_PAGE);
    const uint32_t oks = __ballot_sync(0xffffffffu, ok);
    there_bits = (there_bits & ~(((1u << kSub) - 1) << (kSub * issue_stage))) | oks << (kSub * issue_stage);
    if (lane == 0) mbar_arrive_expect_tx(&bars[issue_stage], __popc(oks) * S::kRec);
    __syncwarp();
    if (ok)
      bulk_load(ring + issue_stage * S::kStageBytes + lane * S::kRec, my_base + static_cast<long long>(next_block) * p.block_bytes, S::kRec,
                &bars[issue_stage]);
    ++to_issue;
    issue_stage = issue_stage + 1 == kStages ? 0 : issue_stage + 1;
    entry += table_step;
    next_block = to_issue < my_steps ? *entry : -1;
  };
#pragma unroll 1
  for (int i = 0; i < kStages && i < steps; ++i) issue();

  // Queries as B operands in fp16: bf16 rows under a power of two that brings
  // their largest to 2^13; `unscale` of rows 2t and 2t + 1 takes it back.
  const float c = p.scale * 1.4426950408889634f;  // base-2 softmax
  uint32_t qb[NT][G][4][2];
  float2 unscale[NT];
  int lim[NT][2], least = INT_MAX;
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    const int row = row0 + n * 8 + r;
    const int j = p.row_of(row), h = head * p.group + row - j * p.group;
    uint32_t w[G][8] = {};
    if (row < rows) {
#pragma unroll
      for (int g = 0; g < G; ++g) {
        const uint4 *src = reinterpret_cast<const uint4 *>(static_cast<const T *>(p.q) + (static_cast<long long>(seq) * p.rps + j) * p.q_stride +
                                                           h * (G * 64) + g * 64 + t * 16);
        const uint4 a = src[0], b = src[1];
        w[g][0] = a.x, w[g][1] = a.y, w[g][2] = a.z, w[g][3] = a.w, w[g][4] = b.x, w[g][5] = b.y, w[g][6] = b.z, w[g][7] = b.w;
      }
    }
    float back = c;
    if (!kF16) {
      uint32_t most = 0;
#pragma unroll
      for (int g = 0; g < G; ++g)
#pragma unroll
        for (int i = 0; i < 8; ++i) most = max(most, max(w[g][i] & 0x7fff, w[g][i] >> 16 & 0x7fff));
      most = max(most, __shfl_xor_sync(0xffffffffu, most, 1));
      most = max(most, __shfl_xor_sync(0xffffffffu, most, 2));
      const int e = max(static_cast<int>(most >> 7) - 127, -100) - 13;
      const float f = two_to(min(-e, 113));
      back = c * two_to(e);
#pragma unroll
      for (int g = 0; g < G; ++g)
#pragma unroll
        for (int i = 0; i < 8; ++i) w[g][i] = pack_f16(make_float2(X::lo(w[g][i]) * f, X::hi(w[g][i]) * f));
    }
    unscale[n] = make_float2(__shfl_sync(0xffffffffu, back, t * 8), __shfl_sync(0xffffffffu, back, t * 8 + 4));
#pragma unroll
    for (int g = 0; g < G; ++g)
#pragma unroll
      for (int k = 0; k < 4; ++k) qb[n][g][k][0] = w[g][2 * k], qb[n][g][k][1] = w[g][2 * k + 1];
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

  float o[NT][G][4][4] = {};
  float2 l[NT], m[NT];  // of rows 2t and 2t + 1; m: the power of two that the weights are relative to
#pragma unroll
  for (int n = 0; n < NT; ++n) l[n] = make_float2(0.f, 0.f), m[n] = make_float2(-INFINITY, -INFINITY);

  // kSub records of 16 positions from k0; `edge`: some are not seen by some row, or are not there.
  auto step = [&](const unsigned char *buf, int k0, uint32_t there, auto edge_c) {
    constexpr bool edge = decltype(edge_c)::value;
    float2 x[kSub][NT][2];  // [record][rows][position r, r + 8] (row 2t, row 2t + 1)
    float without[kSub];    // 2^-ev
    float acc[kSub][NT][4] = {};
#pragma unroll
    for (int g = 0; g < G; ++g) {
      uint4 a0[kSub], a1[kSub];
#pragma unroll
      for (int i = 0; i < kSub; ++i) {
        a0[i] = *reinterpret_cast<const uint4 *>(buf + i * S::kRec + g * kKv8Group + r * 64 + t * 16);
        a1[i] = *reinterpret_cast<const uint4 *>(buf + i * S::kRec + g * kKv8Group + (r + 8) * 64 + t * 16);
      }
      // record by record within a step of 16 dims: the chains of sums interleave
#pragma unroll
      for (int k = 0; k < 4; ++k)
#pragma unroll
        for (int i = 0; i < kSub; ++i) {
          const uint32_t u = k == 0 ? a0[i].x : k == 1 ? a0[i].y : k == 2 ? a0[i].z : a0[i].w;
          const uint32_t v = k == 0 ? a1[i].x : k == 1 ? a1[i].y : k == 2 ? a1[i].z : a1[i].w;
          const uint32_t a[4] = {codes_to_f16(u), codes_to_f16(v), codes_to_f16(u >> 16), codes_to_f16(v >> 16)};
#pragma unroll
          for (int n = 0; n < NT; ++n) mma16(acc[i][n], a, qb[n][g][k][0], qb[n][g][k][1], __half());
        }
    }
    float mx[NT][2];
#pragma unroll
    for (int n = 0; n < NT; ++n) mx[n][0] = mx[n][1] = -INFINITY;
#pragma unroll
    for (int i = 0; i < kSub; ++i) {
      const float2 sc = *reinterpret_cast<const float2 *>(buf + i * S::kRec + G * kKv8Group);
      const int ev = min(max((__float_as_int(sc.y) >> 23 & 255) - 127, kKv8Low), kKv8High);  // (what is not there may be anything)
      const float fe = static_cast<float>(ev);
      without[i] = two_to(-ev);
      const int pos = k0 + i * 16 + r;
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        const float2 f = mul2(unscale[n], make_float2(sc.x, sc.x));
        x[i][n][0] = fma2(make_float2(acc[i][n][0], acc[i][n][1]), f, make_float2(fe, fe));
        x[i][n][1] = fma2(make_float2(acc[i][n][2], acc[i][n][3]), f, make_float2(fe, fe));
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
    // The reference moves only when some row's maximum passes it by 2^8: most steps rescale nothing.
    bool moved = false;
#pragma unroll
    for (int n = 0; n < NT; ++n) moved |= mx[n][0] > m[n].x + 8.f || mx[n][1] > m[n].y + 8.f;
    if (__any_sync(0xffffffffu, moved)) {
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
        for (int g = 0; g < G; ++g)
#pragma unroll
          for (int q = 0; q < 4; ++q) o[n][g][q][0] *= c0, o[n][g][q][1] *= c1, o[n][g][q][2] *= c0, o[n][g][q][3] *= c1;
        m[n] = make_float2(next[0], next[1]);
      }
    }
#pragma unroll
    for (int i = 0; i < kSub; ++i) {
      uint32_t ph[NT][2], sees[NT][2];
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const float2 y = add2(x[i][n][u], make_float2(kK8Bias - m[n].x, kK8Bias - m[n].y));
          float2 w = make_float2(ex2(y.x), ex2(y.y));
          if (edge) {
            const bool sx = x[i][n][u].x != -INFINITY, sy = x[i][n][u].y != -INFINITY;
            if (!sx) w.x = 0.f;
            if (!sy) w.y = 0.f;
            sees[n][u] = (sx ? 0x3c00u : 0u) | (sy ? 0x3c000000u : 0u);
          }
          l[n] = fma2(w, make_float2(without[i], without[i]), l[n]);
          ph[n][u] = transpose8x8(pack_f16(w));
        }
#pragma unroll
      for (int g = 0; g < G; ++g)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const uint4 v4 = *reinterpret_cast<const uint4 *>(buf + i * S::kRec + g * kKv8Group + 1024 + h * 512 + lane * 16);
          uint32_t v[4] = {v4.x, v4.y, v4.z, v4.w};
          if (edge) {
            // codes of NaN among values that some row does not see: zeros in the
            // product, which a weight of 0 would not make of them, and counted
            // apart for the rows that see them
            uint32_t bad[4];
#pragma unroll
            for (int q = 0; q < 4; ++q) bad[q] = nan_bytes(v[q]);
            if (__any_sync(0xffffffffu, (bad[0] | bad[1] | bad[2] | bad[3]) != 0)) {
#pragma unroll
              for (int q = 0; q < 4; ++q) v[q] &= ~((bad[q] >> 7) * 255u);
#pragma unroll
              for (int q = 0; q < 2; ++q) {
                const uint32_t a[4] = {flags_f16(bad[2 * q]), flags_f16(bad[2 * q] >> 16), flags_f16(bad[2 * q + 1]), flags_f16(bad[2 * q + 1] >> 16)};
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                  float count[4] = {};
                  mma16(count, a, transpose8x8(sees[n][0]), transpose8x8(sees[n][1]), __half());
#pragma unroll
                  for (int e = 0; e < 4; ++e)
                    if (count[e] > 0.f) o[n][g][2 * h + q][e] = NAN;
                }
              }
            }
          }
#pragma unroll
          for (int q = 0; q < 2; ++q) {
            const uint32_t a[4] = {codes_to_f16(v[2 * q]), codes_to_f16(v[2 * q] >> 16), codes_to_f16(v[2 * q + 1]), codes_to_f16(v[2 * q + 1] >> 16)};
#pragma unroll
            for (int n = 0; n < NT; ++n) mma16(o[n][g][2 * h + q], a, ph[n][0], ph[n][1], __half());
          }
        }
    }
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
    const uint32_t there = there_bits >> (kSub * stage) & ((1u << kSub) - 1);
    const unsigned char *buf = ring + stage * S::kStageBytes;
    if (k0 + kTile <= least && there == (1u << kSub) - 1)
      step(buf, k0, there, std::false_type());
    else
      step(buf, k0, there, std::true_type());
    __syncwarp();
    if (to_issue < steps) issue();
    k0 += stride;
    if (++stage == kStages) stage = 0, phase ^= 1;
  }

  // the warp's results: sums over its 8 position lanes, rows 2t and 2t + 1
#pragma unroll
  for (int n = 0; n < NT; ++n)
#pragma unroll
    for (int off = 4; off < 32; off <<= 1)
      l[n].x += __shfl_xor_sync(0xffffffffu, l[n].x, off), l[n].y += __shfl_xor_sync(0xffffffffu, l[n].y, off);
  __syncthreads();  // the ring is done with
  float *sm_m = reinterpret_cast<float *>(smem), *sm_l = sm_m + kAtWarps * kRows, *sm_o = sm_l + kAtWarps * kRows;
#pragma unroll
  for (int n = 0; n < NT; ++n)
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int row = warp * kRows + n * 8 + 2 * t + e;
      if (r == 0) sm_m[row] = e ? m[n].y : m[n].x, sm_l[row] = e ? l[n].y : l[n].x;
#pragma unroll
      for (int g = 0; g < G; ++g)
#pragma unroll
        for (int u = 0; u < 2; ++u)
          *reinterpret_cast<float4 *>(sm_o + row * kAtLd<G> + g * 64 + r * 8 + u * 4) =
              make_float4(o[n][g][0][e + 2 * u], o[n][g][1][e + 2 * u], o[n][g][2][e + 2 * u], o[n][g][3][e + 2 * u]);
    }
  __syncthreads();
  paged_finish<T, G, NT>(p, sm_m, sm_l, sm_o, seen, row0, rows, head, seq);
}

}  // namespace wf

using namespace wf;

template <typename T, int G, int NT>
static cudaError_t launch(const PagedAttnParams<Kv8Pool> &p, cudaStream_t s) {
  static PerDevice ready;
  return paged_launch<T, G, NT>(reinterpret_cast<const void *>(kv8_attention_kernel<T, G, NT>), K8Shape<G, NT>::kSmem, ready, p, s);
}

extern "C" {

size_t wf_kv8_attention_scratch_bytes(int32_t n_seq, int32_t rps, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim, int32_t max_len) {
  return paged_scratch_bytes(n_seq, rps, n_heads, n_kv_heads, head_dim, max_len);
}

wf_status wf_kv8_attention(const wf_kv8_pool *pool, int32_t layer, const void *d_q, int64_t q_stride, const int32_t *d_table,
                           int32_t table_stride, const int32_t *d_len, int32_t n_seq, int32_t rps, int32_t n_heads, int32_t causal,
                           float scale, int32_t max_len, void *d_out, int64_t out_stride, void *d_scratch, size_t scratch_bytes,
                           uint32_t *d_err, void *stream) {
  PagedAttnParams<Kv8Pool> p = {};
  wf_status st = kv8_pool_check(pool, layer, &p.pool);
  if (st != WF_OK) return st;
  const size_t block = kv8_block_bytes(pool->block_size, pool->n_kv_heads, pool->head_dim);
  p.block_bytes = static_cast<uint32_t>(block);  // at most 2^26
  st = paged_args(*pool, d_q, q_stride, d_table, table_stride, d_len, n_seq, rps, n_heads, causal, scale, max_len, d_out, out_stride, d_scratch,
                  scratch_bytes, d_err, &p);
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
