// Attention of whole prompts, packed one after another (softmax(scale q K^T) V).
//
// A tile is 128 rows of one sequence and key/value head: a row is a (token,
// query head of the group) pair, heads innermost, so that one block of 128 keys
// serves every head of the group whatever its size.  A CTA has up to two tiles
// that share their key blocks.  Both products run on tcgen05 with fp32 sums in
// TMEM: S = Q K^T from shared memory, O += P V with P in TMEM, over the
// columns that its S was read from.  Four warps a tile turn S into P, a thread a
// row: no shuffles, and O is rescaled only when a row's maximum has risen by
// more than 2^8 over the reference that its weights are relative to.
#include <cuda.h>
#include <cudaTypedefs.h>

#include <algorithm>
#include <climits>
#include <cmath>
#include <mutex>

#include "wf_device.cuh"
#include "wf_ops.cuh"

namespace wf {

constexpr int kPtKeys = 128;     // keys of a block
constexpr int kPtThreads = 384;  // four warps a tile, one for the products, one for the copies, two that look V over
constexpr int kPtMma = 8, kPtLoad = 9, kPtScrub = 10;  // warps

struct PromptParams {
  void *out;
  float *lse;
  long long out_stride;
  const int32_t *q_start, *k_start;
  int n_seq, n_q, n_k, max_k, n_heads, heads, group, causal;  // heads: of keys and values
  int tokens, tiles;  // tokens of a tile, tiles of a CTA
  float scale;
  float *part_o;    // [split][row][head][dim] where the keys are cut up
  float2 *part_ml;  // [split][row][head] (reference, sum)
  uint32_t *err;
};

template <int D>
struct PtShape {
  static constexpr int kHalf = 16384;            // 128 rows of 64 dims
  static constexpr int kTile = kHalf * D / 64;   // queries, keys or values
  static constexpr int kStages = D == 64 ? 6 : 4;
  static constexpr int kMarkOff = 2 * kTile + kStages * kTile;  // [3][D] first position of a value that is not finite
  static constexpr int kBarOff = kMarkOff + 3 * D * 4;
  static constexpr int kBars = 2 + 4 * kStages + 2 + 2 + 2 + 1;
  static constexpr int kSmem = 1024 + kBarOff + kBars * 8 + 64;
  static constexpr uint32_t kCols = 512;
};

// What a CTA works on.
struct PtWork {
  int seq, q0, rows, k0, keys;  // the sequence: first query row, their number, first key, their number
  int token;                    // the first tile's first token
  int first, last;              // key blocks of this CTA
};

// Positions that the token at index j of the sequence sees.
__device__ __forceinline__ int pt_limit(const PtWork &w, int causal, int j) {
  return causal ? min(max(w.keys - (w.rows - 1 - j), 0), w.keys) : w.keys;
}

__device__ __forceinline__ void tma_load_4d(void *dst, const CUtensorMap *m, int x, int y, int z, int u, uint64_t *bar) {
  asm volatile("cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];" ::"r"(
                   smem_u32(dst)),
               "l"(reinterpret_cast<uint64_t>(m)), "r"(x), "r"(y), "r"(z), "r"(u), "r"(smem_u32(bar))
               : "memory");
}

// Descriptor of the values as the second operand of P V: 128-byte swizzled rows
// of 64 dims, a row a key; dims (the operand's rows) are contiguous, the next
// 64 of them `kHalf` bytes on, the next eight keys 1024.
__device__ __forceinline__ uint64_t pt_desc_v(uint32_t addr) {
  uint64_t d = 0;
  d |= static_cast<uint64_t>((addr & 0x3FFFF) >> 4);
  d |= static_cast<uint64_t>(16384 >> 4) << 16;
  d |= static_cast<uint64_t>(1024 >> 4) << 32;
  d |= static_cast<uint64_t>(1) << 46;
  d |= static_cast<uint64_t>(2) << 61;
  return d;
}
template <typename T>
__host__ __device__ constexpr uint32_t pt_idesc(int N, bool b_rows_contiguous) {
  const uint32_t type = std::is_same<T, __nv_bfloat16>::value ? 1u : 0u;
  return (1u << 4) | (type << 7) | (type << 10) | (static_cast<uint32_t>(b_rows_contiguous) << 16) | (static_cast<uint32_t>(N >> 3) << 17) |
         (8u << 24);
}
// D (+)= A B with A in TMEM.
__device__ __forceinline__ void umma_ta(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d),
      "r"(a), "l"(b), "r"(idesc), "r"(accumulate)
      : "memory");
}
// 32 columns of the warp's lanes, without the wait.
__device__ __forceinline__ void tmem_ld32(uint32_t at, float (&v)[32]) {
  uint32_t *r = reinterpret_cast<uint32_t *>(v);
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,"
      "%26,%27,%28,%29,%30,%31}, [%32];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]),
        "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]),
        "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]),
        "=r"(r[31])
      : "r"(at)
      : "memory");
}
__device__ __forceinline__ void tmem_ld_wait() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void tmem_st(uint32_t at, const uint32_t (&r)[N]) {
  static_assert(N == 16 || N == 32, "");
  if constexpr (N == 16) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(at), "r"(r[0]), "r"(r[1]),
        "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]),
        "r"(r[14]), "r"(r[15])
        : "memory");
  } else {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,"
        "%25,%26,%27,%28,%29,%30,%31,%32};" ::"r"(at),
        "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]),
        "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]),
        "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31])
        : "memory");
  }
}

// The sequence and first token of work item `item` (a warp; every lane gets it).
// Items number each sequence's groups of `per` tokens, the last group first.
// False: there is no such item.
__device__ __forceinline__ bool pt_find(const PromptParams &p, int item, int lane, PtWork &w) {
  const int per = p.tokens * p.tiles;
  int before = 0;
  for (int base = 0; base < p.n_seq; base += 32) {
    const int i = base + lane;
    int a = 0, b = 0;
    bool bad = false;
    if (i < p.n_seq) {
      const int ra = p.q_start[i], rb = p.q_start[i + 1];
      a = min(max(ra, 0), p.n_q), b = min(max(rb, a), p.n_q);
      bad = a != ra || b != rb;
    }
    if (bad) set_error(p.err, WF_DEV_ERR_PAGE);
    const int groups = (b - a + per - 1) / per;
    int sum = groups;
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
      const int v = __shfl_up_sync(0xffffffffu, sum, off);
      if (lane >= off) sum += v;
    }
    const uint32_t past = __ballot_sync(0xffffffffu, before + sum > item);
    if (past) {
      const int src = __ffs(past) - 1;
      w.seq = base + src;
      w.q0 = __shfl_sync(0xffffffffu, a, src);
      w.rows = __shfl_sync(0xffffffffu, b, src) - w.q0;
      const int end = __shfl_sync(0xffffffffu, before + sum, src);
      w.token = (end - 1 - item) * per;
      const int rk0 = p.k_start[w.seq], rk1 = p.k_start[w.seq + 1];
      w.k0 = min(max(rk0, 0), p.n_k);
      const int k1 = min(max(rk1, w.k0), p.n_k);
      w.keys = min(k1 - w.k0, p.max_k);
      if (lane == 0 && (w.k0 != rk0 || k1 != rk1)) set_error(p.err, WF_DEV_ERR_PAGE);
      if (lane == 0 && k1 - w.k0 > p.max_k) set_error(p.err, WF_DEV_ERR_CAPACITY);
      return true;
    }
    before += __shfl_sync(0xffffffffu, sum, 31);
  }
  return false;
}

template <typename T>
struct PtType;
template <>
struct PtType<__nv_bfloat16> {
  static constexpr uint32_t kInf = 0x7f80;
  static constexpr float kBias = 0.f;
};
template <>
struct PtType<__half> {
  static constexpr uint32_t kInf = 0x7c00;
  static constexpr float kBias = 7.f;  // weights up to 2^15 in fp16, all 11 bits down to 2^-21 of the row's largest
};

template <typename T, int D>
__global__ void __launch_bounds__(kPtThreads, 1)
    prompt_attention_kernel(const __grid_constant__ CUtensorMap mq, const __grid_constant__ CUtensorMap mk, const __grid_constant__ CUtensorMap mv,
                            const PromptParams p) {
  using X = Type16<T>;
  using S = PtShape<D>;
  constexpr int kStages = S::kStages;
  extern __shared__ uint8_t smem_raw[];
  uint8_t *smem = smem_raw + ((1024 - (smem_u32(smem_raw) & 1023)) & 1023);
  uint8_t *sq = smem, *skv = smem + 2 * S::kTile;
  int *mark = reinterpret_cast<int *>(smem + S::kMarkOff);
  uint64_t *q_full = reinterpret_cast<uint64_t *>(smem + S::kBarOff);
  uint64_t *full = q_full + 2, *empty = full + kStages, *s_full = empty + kStages, *p_full = s_full + 2, *pv_done = p_full + 2;
  uint64_t *look = pv_done + 2, *clean = look + kStages, *done = clean + kStages;
  uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(done + 1);
  int *has_work = reinterpret_cast<int *>(tmem_slot + 1);
  volatile int *marked = has_work + 1;
  PtWork *shared_work = reinterpret_cast<PtWork *>(has_work + 2);

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  pdl_wait();
  pdl_launch_dependents();
  const int head = blockIdx.x % p.heads;
  if (warp == 0) {
    PtWork w = {};
    const bool any = pt_find(p, blockIdx.x / p.heads, lane, w);
    if (any) {
      // key blocks that any row of this CTA sees, and this split's share of them
      const int last_token = min(w.token + p.tokens * p.tiles, w.rows) - 1;
      const int blocks = (pt_limit(w, p.causal, last_token) + kPtKeys - 1) / kPtKeys;
      const int share = (blocks + gridDim.y - 1) / gridDim.y;
      w.first = min(static_cast<int>(blockIdx.y) * share, blocks), w.last = min(w.first + share, blocks);
    }
    if (lane == 0) *shared_work = w, *has_work = any, *marked = 0;
  }
  if (threadIdx.x == 32) {
    for (int i = 0; i < 2; ++i) mbar_init(&q_full[i], 1), mbar_init(&s_full[i], 1), mbar_init(&p_full[i], 128), mbar_init(&pv_done[i], 1);
    for (int i = 0; i < kStages; ++i) mbar_init(&full[i], 1), mbar_init(&empty[i], 1), mbar_init(&look[i], 1), mbar_init(&clean[i], 64);
    mbar_init(done, 1);
    fence_barrier_init();
    fence_proxy_async();
  }
  for (int i = threadIdx.x; i < 3 * D; i += kPtThreads) mark[i] = INT_MAX;
  if (warp == kPtMma) tmem_alloc(tmem_slot, S::kCols);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  const PtWork w = *shared_work;
  // tile i: its tokens and the blocks that its rows see of this CTA's
  const int tokens[2] = {*has_work ? min(p.tokens, w.rows - w.token) : 0,
                         *has_work && p.tiles > 1 ? min(max(w.rows - w.token - p.tokens, 0), p.tokens) : 0};
  int ends[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int seen = tokens[i] ? pt_limit(w, p.causal, w.token + i * p.tokens + tokens[i] - 1) : 0;
    ends[i] = max(min((seen + kPtKeys - 1) / kPtKeys, w.last), w.first);
  }
  const int end = max(ends[0], ends[1]);
  // blocks from here on hold positions that some row does not see
  const int edge = *has_work ? pt_limit(w, p.causal, w.token) / kPtKeys : 0;

  if (warp == kPtLoad) {
    if (lane == 0 && w.first < end) {
      tma_prefetch_desc(&mq), tma_prefetch_desc(&mk), tma_prefetch_desc(&mv);
      const uint32_t q_bytes = static_cast<uint32_t>(p.group * p.tokens) * D * 2;
      const auto load_q = [&](int i) {
        mbar_arrive_expect_tx(&q_full[i], q_bytes);
        for (int c = 0; c < D / 64; ++c)
          tma_load_4d(sq + i * S::kTile + c * S::kHalf, &mq, c * 64, 0, head, w.q0 + w.token + i * p.tokens, &q_full[i]);
      };
      if (ends[0] > w.first) load_q(0);
      int n = 0;  // loads so far
      for (int j = w.first; j < end; ++j) {
        bool ok = true;
        for (int kv = 0; kv < 2 && ok; ++kv, ++n) {
          const int st = n % kStages;
          if (n >= kStages) ok = mbar_wait(&empty[st], ((n / kStages) - 1) & 1, p.err, kSpinLimitCycles);
          if (!ok) break;
          mbar_arrive_expect_tx(&full[st], S::kTile);
          for (int c = 0; c < D / 64; ++c)
            tma_load_3d(skv + st * S::kTile + c * S::kHalf, kv ? &mv : &mk, c * 64, head, w.k0 + j * kPtKeys, &full[st]);
          // The stage's earlier copies have landed: only now is the parity of its barrier one to wait for.
          if (kv && j >= edge) mbar_arrive_cta(&look[st]);
          if (n == 0 && ends[1] > w.first) load_q(1);
        }
        if (!ok) break;
      }
      // a later wait gave up, here or in another warp: the copies still have to land before the CTA ends
      for (int i = 0; i < 2; ++i)
        if (ends[i] > w.first) mbar_drain(&q_full[i], 0);
      for (int i = max(0, n - kStages); i < n; ++i) mbar_drain(&full[i % kStages], (i / kStages) & 1);
    }
  } else if (warp == kPtMma) {
    if (lane == 0 && w.first < end) {
      constexpr uint32_t kIdS = pt_idesc<T>(kPtKeys, false), kIdO = pt_idesc<T>(D, true);
      const uint64_t dq = umma_desc_sw128(smem_u32(sq)), dk = umma_desc_sw128(smem_u32(skv)), dv = pt_desc_v(smem_u32(skv));
      const auto scores = [&](int i, int st) {
#pragma unroll
        for (int k = 0; k < D / 16; ++k) {
          const uint32_t off = (k / 4 * S::kHalf + k % 4 * 32) >> 4;
          umma_bf16(tmem + i * 128, dq + ((i * S::kTile) >> 4) + off, dk + ((st * S::kTile) >> 4) + off, kIdS, k > 0);
        }
        umma_commit(&s_full[i]);
      };
      bool ok = mbar_wait(&full[0], 0, p.err, kSpinLimitCycles);
      for (int i = 0; i < 2 && ok; ++i) {
        if (ends[i] <= w.first) continue;
        ok = mbar_wait(&q_full[i], 0, p.err, kSpinLimitCycles);
        tc_fence_after();
        if (ok) scores(i, 0);
      }
      umma_commit(&empty[0]);
      for (int j = w.first; j < end && ok; ++j) {
        const int n = 2 * (j - w.first), sv = (n + 1) % kStages, sk = (n + 2) % kStages;
        const uint32_t par = (j - w.first) & 1;
        ok = mbar_wait(&full[sv], ((n + 1) / kStages) & 1, p.err, kSpinLimitCycles);
        if (ok && j >= edge) ok = mbar_wait(&clean[sv], (j - max(edge, w.first)) / (kStages / 2) & 1, p.err, kSpinLimitCycles);
        if (ok && j + 1 < end) ok = mbar_wait(&full[sk], ((n + 2) / kStages) & 1, p.err, kSpinLimitCycles);
        for (int i = 0; i < 2 && ok; ++i) {
          if (j >= ends[i]) continue;
          ok = mbar_wait(&p_full[i], par, p.err, kSpinLimitCycles);
          tc_fence_after();
          if (!ok) break;
#pragma unroll
          for (int k = 0; k < kPtKeys / 16; ++k)
            umma_ta(tmem + 256 + i * D, tmem + i * 128 + k * 8, dv + ((sv * S::kTile + k * 2048) >> 4), kIdO, j > w.first || k > 0);
          umma_commit(&pv_done[i]);
          // P's columns are read before the next scores, issued behind, are written
          if (j + 1 < ends[i]) scores(i, sk);
        }
        umma_commit(&empty[sv]);
        if (j + 1 < end) umma_commit(&empty[sk]);
      }
      umma_commit(done);
      mbar_drain(done, 0);
    }
  } else if (warp >= kPtScrub) {
    // Values of positions that some row does not see: zero past the sequence's
    // end, and where they are not finite, which a weight of 0 would not hide;
    // the rows that see those take them from `mark`.
    for (int j = max(edge, w.first); j < end; ++j) {
      const int n = 2 * (j - w.first) + 1, st = n % kStages;
      if (!__all_sync(0xffffffffu, mbar_wait(&look[st], (j - max(edge, w.first)) / (kStages / 2) & 1, p.err, kSpinLimitCycles) &&
                                       mbar_wait(&full[st], (n / kStages) & 1, p.err, kSpinLimitCycles)))
        break;
      const int held = w.keys - j * kPtKeys;
      for (int c = threadIdx.x - kPtScrub * 32; c < S::kTile / 16; c += 64) {
        uint4 *at = reinterpret_cast<uint4 *>(skv + st * S::kTile + c * 16);
        const int row = c / 8 % 128;
        if (row >= held) {
          *at = make_uint4(0, 0, 0, 0);
          continue;
        }
        const uint4 v = *at;
        const uint32_t m = 0x7fff7fffu;
        const uint32_t most = __vmaxu2(__vmaxu2(v.x & m, v.y & m), __vmaxu2(v.z & m, v.w & m));
        if (max(most & 0xffff, most >> 16) < PtType<T>::kInf) continue;
        uint16_t *e = reinterpret_cast<uint16_t *>(at);
        const int dim = c / 1024 * 64 + ((c & 7) ^ (row & 7)) * 8;
        for (int i = 0; i < 8; ++i) {
          const uint32_t u = e[i] & 0x7fff;
          if (u < PtType<T>::kInf) continue;
          atomicMin(&mark[(u > PtType<T>::kInf ? 0 : e[i] >> 15 ? 2 : 1) * D + dim + i], j * kPtKeys + row);
          e[i] = 0;
          *marked = 1;
        }
      }
      fence_proxy_async();
      mbar_arrive_cta(&clean[st]);
    }
  } else {
    const int i = warp >> 2, row = (warp & 3) * 32 + lane;
    const uint32_t lanes = static_cast<uint32_t>((warp & 3) * 32) << 16;
    const uint32_t ts = tmem + i * 128 + lanes, to = tmem + 256 + i * D + lanes;
    const int token = row / p.group, h = head * p.group + row % p.group, index = w.token + i * p.tokens + token;
    const bool live = token < tokens[i];
    const int limit = live ? pt_limit(w, p.causal, index) : 0;
    // the least of the tile's limits: blocks below it need no mask
    const int least = tokens[i] ? pt_limit(w, p.causal, w.token + i * p.tokens) : 0;
    const float c = p.scale * 1.4426950408889634f;
    float ref = -INFINITY, l = 0.f;
    bool ok = true;
    for (int j = w.first; j < ends[i]; ++j) {
      const uint32_t par = (j - w.first) & 1;
      ok = __all_sync(0xffffffffu, mbar_wait(&s_full[i], par, p.err, kSpinLimitCycles));
      if (!ok) break;
      tc_fence_after();
      float s[4][32];
#pragma unroll
      for (int q = 0; q < 4; ++q) tmem_ld32(ts + q * 32, s[q]);
      tmem_ld_wait();
      if ((j + 1) * kPtKeys > least) {
        const int seen = limit - j * kPtKeys;
#pragma unroll
        for (int q = 0; q < 4; ++q)
#pragma unroll
          for (int e = 0; e < 32; ++e)
            if (q * 32 + e >= seen) s[q][e] = -INFINITY;
      }
      float mx[4];
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        mx[q] = s[q][0];
#pragma unroll
        for (int e = 1; e < 31; e += 2) mx[q] = max3(mx[q], s[q][e], s[q][e + 1]);
        mx[q] = fmaxf(mx[q], s[q][31]);
      }
      const float top = fmaxf(max3(mx[0], mx[1], mx[2]), mx[3]);
      if (j == w.first) {
        ref = top;
      } else if (__any_sync(0xffffffffu, (top - ref) * c > 8.f)) {
        const float next = fmaxf(top, ref);
        const float keep = ref == -INFINITY ? 0.f : ex2((ref - next) * c);
        ref = next;
        l *= keep;
        ok = __all_sync(0xffffffffu, mbar_wait(&pv_done[i], par ^ 1, p.err, kSpinLimitCycles));
        if (!ok) break;
        tc_fence_after();
#pragma unroll
        for (int q = 0; q < D / 16; ++q) {
          float o[16];
          tmem_ld16(to + q * 16, o);
#pragma unroll
          for (int e = 0; e < 16; ++e) o[e] *= keep;
          tmem_st16(to + q * 16, o);
        }
      }
      const float base = ref == -INFINITY ? 0.f : PtType<T>::kBias - ref * c;
      float2 sum = make_float2(0.f, 0.f);
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        uint32_t packed[16];
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const float2 y = fma2(make_float2(s[q][2 * e], s[q][2 * e + 1]), make_float2(c, c), make_float2(base, base));
          const float2 x = make_float2(ex2(y.x), ex2(y.y));
          sum = add2(sum, x);
          packed[e] = X::pack(x.x, x.y);
        }
        tmem_st(ts + q * 16, packed);
      }
      l += sum.x + sum.y;
      tmem_st_wait();
      tc_fence_before();
      mbar_arrive_cta(&p_full[i]);
    }
    if (ok && ends[i] > w.first) ok = __all_sync(0xffffffffu, mbar_wait(&pv_done[i], (ends[i] - 1 - w.first) & 1, p.err, kSpinLimitCycles));
    tc_fence_after();
    const bool whole = gridDim.y == 1;
    const long long at = (static_cast<long long>(w.q0 + index)) * p.n_heads + h;
    const float inv = !whole ? 1.f : l == 0.f ? 0.f : 1.f / l;
    const bool fix = *marked;
    if (tokens[i] && ok) {
#pragma unroll
      for (int q = 0; q < D / 32; ++q) {
        float o[32];
        if (ends[i] > w.first) {
          tmem_ld32(to + q * 32, o);
          tmem_ld_wait();
        } else {
#pragma unroll
          for (int e = 0; e < 32; ++e) o[e] = 0.f;
        }
        if (!live) continue;
#pragma unroll
        for (int e = 0; e < 32; ++e) o[e] = l == 0.f ? 0.f : o[e] * inv;
        if (fix) {
#pragma unroll
          for (int e = 0; e < 32; ++e) {
            const bool nan = mark[q * 32 + e] < limit, up = mark[D + q * 32 + e] < limit, down = mark[2 * D + q * 32 + e] < limit;
            if (nan || up || down) o[e] = nan || (up && down) ? NAN : up ? INFINITY : -INFINITY;
          }
        }
        if (whole) {
          uint4 *dst = reinterpret_cast<uint4 *>(static_cast<T *>(p.out) + (w.q0 + index) * p.out_stride + static_cast<long long>(h) * D + q * 32);
#pragma unroll
          for (int e = 0; e < 4; ++e)
            dst[e] = make_uint4(X::pack(o[8 * e], o[8 * e + 1]), X::pack(o[8 * e + 2], o[8 * e + 3]), X::pack(o[8 * e + 4], o[8 * e + 5]),
                                X::pack(o[8 * e + 6], o[8 * e + 7]));
        } else {
          float4 *dst = reinterpret_cast<float4 *>(p.part_o + (static_cast<long long>(blockIdx.y) * p.n_q * p.n_heads + at) * D + q * 32);
#pragma unroll
          for (int e = 0; e < 8; ++e) dst[e] = make_float4(o[4 * e], o[4 * e + 1], o[4 * e + 2], o[4 * e + 3]);
        }
      }
      if (live) {
        if (!whole) {
          p.part_ml[static_cast<long long>(blockIdx.y) * p.n_q * p.n_heads + at] = make_float2(ref, l);
        } else if (p.lse) {
          p.lse[at] = l == 0.f ? -INFINITY : ref * p.scale + logf(l * exp2f(-PtType<T>::kBias));
        }
      }
    }
    tc_fence_before();
  }
  __syncthreads();
  if (warp == kPtMma) {
    tc_fence_after();
    tmem_dealloc(tmem, S::kCols);
  }
}

// Joins the parts of a row and head, in order: a warp each.
template <typename T, int D>
__global__ void __launch_bounds__(128) prompt_join_kernel(const PromptParams p, int splits) {
  using X = Type16<T>;
  pdl_wait();
  pdl_launch_dependents();
  const int lane = threadIdx.x & 31;
  const long long rows = static_cast<long long>(p.n_q) * p.n_heads, at = static_cast<long long>(blockIdx.x) * 4 + (threadIdx.x >> 5);
  if (at >= rows) return;
  const int row = static_cast<int>(at / p.n_heads), h = static_cast<int>(at % p.n_heads);
  if (row < p.q_start[0] || row >= p.q_start[p.n_seq]) return;
  float m = -INFINITY, l = 0.f;
  for (int k = 0; k < splits; ++k) m = fmaxf(m, p.part_ml[k * rows + at].x);
  const float c = p.scale * 1.4426950408889634f;
  float2 o[D / 64] = {};
  for (int k = 0; k < splits; ++k) {
    const float2 ml = p.part_ml[k * rows + at];
    // (nothing seen: zeros; only NaN scores: a sum of NaN)
    const float f = ml.x == -INFINITY ? (ml.y == 0.f ? 0.f : 1.f) : ex2((ml.x - m) * c);
    if (f == 0.f) continue;
    l += f * ml.y;
#pragma unroll
    for (int g = 0; g < D / 64; ++g) {
      const float2 v = *reinterpret_cast<const float2 *>(p.part_o + (k * rows + at) * D + g * 64 + lane * 2);
      o[g].x += f * v.x, o[g].y += f * v.y;
    }
  }
  const float inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
  for (int g = 0; g < D / 64; ++g)
    *reinterpret_cast<uint32_t *>(static_cast<T *>(p.out) + row * p.out_stride + static_cast<long long>(h) * D + g * 64 + lane * 2) =
        X::pack(o[g].x * inv, o[g].y * inv);
  if (p.lse && lane == 0) p.lse[at] = l == 0.f ? -INFINITY : m * p.scale + logf(l * exp2f(-PtType<T>::kBias));
}

}  // namespace wf

using namespace wf;

// How a call is cut up: a function of its sizes alone.
struct PtPlan {
  int tokens, tiles, splits;
  int64_t items;
};
static PtPlan pt_plan(int64_t n_seq, int64_t n_q, int64_t max_k, int64_t heads, int64_t group) {
  PtPlan a;
  a.tokens = static_cast<int>(128 / group);
  const auto items = [&](int tiles) { return std::min(n_q, n_q / (a.tokens * tiles) + n_seq); };
  a.tiles = items(2) * heads >= kSms ? 2 : 1;
  a.items = items(a.tiles);
  // Few rows behind many keys: cut until there are four CTAs an SM, eight blocks of keys each at least.
  const int64_t blocks = (max_k + kPtKeys - 1) / kPtKeys;
  a.splits = static_cast<int>(std::max<int64_t>(1, std::min<int64_t>({blocks / 8, kSms * 4 / std::max<int64_t>(1, a.items * heads), 64})));
  return a;
}

static PFN_cuTensorMapEncodeTiled_v12000 pt_encode() {
  static PFN_cuTensorMapEncodeTiled_v12000 fn = nullptr;
  static std::once_flag once;
  std::call_once(once, [] {
    void *ptr = nullptr;
    cudaDriverEntryPointQueryResult q;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &ptr, 12000, cudaEnableDefault, &q) == cudaSuccess &&
        q == cudaDriverEntryPointSuccess)
      fn = reinterpret_cast<PFN_cuTensorMapEncodeTiled_v12000>(ptr);
  });
  return fn;
}

template <typename T, int D>
static cudaError_t pt_launch(const CUtensorMap &mq, const CUtensorMap &mk, const CUtensorMap &mv, const PromptParams &p, const PtPlan &a, cudaStream_t s) {
  static PerDevice ready;
  const void *fn = reinterpret_cast<const void *>(prompt_attention_kernel<T, D>);
  cudaError_t e = cudaSuccess;
  if (!ready.get(current_device(), [&]() -> int {
        e = cudaFuncSetAttribute(fn, cudaFuncAttributeMaxDynamicSharedMemorySize, PtShape<D>::kSmem);
        if (e == cudaSuccess) e = prefer_max_shared(fn);
        return e == cudaSuccess;
      }))
    return e;
  void *args[] = {const_cast<CUtensorMap *>(&mq), const_cast<CUtensorMap *>(&mk), const_cast<CUtensorMap *>(&mv), const_cast<PromptParams *>(&p)};
  e = launch_pdl(fn, dim3(static_cast<unsigned>(a.items * p.heads), a.splits), kPtThreads, PtShape<D>::kSmem, args, s);
  if (e == cudaSuccess && a.splits > 1) {
    int splits = a.splits;
    void *join[] = {const_cast<PromptParams *>(&p), &splits};
    e = launch_pdl(reinterpret_cast<const void *>(prompt_join_kernel<T, D>),
                   static_cast<unsigned>((static_cast<int64_t>(p.n_q) * p.n_heads + 3) / 4), 128, 0, join, s);
  }
  return e;
}

extern "C" {

size_t wf_prompt_attention_scratch_bytes(int32_t n_seq, int32_t n_q, int32_t max_k, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim) {
  if (n_seq <= 0 || n_q <= 0 || max_k < 0 || n_heads <= 0 || n_kv_heads <= 0 || n_heads % n_kv_heads || n_heads / n_kv_heads > 64 ||
      (head_dim != 64 && head_dim != 128))
    return 0;
  const PtPlan a = pt_plan(n_seq, n_q, max_k, n_kv_heads, n_heads / n_kv_heads);
  return a.splits == 1 ? 0 : static_cast<size_t>(a.splits) * n_q * n_heads * (head_dim + 2) * sizeof(float);
}

wf_status wf_prompt_attention(const void *d_q, int64_t q_stride, const void *d_k, int64_t k_stride, const void *d_v, int64_t v_stride,
                              const int32_t *d_q_start, const int32_t *d_k_start, int32_t n_seq, int32_t n_q, int32_t n_k, int32_t max_k,
                              int32_t n_heads, int32_t n_kv_heads, int32_t head_dim, int32_t dtype, int32_t causal, float scale,
                              void *d_out, int64_t out_stride, float *d_lse, void *d_scratch, size_t scratch_bytes, uint32_t *d_err,
                              void *stream) {
  const int64_t qd = static_cast<int64_t>(n_heads) * head_dim, kd = static_cast<int64_t>(n_kv_heads) * head_dim;
  if (!d_q || !d_k || !d_v || !d_q_start || !d_k_start || !d_out || n_seq <= 0 || n_q < 0 || n_k < 0 || max_k < 0 || n_heads <= 0 ||
      n_kv_heads <= 0 || n_heads % n_kv_heads || !(scale > 0.f) || !std::isfinite(scale))
    return WF_ERR_INVALID;
  if ((head_dim != 64 && head_dim != 128) || (dtype != WF_BF16 && dtype != WF_F16) || n_heads / n_kv_heads > 64 || n_heads > 4096)
    return WF_ERR_UNSUPPORTED;
  if (!aligned16(d_q) || !aligned16(d_k) || !aligned16(d_v) || !aligned16(d_out) || q_stride % 8 || k_stride % 8 || v_stride % 8 ||
      out_stride % 8 || q_stride < qd || k_stride < kd || v_stride < kd || out_stride < qd || (reinterpret_cast<uintptr_t>(d_lse) & 3))
    return WF_ERR_INVALID;
  if (n_q == 0) return WF_OK;
  const int group = n_heads / n_kv_heads;
  const PtPlan a = pt_plan(n_seq, n_q, max_k, n_kv_heads, group);
  if (a.items * n_kv_heads > INT32_MAX || static_cast<int64_t>(n_q) * n_heads > INT32_MAX * 4LL) return WF_ERR_UNSUPPORTED;
  PromptParams p = {};
  p.out = d_out, p.lse = d_lse, p.out_stride = out_stride, p.q_start = d_q_start, p.k_start = d_k_start;
  p.n_seq = n_seq, p.n_q = n_q, p.n_k = n_k, p.max_k = max_k;
  p.n_heads = n_heads, p.heads = n_kv_heads, p.group = group, p.causal = causal != 0, p.scale = scale, p.err = d_err;
  p.tokens = a.tokens, p.tiles = a.tiles;
  if (a.splits > 1) {
    if (!d_scratch || !aligned16(d_scratch)) return WF_ERR_INVALID;
    if (scratch_bytes < wf_prompt_attention_scratch_bytes(n_seq, n_q, max_k, n_heads, n_kv_heads, head_dim)) return WF_ERR_CAPACITY;
    p.part_o = static_cast<float *>(d_scratch);
    p.part_ml = reinterpret_cast<float2 *>(p.part_o + static_cast<size_t>(a.splits) * n_q * n_heads * head_dim);
  }
  const auto encode = pt_encode();
  if (!encode) return WF_ERR_CUDA;
  const CUtensorMapDataType type = dtype == WF_F16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16;
  const cuuint32_t step[4] = {1, 1, 1, 1};
  CUtensorMap mq, mk, mv;
  const cuuint64_t dim = head_dim;
  {  // queries: dims, heads of a group, groups, rows
    const cuuint64_t size[4] = {dim, static_cast<cuuint64_t>(group), static_cast<cuuint64_t>(n_kv_heads), static_cast<cuuint64_t>(n_q)};
    const cuuint64_t stride[3] = {dim * 2, dim * 2 * group, static_cast<cuuint64_t>(q_stride) * 2};
    const cuuint32_t box[4] = {64, static_cast<cuuint32_t>(group), 1, static_cast<cuuint32_t>(a.tokens)};
    if (encode(&mq, type, 4, const_cast<void *>(d_q), size, stride, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
               CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
      return WF_ERR_CUDA;
  }
  for (int i = 0; i < 2; ++i) {  // keys, values: dims, heads, rows
    const cuuint64_t size[3] = {dim, static_cast<cuuint64_t>(n_kv_heads), static_cast<cuuint64_t>(std::max(n_k, 1))};
    const cuuint64_t stride[2] = {dim * 2, static_cast<cuuint64_t>(i ? v_stride : k_stride) * 2};
    const cuuint32_t box[3] = {64, 1, kPtKeys};
    if (encode(i ? &mv : &mk, type, 3, const_cast<void *>(i ? d_v : d_k), size, stride, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
               CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
      return WF_ERR_CUDA;
  }
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  using B = __nv_bfloat16;
  cudaError_t e;
  if (dtype == WF_F16)
    e = head_dim == 128 ? pt_launch<__half, 128>(mq, mk, mv, p, a, s) : pt_launch<__half, 64>(mq, mk, mv, p, a, s);
  else
    e = head_dim == 128 ? pt_launch<B, 128>(mq, mk, mv, p, a, s) : pt_launch<B, 64>(mq, mk, mv, p, a, s);
  return e == cudaSuccess ? WF_OK : WF_ERR_CUDA;
}

}  // extern "C"
