// Attention of whole prompts, packed one after another (softmax(scale q K^T) V).
//
// A tile is 128 rows of one sequence and key/value head: a row is a (token,
// query head of the group) pair, heads innermost, so that one block of 128 keys
// serves every head of the group whatever its size.  A CTA has up to two tiles
// that share their key blocks.  Both products run on tcgen05 with fp32 sums in
// TMEM: S = Q K^T from shared memory, O += P V with P in TMEM, over the
// columns that its S was read from.  Four warps a tile turn S into P, a thread a
// row: no shuffles.  A row's weights are relative to the maximum of its first
// block, and O is rescaled only where a later weight would pass 2^16, so that no
// maximum is taken of most blocks.  A weight is rounded to the rows' type, as the
// product's two operands are of one type: up to 2^-8 of it in bf16, 2^-11 in fp16; its
// row's sum is of the weights in fp32.
//   one prompt of 8192 tokens, 32 heads on 8, 128 wide, causal, bf16: 356 us,
//     1.54 PFLOP/s, by the tensor unit and shared memory (58% busy at 4096 tokens),
//     and the way from a tile's weights to its next scores
//   32 x 1500 frames, 20 heads, 64 wide: 379 us, 0.97 PFLOP/s, by that way (the tensor unit works 66% of the time)
//   16 prompts of 5 to 224 tokens, 20 heads, 64 wide: 10 to 11.8 us, two rounds of CTAs
//     of 1 us to find their rows, 1 us to the first scores, 0.8 us a block and 1 us of results
//   three pieces of 2 to 300 tokens behind 15000 to 30000, 32 heads on 8, 128 wide,
//     fp16: 177 to 200 us, 0.95 PFLOP/s, tiles that are not full and the join
#include <cuda.h>
#include <cudaTypedefs.h>

#include <algorithm>
#include <climits>
#include <cmath>
#include <mutex>

#include "wf_device.cuh"
#include "wf_ops.cuh"

namespace wf {

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

// At 128 dims a CTA has the SM: blocks of 128 keys, all of TMEM; the products
// take as long as the tensor unit's way to shared memory, 128 bytes a clock.  At
// 64 dims what a tile waits for is the way from a block's weights to its next
// scores (without any exponentials the case below takes 360 us), so two CTAs
// share the SM, with blocks of 64 keys, and four tiles' ways overlap.
//   32 x 1500 frames, 20 heads: 379 us.  One CTA with 128 keys and a third buffer
//   of scores 442; one with weights beside the scores, so that the next ones are
//   there when a softmax ends: three tiles and 64 keys 414, two and 128 479.
template <int D>
struct PtShape {
  static constexpr int kKeys = D == 64 ? 64 : 128;  // of a block
  static constexpr int kParts = kKeys / 64;         // in which a block's weights are handed over
  static constexpr int kPerSm = D == 64 ? 2 : 1;
  static constexpr int kHalf = 16384;               // 128 rows of 64 dims
  static constexpr int kTile = kHalf * D / 64;      // queries
  static constexpr int kKvHalf = kKeys * 128, kKv = kKvHalf * D / 64;  // keys or values
  static constexpr int kKStages = D == 64 ? 4 : 2, kVStages = D == 64 ? 4 : 3;
  static constexpr int kScores = 2;                 // buffers of scores in TMEM, before the tiles' sums
  static constexpr int kSumCol = kScores * kKeys;
  static constexpr uint32_t kCols = D == 64 ? 256 : 512;
  static constexpr int kRegs = D == 64 ? 80 : 168, kRegsMore = D == 64 ? 96 : 208, kRegsLess = D == 64 ? 48 : 88;
  static_assert(256 * kRegsMore + 128 * kRegsLess == kPtThreads * kRegs && kPerSm * kPtThreads * kRegs <= 65536, "");
  static constexpr int kMarkOff = 2 * kTile + (kKStages + kVStages) * kKv;  // [3][D] first position of a value that is not finite
  static constexpr int kBarOff = kMarkOff + 3 * D * 4;
  static constexpr int kBars = 2 + 2 * kKStages + 4 * kVStages + (1 + kParts) * kScores + 2 + 1;
  static constexpr int kSmem = 1024 + kBarOff + kBars * 8 + 64;
  static_assert(kSumCol + 2 * D <= static_cast<int>(kCols), "");
};

// A warp's waits on barriers, all lanes together.  After one that gave up the
// others ask once: the kernel comes to its end, with the error recorded.
struct PtWaits {
  uint32_t *err;
  long long limit;
};
__device__ __forceinline__ bool pt_try(uint32_t bar, uint32_t parity) {
  uint32_t ok;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(ok)
      : "r"(bar), "r"(parity)
      : "memory");
  return __all_sync(0xffffffffu, ok) != 0;
}
__device__ __forceinline__ void pt_wait(PtWaits &w, uint32_t bar, uint32_t parity) {
  if (pt_try(bar, parity)) return;
  const long long t0 = clock64();
  while (!pt_try(bar, parity)) {
    if (__any_sync(0xffffffffu, clock64() - t0 > w.limit)) {
      set_error(w.err, WF_DEV_ERR_TIMEOUT);
      w.limit = 0;
      return;
    }
  }
}

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
// One lane of a converged warp.
__device__ __forceinline__ uint32_t elect_one() {
  uint32_t e;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(e));
  return e;
}
// The products are issued by a whole warp under a predicate that one lane has:
// behind a branch on the lane each instruction's operands took the slow way to
// the uniform registers, 76 clocks an instruction instead of the product's own 32 to 64.
// D (+)= A B^T, both in shared memory.
__device__ __forceinline__ void pt_mma_ss(uint32_t lead, uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "setp.ne.b32 q, %5, 0;\n\t"
      "@q tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
      "l"(a), "l"(b), "r"(idesc), "r"(accumulate), "r"(lead)
      : "memory");
}
// D (+)= A B with A in TMEM.
__device__ __forceinline__ void pt_mma_ts(uint32_t lead, uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "setp.ne.b32 q, %5, 0;\n\t"
      "@q tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d),
      "r"(a), "l"(b), "r"(idesc), "r"(accumulate), "r"(lead)
      : "memory");
}
__device__ __forceinline__ void pt_commit(uint32_t lead, uint32_t bar) {
  asm volatile(
      "{\n\t.reg .pred q;\n\t"
      "setp.ne.b32 q, %1, 0;\n\t"
      "@q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t}" ::"r"(bar),
      "r"(lead)
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
// Behind tmem_ld_wait: what is computed from v stays behind it too.
__device__ __forceinline__ void tmem_loaded(float (&v)[32]) {
  asm volatile(""
               : "+f"(v[0]),"+f"(v[1]),"+f"(v[2]),"+f"(v[3]),"+f"(v[4]),"+f"(v[5]),"+f"(v[6]),"+f"(v[7]),"+f"(v[8]),"+f"(v[9]),"+f"(v[10]),"+f"(v[11]),"+f"(v[12]),"+f"(v[13]),"+f"(v[14]),"+f"(v[15]),
                 "+f"(v[16]),"+f"(v[17]),"+f"(v[18]),"+f"(v[19]),"+f"(v[20]),"+f"(v[21]),"+f"(v[22]),"+f"(v[23]),"+f"(v[24]),"+f"(v[25]),"+f"(v[26]),"+f"(v[27]),"+f"(v[28]),"+f"(v[29]),"+f"(v[30]),"+f"(v[31]));
}
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

// The query rows that starts may name: from the first start to the last.
struct PtRange {
  int from, to;
};
__device__ __forceinline__ PtRange pt_range(const PromptParams &p, int first, int last) {
  PtRange r;
  r.from = min(max(first, 0), p.n_q);
  r.to = max(min(last, p.n_q), r.from);
  return r;
}

// The sequence and first token of work item `item` (a warp; every lane gets it).
// Items number each sequence's groups of `per` tokens, the last group first.
// Starts that are none are brought into pt_range and made ascending, so that no
// two sequences have a row in common and there are no more items than CTAs for them.
// False: there is no such item.
__device__ __forceinline__ bool pt_find(const PromptParams &p, int item, int lane, PtWork &w) {
  const int per = p.tokens * p.tiles;
  const int end_row = p.q_start[p.n_seq];
  int before = 0, latest = 0;  // latest: of starts that are none, the largest so far
  bool bent = false;
  for (int base = 0; base < p.n_seq; base += 32) {
    const int i = base + lane;
    int a = 0, b = 0, rk0 = 0, rk1 = 0;
    if (i < p.n_seq) {
      a = p.q_start[i], b = p.q_start[i + 1];
      rk0 = p.k_start[i], rk1 = p.k_start[i + 1];
    }
    // (every pair up to here in order and none above the last start: so is the whole)
    bent |= __any_sync(0xffffffffu, i < p.n_seq && (a < 0 || b < a || b > end_row || end_row > p.n_q)) != 0;
    if (bent) {
      const PtRange range = pt_range(p, p.q_start[0], end_row);
      int most = i < p.n_seq ? max(a, latest) : 0;
      for (int off = 1; off < 32; off <<= 1) {
        const int v = __shfl_up_sync(0xffffffffu, most, off);
        if (lane >= off) most = max(most, v);
      }
      a = min(max(most, range.from), range.to), b = i < p.n_seq ? min(max(most, b), range.to) : a;
      b = max(b, a);
      latest = __shfl_sync(0xffffffffu, most, 31);
    }
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
      rk0 = __shfl_sync(0xffffffffu, rk0, src), rk1 = __shfl_sync(0xffffffffu, rk1, src);
      w.k0 = min(max(rk0, 0), p.n_k);
      const int k1 = min(max(rk1, w.k0), p.n_k);
      w.keys = min(k1 - w.k0, p.max_k);
      if (lane == 0 && k1 - w.k0 > p.max_k) set_error(p.err, WF_DEV_ERR_CAPACITY);
      return true;
    }
    before += __shfl_sync(0xffffffffu, sum, 31);
  }
  return false;
}

// Tells of starts that descend or leave the buffers (a warp).
__device__ __forceinline__ void pt_check_starts(const PromptParams &p, int lane) {
  bool bad = false;
  for (int i = lane; i < p.n_seq; i += 32) {
    const int a = p.q_start[i], b = p.q_start[i + 1], k0 = p.k_start[i], k1 = p.k_start[i + 1];
    bad |= a < 0 || b < a || b > p.n_q || k0 < 0 || k1 < k0 || k1 > p.n_k;
  }
  if (bad) set_error(p.err, WF_DEV_ERR_PAGE);
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
__global__ void __launch_bounds__(kPtThreads, PtShape<D>::kPerSm)
    prompt_attention_kernel(const __grid_constant__ CUtensorMap mq, const __grid_constant__ CUtensorMap mk, const __grid_constant__ CUtensorMap mv,
                            const PromptParams p) {
  using X = Type16<T>;
  using S = PtShape<D>;
  constexpr int kKStages = S::kKStages, kVStages = S::kVStages, kKeys = S::kKeys, kParts = S::kParts;
  extern __shared__ uint8_t smem_raw[];
  uint8_t *smem = smem_raw + ((1024 - (smem_u32(smem_raw) & 1023)) & 1023);
  uint8_t *sq = smem, *sk = smem + 2 * S::kTile, *sv = sk + kKStages * S::kKv;
  int *mark = reinterpret_cast<int *>(smem + S::kMarkOff);
  uint64_t *q_full = reinterpret_cast<uint64_t *>(smem + S::kBarOff);
  uint64_t *k_full = q_full + 2, *k_empty = k_full + kKStages, *v_full = k_empty + kKStages, *v_empty = v_full + kVStages;
  uint64_t *look = v_empty + kVStages, *clean = look + kVStages;
  uint64_t *s_full = clean + kVStages, *p_full = s_full + S::kScores, *o_done = p_full + kParts * S::kScores, *done = o_done + 2;
  uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(done + 1);
  int *has_work = reinterpret_cast<int *>(tmem_slot + 1);
  volatile int *marked = has_work + 1;
  PtWork *shared_work = reinterpret_cast<PtWork *>(has_work + 2);

  const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
  if (threadIdx.x == kPtLoad * 32) tma_prefetch_desc(&mq), tma_prefetch_desc(&mk), tma_prefetch_desc(&mv);
  pdl_wait();
  const int head = blockIdx.x % p.heads;
  if (warp == 0) {
    PtWork w = {};
    const bool any = pt_find(p, blockIdx.x / p.heads, lane, w);
    if (any) {
      // key blocks that any row of this CTA sees, and this split's share of them
      const int last_token = min(w.token + p.tokens * p.tiles, w.rows) - 1;
      const int blocks = (pt_limit(w, p.causal, last_token) + kKeys - 1) / kKeys;
      const int share = (blocks + gridDim.y - 1) / gridDim.y;
      w.first = min(static_cast<int>(blockIdx.y) * share, blocks), w.last = min(w.first + share, blocks);
    }
    if (lane == 0) *shared_work = w, *has_work = any, *marked = 0;
  }
  if (threadIdx.x == 32) {
    for (int i = 0; i < 2; ++i) mbar_init(&q_full[i], 1), mbar_init(&o_done[i], 1);
    for (int i = 0; i < kKStages; ++i) mbar_init(&k_full[i], 1), mbar_init(&k_empty[i], 1);
    for (int i = 0; i < kVStages; ++i) {
      mbar_init(&v_full[i], 1), mbar_init(&v_empty[i], 1);
      mbar_init(&look[i], 1), mbar_init(&clean[i], 64);
    }
    for (int i = 0; i < S::kScores; ++i) mbar_init(&s_full[i], 1);
    for (int i = 0; i < kParts * S::kScores; ++i) mbar_init(&p_full[i], 4);
    mbar_init(done, 1);
    fence_barrier_init();
    fence_proxy_async();
  }
  for (int i = threadIdx.x; i < 3 * D; i += kPtThreads) mark[i] = INT_MAX;
  if (warp == kPtMma) tmem_alloc(tmem_slot, S::kCols);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  // Not before this CTA has its TMEM: a kernel that follows may take its own before it
  // waits for this one, and each would then wait for the other.
  pdl_launch_dependents();
  // Broadcast, so that the compiler knows that they are the same in all of a warp
  // and keeps what follows from them in uniform registers.
  const auto uniform = [](int v) { return __shfl_sync(0xffffffffu, v, 0); };
  const uint32_t tmem = uniform(*tmem_slot);
  const PtWork w = {uniform(shared_work->seq),  uniform(shared_work->q0),    uniform(shared_work->rows),  uniform(shared_work->k0),
                    uniform(shared_work->keys), uniform(shared_work->token), uniform(shared_work->first), uniform(shared_work->last)};
  const bool any_work = uniform(*has_work) != 0;
  // tile i: its tokens and the blocks that its rows see of this CTA's
  const int tokens[2] = {any_work ? min(p.tokens, w.rows - w.token) : 0,
                         any_work && p.tiles > 1 ? min(max(w.rows - w.token - p.tokens, 0), p.tokens) : 0};
  int ends[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int seen = tokens[i] ? pt_limit(w, p.causal, w.token + i * p.tokens + tokens[i] - 1) : 0;
    ends[i] = max(min((seen + kKeys - 1) / kKeys, w.last), w.first);
  }
  const int end = max(ends[0], ends[1]);
  // blocks from here on hold positions that some row does not see
  const int edge = any_work ? pt_limit(w, p.causal, w.token) / kKeys : 0;
  // The products go through the blocks, tile by tile; number n is block j of tile
  // i, its scores in buffer n % kScores.
  const int both = min(ends[0], ends[1]);  // blocks before it are both tiles'
  const int products = ends[0] + ends[1] - 2 * w.first;

  // The block's registers go to the softmax: kRegs a thread at launch, kRegsMore
  // for its 256 threads and kRegsLess for the other 128, the same sum.
  if (warp >= kPtMma) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(S::kRegsLess));
    if (warp == kPtLoad) {
      if (lane == 0 && w.first < end) {
        const uint32_t q_bytes = static_cast<uint32_t>(p.group * p.tokens) * D * 2;
        const auto load_q = [&](int i) {
          mbar_arrive_expect_tx(&q_full[i], q_bytes);
          for (int c = 0; c < D / 64; ++c)
            tma_load_4d(sq + i * S::kTile + c * S::kHalf, &mq, c * 64, 0, head, w.q0 + w.token + i * p.tokens, &q_full[i]);
        };
        if (ends[0] > w.first) load_q(0);
        int n = 0;  // blocks so far, keys and values
        bool ok = true;
        for (int j = w.first; j < end && ok; ++j, ++n) {
          const int ks = n % kKStages, vs = n % kVStages;
          if (n >= kKStages) ok = mbar_wait(&k_empty[ks], ((n / kKStages) - 1) & 1, p.err, kSpinLimitCycles);
          if (!ok) break;
          mbar_arrive_expect_tx(&k_full[ks], S::kKv);
          for (int c = 0; c < D / 64; ++c) tma_load_3d(sk + ks * S::kKv + c * S::kKvHalf, &mk, c * 64, head, w.k0 + j * kKeys, &k_full[ks]);
          if (n == 0 && ends[1] > w.first) load_q(1);
          if (n >= kVStages) ok = mbar_wait(&v_empty[vs], ((n / kVStages) - 1) & 1, p.err, kSpinLimitCycles);
          if (!ok) {
            mbar_drain(&k_full[ks], (n / kKStages) & 1);
            break;
          }
          mbar_arrive_expect_tx(&v_full[vs], S::kKv);
          for (int c = 0; c < D / 64; ++c) tma_load_3d(sv + vs * S::kKv + c * S::kKvHalf, &mv, c * 64, head, w.k0 + j * kKeys, &v_full[vs]);
          // The stage's earlier copies have landed: only now is the parity of its barrier one to wait for.
          if (j >= edge) mbar_arrive_cta(&look[vs]);
        }
        // a wait gave up, here or in another warp: the copies still have to land before the CTA ends
        for (int i = 0; i < 2; ++i)
          if (ends[i] > w.first) mbar_drain(&q_full[i], 0);
        for (int i = max(0, n - kKStages); i < n; ++i) mbar_drain(&k_full[i % kKStages], (i / kKStages) & 1);
        for (int i = max(0, n - kVStages); i < n; ++i) mbar_drain(&v_full[i % kVStages], (i / kVStages) & 1);
      }
    } else if (warp == kPtMma) {
      if (w.first < end) {
        const uint32_t lead = elect_one();
        constexpr uint32_t kIdS = pt_idesc<T>(kKeys, false), kIdO = pt_idesc<T>(D, true);
        const uint64_t dq = umma_desc_sw128(smem_u32(sq)), dk = umma_desc_sw128(smem_u32(sk)), dv = pt_desc_v(smem_u32(sv));
        const uint32_t bars = smem_u32(q_full);
        const auto at = [&](const uint64_t *bar) { return bars + static_cast<uint32_t>(bar - q_full) * 8; };
        PtWaits waits = {p.err, kSpinLimitCycles};
        // The next scores are of block qj of tile qi, in buffer q_buf, with keys of
        // stage q_st; the next product with values has the same of its own.
        int qj = w.first, qi = qj < ends[0] ? 0 : 1, q_buf = 0, q_st = 0;
        int pj = qj, pi = qi, p_buf = 0, p_st = 0;
        uint32_t q_phase = 0, p_phase = 0, v_phase = 0;
        const auto scores_inputs = [&]() {
          if (qi == 0 || qj >= ends[0]) pt_wait(waits, at(k_full) + q_st * 8, q_phase);
          if (qj == w.first) pt_wait(waits, at(q_full) + qi * 8, 0);
        };
        const auto scores = [&]() {
          const uint64_t a = dq + qi * (S::kTile >> 4), b = dk + q_st * (S::kKv >> 4);
          const uint32_t d = tmem + q_buf * kKeys;
#pragma unroll
          for (int k = 0; k < D / 16; ++k)
            pt_mma_ss(lead, d, a + ((k / 4 * S::kHalf + k % 4 * 32) >> 4), b + ((k / 4 * S::kKvHalf + k % 4 * 32) >> 4), kIdS, k > 0);
          pt_commit(lead, at(s_full) + q_buf * 8);
        };
        const auto scores_issued = [&]() {
          q_buf = q_buf + 1 == S::kScores ? 0 : q_buf + 1;
          if (qi == 0 && qj < ends[1]) {
            qi = 1;
          } else {  // the block's last
            pt_commit(lead, at(k_empty) + q_st * 8);
            ++qj;
            qi = qj < ends[0] ? 0 : 1;
            if (++q_st == kKStages) q_st = 0, q_phase ^= 1;
          }
        };
#pragma unroll 1
        for (int n = 0; n < S::kScores && n < products; ++n) scores_inputs(), tc_fence_after(), scores(), scores_issued();
#pragma unroll 1
        for (int n = 0; n < products; ++n) {
          // what can be told afterwards is: the way from a block's weights to its
          // tile's next scores is the longest there is
          const bool more_scores = n + S::kScores < products;
          if (pi == 0 || pj >= ends[0]) {
            pt_wait(waits, at(v_full) + p_st * 8, v_phase);
            if (pj >= edge) pt_wait(waits, at(clean) + p_st * 8, (pj - max(edge, w.first)) / kVStages & 1);
          }
          // with 64 dims the keys are there long before the weights are, and the look at their barrier costs less here
          if (D == 64 && more_scores) scores_inputs();
          const uint64_t b = dv + p_st * (S::kKv >> 4);
          const uint32_t d = tmem + S::kSumCol + pi * D, a = tmem + p_buf * kKeys;
          const uint32_t more = pj > w.first;
#pragma unroll
          for (int h = 0; h < kParts; ++h) {
            pt_wait(waits, at(p_full) + (p_buf * kParts + h) * 8, p_phase);
            tc_fence_after();
#pragma unroll
            for (int k = 4 * h; k < 4 * h + 4; ++k) pt_mma_ts(lead, d, a + k * 8, b + ((k * 2048) >> 4), kIdO, k > 0 ? 1u : more);
          }
          pt_commit(lead, at(o_done) + pi * 8);
          const bool block_done = pi == 1 || pj >= ends[1];
          if (block_done) pt_commit(lead, at(v_empty) + p_st * 8);
          // P's columns are read before the scores that are issued behind are written over them
          if (D != 64 && more_scores) scores_inputs();
          if (more_scores) scores();
          if (++p_buf == S::kScores) p_buf = 0, p_phase ^= 1;
          if (!block_done) {
            pi = 1;
          } else {
            ++pj;
            pi = pj < ends[0] ? 0 : 1;
            if (++p_st == kVStages) p_st = 0, v_phase ^= 1;
          }
          if (more_scores) scores_issued();
        }
        pt_commit(lead, at(done));
        mbar_drain(done, 0);
      }
    } else if (warp >= kPtScrub) {
      // Values of positions that some row does not see: zero past the sequence's
      // end, and where they are not finite, which a weight of 0 would not hide;
      // the rows that see those take them from `mark`.
      for (int j = max(edge, w.first); j < end; ++j) {
        const int n = j - w.first, st = n % kVStages;
        if (!__all_sync(0xffffffffu, mbar_wait(&look[st], (j - max(edge, w.first)) / kVStages & 1, p.err, kSpinLimitCycles) &&
                                         mbar_wait(&v_full[st], (n / kVStages) & 1, p.err, kSpinLimitCycles)))
          break;
        const int held = w.keys - j * kKeys;
        // (some vectors at a time, all of them on their way before the first is looked at)
        constexpr int kBatch = D / 16;
        for (int c0 = threadIdx.x - kPtScrub * 32; c0 < S::kKv / 16; c0 += 64 * kBatch) {
          uint4 v[kBatch];
          uint4 *at = reinterpret_cast<uint4 *>(sv + st * S::kKv + c0 * 16);
#pragma unroll
          for (int b = 0; b < kBatch; ++b) v[b] = at[b * 64];
          uint32_t odd = 0;
#pragma unroll
          for (int b = 0; b < kBatch; ++b) {
            const uint32_t m = 0x7fff7fffu;
            const uint32_t most = __vmaxu2(__vmaxu2(v[b].x & m, v[b].y & m), __vmaxu2(v[b].z & m, v[b].w & m));
            if ((c0 + b * 64) / 8 % kKeys >= held) {
              at[b * 64] = make_uint4(0, 0, 0, 0);
            } else if (max(most & 0xffff, most >> 16) >= PtType<T>::kInf) {
              odd |= 1u << b;
            }
          }
          for (; odd; odd &= odd - 1) {
            const int c = c0 + (__ffs(odd) - 1) * 64, row = c / 8 % kKeys;
            uint16_t *e = reinterpret_cast<uint16_t *>(sv + st * S::kKv + c * 16);
            const int dim = c / (8 * kKeys) * 64 + ((c & 7) ^ (row & 7)) * 8;
            for (int i = 0; i < 8; ++i) {
              const uint32_t u = e[i] & 0x7fff;
              if (u < PtType<T>::kInf) continue;
              atomicMin(&mark[(u > PtType<T>::kInf ? 0 : e[i] >> 15 ? 2 : 1) * D + dim + i], j * kKeys + row);
              e[i] = 0;
              *marked = 1;
            }
          }
        }
        fence_proxy_async();
        mbar_arrive_cta(&clean[st]);
      }
      if (blockIdx.x == 0 && blockIdx.y == 0 && warp == kPtScrub) pt_check_starts(p, lane);
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(S::kRegsMore));
    const int i = warp >> 2, row = (warp & 3) * 32 + lane;
    const uint32_t lanes = static_cast<uint32_t>((warp & 3) * 32) << 16;
    const uint32_t to = tmem + S::kSumCol + i * D + lanes;
    const int token = row / p.group, h = head * p.group + row % p.group, index = w.token + i * p.tokens + token;
    const bool live = token < tokens[i];
    const int limit = live ? pt_limit(w, p.causal, index) : 0;
    // the least of the tile's limits: blocks below it need no mask
    const int least = tokens[i] ? pt_limit(w, p.causal, w.token + i * p.tokens) : 0;
    const float c = p.scale * 1.4426950408889634f;
    float ref = -INFINITY, base = 0.f, l = 0.f;  // weights are 2^(score c + base)
    bool unset = true;  // some row of the warp has no reference
    PtWaits waits = {p.err, kSpinLimitCycles};
    // Waits until the products of the tile's block j are in its sums.  Every
    // block's in turn: a barrier tells a phase from the one before it, not from
    // the one before that.
    int waited = w.first;
    const auto added = [&](int j) {
      // (with two buffers and two tiles a tile's scores are behind its last products)
      if (waited > j || (S::kScores == 2 && j + 1 < both)) return;
      waited = j + 1;
      pt_wait(waits, smem_u32(&o_done[i]), (j - w.first) & 1);
      tc_fence_after();
    };
    int buf = w.first < both ? i : 0;  // of the scores, and the parity of its barrier
    uint32_t phase = 0;
    for (int j = w.first; j < ends[i]; ++j) {
      const uint32_t ts = tmem + buf * kKeys + lanes;
      pt_wait(waits, smem_u32(s_full) + buf * 8, phase);
      tc_fence_after();
      float s[2 * kParts][32];
      const int seen = limit - j * kKeys;
      const bool mask = (j + 1) * kKeys > least;
      const auto load = [&](int q) {
        tmem_ld32(ts + q * 32, s[q]);
      };
      // (one branch around all of it: a select for each column would cost as much as the rest)
      const auto loaded = [&](int first, int last) {
#pragma unroll
        for (int q = first; q < last; ++q) tmem_loaded(s[q]);
        if (mask) {
#pragma unroll
          for (int q = first; q < last; ++q)
#pragma unroll
            for (int e = 0; e < 32; ++e)
              if (q * 32 + e >= seen) s[q][e] = -INFINITY;
        }
      };
      const auto largest = [&](int q) {
        float m0 = max3(s[q][0], s[q][1], s[q][2]), m1 = max3(s[q][3], s[q][4], s[q][5]);
#pragma unroll
        for (int e = 6; e < 30; e += 4) m0 = max3(m0, s[q][e], s[q][e + 1]), m1 = max3(m1, s[q][e + 2], s[q][e + 3]);
        return max3(fmaxf(m0, m1), s[q][30], s[q][31]);
      };
      // Brings the reference up to the block's maximum, and the sums with it, where
      // `mine`: a row's bits do not turn on what the others of its warp hold.
      const auto raise = [&](bool mine) {
        float next = max3(largest(0), largest(1), ref);
        if constexpr (kParts == 2) next = max3(largest(2), largest(3), next);
        if (!mine) next = ref;
        const float keep = !mine ? 1.f : ref == -INFINITY ? 0.f : ex2((ref - next) * c);
        ref = next;
        base = ref == -INFINITY ? 0.f : PtType<T>::kBias - ref * c;
        unset = __any_sync(0xffffffffu, ref == -INFINITY);
        l *= keep;
        if (j == w.first) return;
        added(j - 1);
#pragma unroll 1
        for (int q = 0; q < D / 32; ++q) {
          float o[32];
          tmem_ld32(to + q * 32, o);
          tmem_ld_wait();
          tmem_loaded(o);
          uint32_t kept[32];
#pragma unroll
          for (int e = 0; e < 32; ++e) kept[e] = __float_as_uint(o[e] * keep);
          tmem_st(to + q * 32, kept);
        }
        // (read again rather than held in registers meanwhile)
        load(0), load(1);
        tmem_ld_wait();
        loaded(0, 2);
      };
      uint32_t packed[32];
      float2 sums[4];
      // Weights of 64 columns: pair by pair in three steps that are some pairs
      // apart, so that no instruction waits for the one before it and the
      // exponentials, which take the longest, have the others between them.
      const auto weights = [&](int half, auto between) {
        constexpr int kAhead = 6, kBehind = 4;
        float(&x)[2][32] = *reinterpret_cast<float(*)[2][32]>(&s[2 * half]);
#pragma unroll
        for (int g = -kAhead; g < 32 + kBehind; ++g) {
          const int f = g + kAhead, h = g - kBehind;
          if (f < 32) {
            const float2 y = fma2(make_float2(x[f / 16][f % 16 * 2], x[f / 16][f % 16 * 2 + 1]), make_float2(c, c), make_float2(base, base));
            x[f / 16][f % 16 * 2] = y.x, x[f / 16][f % 16 * 2 + 1] = y.y;
          }
          if (g >= 0 && g < 32) x[g / 16][g % 16 * 2] = ex2(x[g / 16][g % 16 * 2]);
          if (h >= 0) {
            const float2 v = make_float2(x[h / 16][h % 16 * 2], x[h / 16][h % 16 * 2 + 1]);
            sums[h % 4] = half == 0 && h < 4 ? v : add2(sums[h % 4], v);
            packed[h] = X::pack(v.x, v.y);
          }
          if (g >= 0 && g < 32) x[g / 16][g % 16 * 2 + 1] = ex2(x[g / 16][g % 16 * 2 + 1]);
          between(g);
        }
      };
      const auto nothing = [](int) {};
      const auto hand_over = [&](int part) {
        tmem_st_wait();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive_cta(&p_full[kParts * buf + part]);
      };
#pragma unroll
      for (int q = 0; q < 2 * kParts; ++q) load(q);
      tmem_ld_wait();
      loaded(0, 2 * kParts);
      // A row's reference is the maximum of its first block, and then stands
      // while the weights stay below 2^16, which the first part's sum and the
      // second part's maximum tell before any of them is handed over.
      bool low = unset && ref == -INFINITY;  // the row's reference has to be raised
      if (unset) raise(low);
      for (bool again = false;; again = true) {
        weights(0, nothing);
        const float2 sum = add2(add2(sums[0], sums[1]), add2(sums[2], sums[3]));
        low = sum.x + sum.y > 65000.f;
        if constexpr (kParts == 2) low |= fmaf(fmaxf(largest(2), largest(3)), c, base) > 15.9f;
        if (again || !__any_sync(0xffffffffu, low)) break;  // (infinite scores stay above)
        load(0), load(1);
        tmem_ld_wait();
        loaded(0, 2);
        raise(low);
      }
      if (j > w.first) added(j - 1);
      tmem_st(ts, packed);
      if constexpr (kParts == 2) {
        weights(1, [&](int g) {
          if (g != 2) return;  // the stores have had time; the product of the first part may begin
          hand_over(0);
        });
        tmem_st(ts + 32, packed);
      }
      hand_over(kParts - 1);
      const float2 sum = add2(add2(sums[0], sums[1]), add2(sums[2], sums[3]));
      l += sum.x + sum.y;
      // the next block's number is two on while both tiles have one, else the next
      buf += j + 1 < both ? 2 : j + 1 == both ? 2 - i : 1;
      if (buf >= S::kScores) buf -= S::kScores, phase ^= 1;
    }
    if (ends[i] > w.first) added(ends[i] - 1);
    const bool whole = gridDim.y == 1;
    const long long at = (static_cast<long long>(w.q0 + index)) * p.n_heads + h;
    const float inv = !whole ? 1.f : l == 0.f ? 0.f : 1.f / l;
    const bool fix = *marked;
    if (tokens[i]) {
      // A lane has a row, and rows are apart in memory.  With 128 dims 32 rows of 256
      // bytes at a time go through the tile's queries, which nothing reads any more,
      // each 16 bytes at their place xor the row, and leave in whole rows: 1% of a
      // long prompt, 5% where keys are split.  (With 64 the registers for it cost the
      // loop above more than that.)
      uint8_t *stage = sq + i * S::kTile + (warp & 3) * (S::kTile / 4);
      uint8_t *dst = !live ? nullptr
                     : whole ? reinterpret_cast<uint8_t *>(static_cast<T *>(p.out) + (w.q0 + index) * p.out_stride + static_cast<long long>(h) * D)
                             : reinterpret_cast<uint8_t *>(p.part_o + (static_cast<long long>(blockIdx.y) * p.n_q * p.n_heads + at) * D);
      const auto put = [&](int chunk, uint4 v) {
        if constexpr (D == 64) {
          if (live) *reinterpret_cast<uint4 *>(dst + chunk * 16) = v;
        } else {
          *reinterpret_cast<uint4 *>(stage + lane * 256 + (chunk % 16 ^ (lane & 7)) * 16) = v;
        }
      };
      const auto leave = [&](int offset) {
        if constexpr (D == 64) return;
        __syncwarp();
#pragma unroll
        for (int r = 0; r < 32; r += 2) {
          const int from = r + lane / 16, chunk = lane % 16;
          uint8_t *to_row = reinterpret_cast<uint8_t *>(__shfl_sync(0xffffffffu, reinterpret_cast<unsigned long long>(dst), from));
          const uint4 v = *reinterpret_cast<const uint4 *>(stage + from * 256 + (chunk ^ (from & 7)) * 16);
          if (to_row) *reinterpret_cast<uint4 *>(to_row + offset + chunk * 16) = v;
        }
        __syncwarp();
      };
#pragma unroll 1
      for (int q = 0; q < D / 32; ++q) {
        float o[32];
        if (ends[i] > w.first) {
          tmem_ld32(to + q * 32, o);
          tmem_ld_wait();
          tmem_loaded(o);
        } else {
#pragma unroll
          for (int e = 0; e < 32; ++e) o[e] = 0.f;
        }
#pragma unroll
        for (int e = 0; e < 32; ++e) o[e] = l == 0.f ? 0.f : o[e] * inv;
        if (fix) {
#pragma unroll
          for (int e = 0; e < 32; ++e) {
            // added, not put in their place: the row may be NaN already, or hold the opposite infinity
            if (mark[q * 32 + e] < limit) o[e] = NAN;
            if (mark[D + q * 32 + e] < limit) o[e] += INFINITY;
            if (mark[2 * D + q * 32 + e] < limit) o[e] -= INFINITY;
          }
        }
        if (whole) {
#pragma unroll
          for (int e = 0; e < 4; ++e)
            put(q * 4 + e, make_uint4(X::pack(o[8 * e], o[8 * e + 1]), X::pack(o[8 * e + 2], o[8 * e + 3]), X::pack(o[8 * e + 4], o[8 * e + 5]),
                                      X::pack(o[8 * e + 6], o[8 * e + 7])));
          if (q + 1 == D / 32) leave(0);
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e)
            put(q * 8 + e, make_uint4(__float_as_uint(o[4 * e]), __float_as_uint(o[4 * e + 1]), __float_as_uint(o[4 * e + 2]), __float_as_uint(o[4 * e + 3])));
          if (q % 2) leave(q / 2 * 256);
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
  const PtRange range = pt_range(p, p.q_start[0], p.q_start[p.n_seq]);
  if (row < range.from || row >= range.to) return;
  float m = -INFINITY, l = 0.f;
  for (int k = 0; k < splits; ++k) m = fmaxf(m, p.part_ml[k * rows + at].x);
  const float c = p.scale * 1.4426950408889634f;
  float2 o[D / 64] = {};
  for (int k = 0; k < splits; ++k) {
    const float2 ml = p.part_ml[k * rows + at];
    // (nothing seen: zeros; only NaN scores: a sum of NaN)
    const float f = ml.x == -INFINITY ? (ml.y == 0.f ? 0.f : 1.f) : ex2((ml.x - m) * c);
    // What is not finite stays so however small the part's factor: an infinity times a 0 would be NaN.
    const auto share = [f](float v) { return isinf(v) ? v : f * v; };
    l += f * ml.y;
#pragma unroll
    for (int g = 0; g < D / 64; ++g) {
      const float2 v = *reinterpret_cast<const float2 *>(p.part_o + (k * rows + at) * D + g * 64 + lane * 2);
      o[g].x += share(v.x), o[g].y += share(v.y);
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
  // Few rows behind many keys: cut until there are four CTAs an SM, 1024 keys each at least.
  a.splits = static_cast<int>(std::max<int64_t>(1, std::min<int64_t>({max_k / 1024, kSms * 4 / std::max<int64_t>(1, a.items * heads), 64})));
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
        // a softmax warp waits for its registers, so the launch has to bring as many as the split counts on
        cudaFuncAttributes attr;
        if (e == cudaSuccess) e = cudaFuncGetAttributes(&attr, fn);
        if (e == cudaSuccess && attr.numRegs != PtShape<D>::kRegs) e = cudaErrorInvalidKernelImage;
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
  if (n_q > 1 << 30 || n_k > 1 << 30 || max_k > 1 << 30) return WF_ERR_UNSUPPORTED;
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
    const cuuint32_t box[3] = {64, 1, static_cast<cuuint32_t>(head_dim == 64 ? PtShape<64>::kKeys : PtShape<128>::kKeys)};
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
