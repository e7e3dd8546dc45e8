// What the attentions over the paged caches share: how a call is cut up, the
// operands of mma.sync, the join of warps, chunks and clusters, and the host's checks.
#pragma once
#include <algorithm>
#include <climits>

#include "wf_device.cuh"
#include "wf_ops.cuh"

namespace wf {

template <typename Pool>
struct PagedAttnParams {
  Pool pool;  // the cache at one layer, checked
  uint32_t block_bytes;
  const void *q;
  void *out;
  long long q_stride, out_stride;
  const int32_t *table, *len;
  int table_stride, n_seq, rps, group, causal, max_len;
  uint32_t group_inv;  // 2^32 / group, rounded up (group > 1)
  float scale;
  // A unit is (sequence, key/value head, group of query rows); it is cut into
  // chunks of positions, one CTA each, which a cluster or a second kernel joins.
  int tiles, row_groups, chunk, chunks, cluster;  // tiles: of 8 query rows
  float *part_o;    // [unit][chunks][rows][dim] weighted values of a chunk
  float2 *part_ml;  // [unit][chunks][rows] (maximum, sum)
  uint32_t *err;
  // Row of a key/value head -> query position.  Exact: row < 2^20, group <= 4096.
  __device__ __forceinline__ int row_of(int row) const { return group == 1 ? row : static_cast<int>(__umulhi(row, group_inv)); }
};

constexpr int kAtWarps = 4;
constexpr int kAtThreads = kAtWarps * 32;
constexpr int kAtLeast = 256;  // positions of a chunk at least: 64 a warp
constexpr int kAtCluster = 8;  // chunks that a cluster joins
constexpr int kAtShort = 2048; // positions of a chunk that two CTAs an SM may have
constexpr int kAtLongest = INT_MAX - 1023;  // a step past the last position is still an int
template <int G>
constexpr int kAtLd = G * 64 + 4;  // floats between the rows of a warp's results in shared memory

// None of these is volatile: the compiler may interleave independent chains.
__device__ __forceinline__ uint32_t transpose8x8(uint32_t v) {
  uint32_t r;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
  return r;
}
__device__ __forceinline__ void mma16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1, __nv_bfloat16) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1, __half) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t pack_f16(float2 v) {
  const __half2 h = __floats2half2_rn(v.x, v.y);
  return *reinterpret_cast<const uint32_t *>(&h);
}

__device__ __forceinline__ void bulk_load(void *smem_dst, const void *src, uint32_t bytes, uint64_t *bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(smem_u32(smem_dst)),
               "l"(reinterpret_cast<uint64_t>(src)), "r"(bytes), "r"(smem_u32(bar))
               : "memory");
}

// A row's limit: positions it sees.
template <typename P>
__device__ __forceinline__ int row_limit(const P &p, int row, int len) {
  return max(p.causal ? len - (p.rps - 1 - p.row_of(row)) : len, 0);
}
template <typename P>
__device__ __forceinline__ int clamp_len(const P &p, int len) { return min(max(len, 0), p.max_len); }

// A CTA's results from those of its warps, which they left in shared memory:
// of every warp and row the reference and sum, and the weighted values kAtLd
// floats apart (behind them there is room for one row's worth of each row).
template <typename T, int G, int NT, typename P>
__device__ __forceinline__ void paged_finish(const P &p, float *sm_m, float *sm_l, float *sm_o, int seen, int row0, int rows, int head, int seq) {
  using X = Type16<T>;
  constexpr int kRows = NT * 8, kLd = kAtLd<G>;
  // the warps join in order; kAtThreads / kRows threads a row, by four dims
  const bool whole = seen <= p.chunk;  // no other chunk has positions
  const size_t unit_at = static_cast<size_t>(blockIdx.x) * gridDim.z + blockIdx.z;
  float *cl_m = sm_o + kAtWarps * kRows * kLd, *cl_l = cl_m + kRows, *cl_o = cl_l + kRows;  // for the cluster
  constexpr int kTeam = kAtThreads / kRows;
  const int row = threadIdx.x / kTeam;
  if (row0 + row < rows) {
    float f[kAtWarps], mm = -INFINITY, ll = 0.f;
#pragma unroll
    for (int w = 0; w < kAtWarps; ++w) mm = fmaxf(mm, sm_m[w * kRows + row]);
#pragma unroll
    for (int w = 0; w < kAtWarps; ++w) {
      const float at = sm_m[w * kRows + row];
      f[w] = at == -INFINITY ? 0.f : ex2(at - mm);  // (a warp that saw nothing has zeros, one of NaN scores NaN)
      ll += f[w] * sm_l[w * kRows + row];
    }
    const float inv = ll == 0.f ? 0.f : 1.f / ll;
    const int j = p.row_of(row0 + row), h = head * p.group + row0 + row - j * p.group;
    T *dst = static_cast<T *>(p.out) + (static_cast<long long>(seq) * p.rps + j) * p.out_stride + h * (G * 64);
    const size_t part = (unit_at * p.chunks + blockIdx.y) * kRows + row;
    if (p.cluster) {
      if (threadIdx.x % kTeam == 0) cl_m[row] = mm, cl_l[row] = ll;
    } else if (!whole) {
      if (threadIdx.x % kTeam == 0) p.part_ml[part] = make_float2(mm, ll);
    }
#pragma unroll
    for (int d = threadIdx.x % kTeam * 4; d < G * 64; d += kTeam * 4) {
      float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int w = 0; w < kAtWarps; ++w) {
        const float4 u = *reinterpret_cast<const float4 *>(sm_o + (w * kRows + row) * kLd + d);
        v.x = fmaf(f[w], u.x, v.x), v.y = fmaf(f[w], u.y, v.y), v.z = fmaf(f[w], u.z, v.z), v.w = fmaf(f[w], u.w, v.w);
      }
      if (p.cluster) {
        *reinterpret_cast<float4 *>(cl_o + row * (G * 64) + d) = v;
      } else if (whole) {
        *reinterpret_cast<uint2 *>(dst + d) = make_uint2(X::pack(v.x * inv, v.y * inv), X::pack(v.z * inv, v.w * inv));
      } else {
        float2 *to = reinterpret_cast<float2 *>(p.part_o + part * (G * 64) + d);
        to[0] = make_float2(v.x, v.y), to[1] = make_float2(v.z, v.w);
      }
    }
  }
  if (!p.cluster) return;
  // the chunks of a unit are a cluster: every CTA joins some of the outputs over all of them, in chunk order
  cluster_sync();
  const int chunks = p.chunks, live_rows = min(rows - row0, kRows);
  for (int i = threadIdx.x * chunks + blockIdx.y; i < live_rows * G * 32; i += kAtThreads * chunks) {
    const int row = i / (G * 32), d = i % (G * 32) * 2;
    // no maximum: a chunk that the row sees nothing of, whose sums are zeros, or one of NaN scores, which stay NaN
    float cm[kAtCluster], cl[kAtCluster], ca[kAtCluster], cb[kAtCluster], mm = -INFINITY, ll = 0.f, a = 0.f, b = 0.f;
#pragma unroll
    for (int k = 0; k < kAtCluster; ++k) {
      if (k >= chunks) continue;
      const uint32_t at = dsmem_map(smem_u32(cl_o + row * (G * 64) + d), k);
      cm[k] = dsmem_ld_f32(dsmem_map(smem_u32(cl_m + row), k)), cl[k] = dsmem_ld_f32(dsmem_map(smem_u32(cl_l + row), k));
      ca[k] = dsmem_ld_f32(at), cb[k] = dsmem_ld_f32(at + 4);
      mm = fmaxf(mm, cm[k]);
    }
#pragma unroll
    for (int k = 0; k < kAtCluster; ++k) {
      if (k >= chunks) continue;
      const float f = cm[k] == -INFINITY ? 0.f : ex2(cm[k] - mm);
      ll += f * cl[k], a += f * ca[k], b += f * cb[k];
    }
    const float inv = ll == 0.f ? 0.f : 1.f / ll;
    const int j = p.row_of(row0 + row), h = head * p.group + row0 + row - j * p.group;
    T *dst = static_cast<T *>(p.out) + (static_cast<long long>(seq) * p.rps + j) * p.out_stride + h * (G * 64) + d;
    *reinterpret_cast<uint32_t *>(dst) = X::pack(a * inv, b * inv);
  }
  cluster_sync();  // no CTA leaves while another reads it
}

// Joins a row's chunks in order: a CTA per row, each of whose warps takes a
// quarter of the chunks, eight at a time, and whose lanes hold 2 G dims each.
// A chunk that the row sees nothing of holds zeros.
template <typename T, int G, int NT, typename P>
__global__ void __launch_bounds__(kAtThreads) paged_join_kernel(const P p) {
  using X = Type16<T>;
  constexpr int kRows = NT * 8, kAhead = 8;
  __shared__ float2 part[kAtWarps][G][32];
  __shared__ float2 part_ml[kAtWarps];
  pdl_wait();
  pdl_launch_dependents();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int head = blockIdx.x % p.pool.heads, seq = blockIdx.x / p.pool.heads;
  const int group = blockIdx.y, row = blockIdx.z, row0 = group * kRows, rows = p.rps * p.group;
  if (row0 + row >= rows) return;
  const int seen = row_limit(p, min(row0 + kRows, rows) - 1, clamp_len(p, p.len[seq]));
  if (seen <= p.chunk) return;
  const int chunks = (seen + p.chunk - 1) / p.chunk, per = (chunks + kAtWarps - 1) / kAtWarps;
  const size_t task = (static_cast<size_t>(blockIdx.x) * p.row_groups + group) * p.chunks;
  const int last = min(chunks, (warp + 1) * per);
  float m = -INFINITY, l = 0.f;
  float2 o[G] = {};
  for (int k = warp * per; k < last; k += kAhead) {
    float2 ml[kAhead], v[kAhead][G];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const size_t at = (task + k + i) * kRows + row;
      const bool has = k + i < last;
      ml[i] = has ? p.part_ml[at] : make_float2(-INFINITY, 0.f);
#pragma unroll
      for (int g = 0; g < G; ++g) v[i][g] = !has ? make_float2(0.f, 0.f) : *reinterpret_cast<const float2 *>(p.part_o + at * (G * 64) + g * 64 + lane * 2);
    }
    float top = m;
#pragma unroll
    for (int i = 0; i < kAhead; ++i) top = fmaxf(top, ml[i].x);
    const float keep = m == -INFINITY ? 0.f : ex2(m - top);
    m = top, l *= keep;
#pragma unroll
    for (int g = 0; g < G; ++g) o[g].x *= keep, o[g].y *= keep;
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const float f = ml[i].x == -INFINITY ? 0.f : ex2(ml[i].x - m);
      l += f * ml[i].y;
#pragma unroll
      for (int g = 0; g < G; ++g) o[g].x += f * v[i][g].x, o[g].y += f * v[i][g].y;
    }
  }
  if (lane == 0) part_ml[warp] = make_float2(m, l);
#pragma unroll
  for (int g = 0; g < G; ++g) part[warp][g][lane] = o[g];
  __syncthreads();
  if (warp >= G) return;
  float mm = part_ml[0].x, ll = 0.f;
#pragma unroll
  for (int w = 1; w < kAtWarps; ++w) mm = fmaxf(mm, part_ml[w].x);
  float2 sum = make_float2(0.f, 0.f);
#pragma unroll
  for (int w = 0; w < kAtWarps; ++w) {
    const float f = part_ml[w].x == -INFINITY ? 0.f : ex2(part_ml[w].x - mm);
    ll += f * part_ml[w].y;
    sum.x += f * part[w][warp][lane].x, sum.y += f * part[w][warp][lane].y;
  }
  const float inv = ll == 0.f ? 0.f : 1.f / ll;
  const int j = p.row_of(row0 + row), h = head * p.group + row0 + row - j * p.group;
  T *dst = static_cast<T *>(p.out) + (static_cast<long long>(seq) * p.rps + j) * p.out_stride + h * (G * 64) + warp * 64 + lane * 2;
  *reinterpret_cast<uint32_t *>(dst) = X::pack(sum.x * inv, sum.y * inv);
}

// How a call is cut up: a function of its sizes alone.
struct AtPlan {
  int tiles;            // 8 query rows each
  int64_t row_groups, units;
  int chunk, chunks;
};
inline AtPlan at_plan(int64_t n_seq, int64_t heads, int64_t rows, int max_len) {
  AtPlan a;
  a.tiles = rows > 8 ? 2 : 1;
  a.row_groups = (rows + a.tiles * 8 - 1) / (a.tiles * 8);
  a.units = n_seq * heads * a.row_groups;
  // A CTA's four warps take at least 64 positions each.  Short sequences: cut
  // into even chunks, a cluster each, until there are two CTAs an SM, for a
  // cluster stays until its last is done (1500 positions, 20 heads: 50 sequences
  // x 9 rows 41 us, 8 x 5 rows 10.3; cut until there are eight CTAs an SM 54 and
  // 13.8).  Long ones: eight CTAs an SM, so that SMs whose sequences are short
  // find other work (12 sequences of 3000 to 9000 positions, 32 heads on 8: 32 us
  // against 34; 6 of 5000 to 65001: 38 against 108).
  const auto cut = [&](int64_t want) {
    const int64_t least = kAtLeast, longest = max_len;
    const int64_t per = std::max(least, (a.units * longest + want - 1) / want);
    const int64_t chunks = (longest + per - 1) / per;
    const int64_t chunk = (longest + chunks * least - 1) / (chunks * least) * least;
    a.chunk = static_cast<int>(std::min<int64_t>(chunk, 1 << 30));
    a.chunks = static_cast<int>((longest + a.chunk - 1) / a.chunk);
  };
  cut(kSms * 2);
  if (a.chunks > kAtCluster || a.chunk > kAtShort) cut(kSms * 8);
  return a;
}

inline size_t paged_scratch_bytes(int32_t n_seq, int32_t rps, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim, int32_t max_len) {
  if (n_seq <= 0 || rps <= 0 || n_heads <= 0 || n_kv_heads <= 0 || n_heads % n_kv_heads || max_len <= 0 || max_len > kAtLongest ||
      (head_dim != 64 && head_dim != 128))
    return 0;
  const AtPlan a = at_plan(n_seq, n_kv_heads, static_cast<int64_t>(rps) * (n_heads / n_kv_heads), max_len);
  return a.chunks > kAtCluster ? static_cast<size_t>(a.units * a.chunks * a.tiles * 8) * (head_dim + 2) * sizeof(float) : 0;
}

// Host checks of a call's arguments behind its pool, and its parameters.
template <typename CPool, typename P>
wf_status paged_args(const CPool &pool, const void *d_q, int64_t q_stride, const int32_t *d_table, int32_t table_stride, const int32_t *d_len,
                     int32_t n_seq, int32_t rps, int32_t n_heads, int32_t causal, float scale, int32_t max_len, void *d_out, int64_t out_stride,
                     void *d_scratch, size_t scratch_bytes, uint32_t *d_err, P *p) {
  const int64_t d = static_cast<int64_t>(n_heads) * pool.head_dim;
  if (!d_q || !d_table || !d_len || !d_out || n_seq <= 0 || rps <= 0 || n_heads <= 0 || n_heads % pool.n_kv_heads || max_len <= 0 ||
      table_stride < 0 || !aligned16(d_q) || !aligned16(d_out) || q_stride % 8 || out_stride % 8 || q_stride < d || out_stride < d ||
      !(scale == scale))
    return WF_ERR_INVALID;
  // every position up to max_len needs a table column (stride 0: one row that the caller made long enough)
  if (table_stride && static_cast<int64_t>(table_stride) * pool.block_size < max_len) return WF_ERR_INVALID;
  const int group = n_heads / pool.n_kv_heads;
  const int64_t rows = static_cast<int64_t>(rps) * group;
  if (static_cast<int64_t>(n_seq) * pool.n_kv_heads > INT32_MAX || rows > 65535 * 8LL || group > 4096 || max_len > kAtLongest)
    return WF_ERR_UNSUPPORTED;
  p->q = d_q, p->out = d_out, p->q_stride = q_stride, p->out_stride = out_stride;
  p->table = d_table, p->len = d_len, p->table_stride = table_stride;
  p->n_seq = n_seq, p->rps = rps, p->group = group;
  p->group_inv = static_cast<uint32_t>(((1ull << 32) + group - 1) / group);
  p->causal = causal != 0, p->max_len = max_len, p->scale = scale, p->err = d_err;
  const AtPlan a = at_plan(n_seq, pool.n_kv_heads, rows, max_len);
  if (a.chunks > 65535) return WF_ERR_UNSUPPORTED;
  p->tiles = a.tiles, p->row_groups = static_cast<int>(a.row_groups);
  p->chunk = a.chunk, p->chunks = a.chunks;
  p->cluster = p->chunks > 1 && p->chunks <= kAtCluster;
  if (p->chunks > 1 && !p->cluster) {
    if (!d_scratch || !aligned16(d_scratch)) return WF_ERR_INVALID;
    if (scratch_bytes < paged_scratch_bytes(n_seq, rps, n_heads, pool.n_kv_heads, pool.head_dim, max_len)) return WF_ERR_CAPACITY;
    p->part_o = static_cast<float *>(d_scratch);
    p->part_ml = reinterpret_cast<float2 *>(p->part_o + a.units * a.chunks * a.tiles * 8 * pool.head_dim);
  }
  return WF_OK;
}

// One call: the attention kernel `fn`, and the join where its chunks are more than a cluster's.
template <typename T, int G, int NT, typename P>
cudaError_t paged_launch(const void *fn, size_t smem, PerDevice &ready, const P &p, cudaStream_t s) {
  cudaError_t e = cudaSuccess;
  if (!ready.get(current_device(), [&]() -> int {
        e = cudaFuncSetAttribute(fn, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(smem));
        if (e == cudaSuccess) e = prefer_max_shared(fn);
        return e == cudaSuccess;
      }))
    return e;
  const dim3 grid(p.n_seq * p.pool.heads, p.chunks, p.row_groups);
  void *args[] = {const_cast<P *>(&p)};
  e = launch_pdl(fn, grid, kAtThreads, smem, args, s, p.cluster ? p.chunks : 1);
  if (e == cudaSuccess && p.chunks > 1 && !p.cluster)
    e = launch_pdl(reinterpret_cast<const void *>(paged_join_kernel<T, G, NT, P>), dim3(grid.x, p.row_groups, NT * 8), kAtThreads, 0, args, s);
  return e;
}

}  // namespace wf
