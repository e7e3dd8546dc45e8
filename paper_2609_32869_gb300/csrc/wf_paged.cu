// The paged 4-bit cache around its attention: block tables and slot maps from
// request lengths, rows into and out of the cache, and the reordering of the
// beams' tables after a selection.
#include <algorithm>

#include "wf_device.cuh"
#include "wf_kv4.cuh"

namespace wf {

// ----------------------------------------------------- tables and slots --
struct PlanParams {
  const int32_t *old_len, *new_len, *free_ids, *n_free;
  int32_t *table, *offsets, *slots, *len, *n_free_out;
  int n, bs_shift, n_blocks, stride, cap;
  uint32_t *err;
};
constexpr int kPlanThreads = 256;
constexpr int kPlanOwned = 64;  // requests of one CTA

// Inclusive scan over the CTA of two counts at a time.
__device__ __forceinline__ void block_scan2(long long &a, long long &b, long long (*sm)[2], long long &ta, long long &tb) {
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5, nw = blockDim.x >> 5;
#pragma unroll
  for (int off = 1; off < 32; off <<= 1) {
    const long long pa = __shfl_up_sync(0xffffffffu, a, off), pb = __shfl_up_sync(0xffffffffu, b, off);
    if (lane >= off) a += pa, b += pb;
  }
  __syncthreads();
  if (lane == 31) sm[w][0] = a, sm[w][1] = b;
  __syncthreads();
  ta = tb = 0;
  for (int i = 0; i < nw; ++i) {
    if (i < w) a += sm[i][0], b += sm[i][1];
    ta += sm[i][0], tb += sm[i][1];
  }
}

// Every CTA scans all the lengths (n is a few hundred; the scan is a few
// passes of 256) and keeps the prefixes of the requests it owns, i = blockIdx
// mod gridDim; then it fills those requests' table columns and slots.  Counts
// only grow along the requests, so the granted ones are a prefix.
__global__ void __launch_bounds__(kPlanThreads) page_plan_kernel(const PlanParams p) {
  pdl_wait();
  pdl_launch_dependents();
  __shared__ long long sm[kPlanThreads / 32][2];
  __shared__ int own_block[kPlanOwned], own_tok[kPlanOwned], own_ok[kPlanOwned];
  const int bs = 1 << p.bs_shift;
  int nf = *p.n_free;
  uint32_t err = 0;
  if (nf < 0 || nf > p.n_blocks) nf = 0, err = WF_DEV_ERR_PAGE;
  long long done_b = 0, done_t = 0;    // of the requests before this pass
  long long grant_b = 0, grant_t = 0;  // of the granted ones
  for (int i0 = 0; i0 < p.n; i0 += kPlanThreads) {
    const int i = i0 + threadIdx.x;
    long long nb = 0, nt = 0;
    bool valid = false;
    if (i < p.n) {
      const int a = p.old_len[i], b = p.new_len[i];
      valid = a >= 0 && b >= a && (static_cast<long long>(b) + bs - 1) >> p.bs_shift <= p.stride;
      if (valid) {
        nt = b - a;
        nb = ((static_cast<long long>(b) + bs - 1) >> p.bs_shift) - ((static_cast<long long>(a) + bs - 1) >> p.bs_shift);
      } else {
        err |= WF_DEV_ERR_PAGE;
      }
    }
    long long cb = nb, ct = nt, tb, tt;
    block_scan2(cb, ct, sm, tb, tt);
    cb += done_b, ct += done_t;
    const bool ok = valid && cb <= nf && ct <= p.cap;
    if (valid && !ok) err |= WF_DEV_ERR_CAPACITY;
    if (i < p.n && i % gridDim.x == blockIdx.x) {
      const int k = i / gridDim.x;
      own_block[k] = ok ? static_cast<int>(cb - nb) : 0;
      own_tok[k] = static_cast<int>(min(ct - nt, static_cast<long long>(p.cap)));
      own_ok[k] = ok;
    }
    done_b += tb, done_t += tt;
    // the granted prefix: the largest granted counts of this pass
    long long gb = ok ? cb : 0, gt = ok ? ct : 0;
#pragma unroll
    for (int off = 16; off; off >>= 1) {
      gb = max(gb, __shfl_xor_sync(0xffffffffu, gb, off));
      gt = max(gt, __shfl_xor_sync(0xffffffffu, gt, off));
    }
    __syncthreads();
    if ((threadIdx.x & 31) == 0) sm[threadIdx.x >> 5][0] = gb, sm[threadIdx.x >> 5][1] = gt;
    __syncthreads();
    for (int w = 0; w < kPlanThreads / 32; ++w) grant_b = max(grant_b, sm[w][0]), grant_t = max(grant_t, sm[w][1]);
  }
  __syncthreads();
  const int total = static_cast<int>(grant_t);
  if (blockIdx.x == 0) {
    if (threadIdx.x == 0) {
      p.offsets[p.n] = total;
      *p.n_free_out = nf - static_cast<int>(grant_b);
    }
    if (err) set_error(p.err, err);
  }
  for (int i = blockIdx.x, k = 0; i < p.n; i += gridDim.x, ++k) {
    const int a = p.old_len[i], b = p.new_len[i];
    const bool ok = own_ok[k];
    // requests after the first that did not fit start where the granted ones end
    const int at = min(own_tok[k], total);
    if (threadIdx.x == 0) {
      p.offsets[i] = at;
      p.len[i] = ok ? b : a;
    }
    if (!ok) continue;
    int32_t *row = p.table + static_cast<size_t>(i) * p.stride;
    const int c0 = (a + bs - 1) >> p.bs_shift, c1 = (b + bs - 1) >> p.bs_shift;
    const int32_t *ids = p.free_ids + (nf - 1 - own_block[k]);
    for (int c = c0 + threadIdx.x; c < c1; c += kPlanThreads) row[c] = ids[-(c - c0)];
    const int part = (a & (bs - 1)) ? row[a >> p.bs_shift] : 0;  // the block that old length ends in
    for (int t = threadIdx.x; t < b - a; t += kPlanThreads) {
      const int pos = a + t, c = pos >> p.bs_shift;
      const int id = c < c0 ? part : ids[-(c - c0)];
      p.slots[at + t] = id < 0 || id >= p.n_blocks ? -1 : (id << p.bs_shift) + (pos & (bs - 1));
      if (id < 0 || id >= p.n_blocks) set_error(p.err, WF_DEV_ERR_PAGE);
    }
  }
  for (int t = total + blockIdx.x * kPlanThreads + threadIdx.x; t < p.cap; t += gridDim.x * kPlanThreads) p.slots[t] = -1;
}

// ------------------------------------------------------ rows in and out --
struct StoreParams {
  Kv4Pool pool;
  const void *k, *v;
  void *k_out, *v_out;
  long long k_stride, v_stride;
  const int32_t *slots;
  int n;
  uint32_t *err;
};
constexpr int kRowThreads = 256;

// Eight lanes quantise one group of a row: 8 values each, the extremes by
// three exchanges.
template <typename T>
__global__ void __launch_bounds__(kRowThreads) kv4_store_kernel(const StoreParams p) {
  pdl_wait();
  pdl_launch_dependents();
  using X = Kv4Type<T>;
  const int slabs = p.pool.heads * p.pool.groups;
  const long long units = static_cast<long long>(p.n) * slabs * 2;
  const int j = threadIdx.x & 7;
  const long long step = static_cast<long long>(gridDim.x) * (kRowThreads / 8);
  // whole warps iterate together: the exchanges below need all their lanes
  const long long first = static_cast<long long>(blockIdx.x) * (kRowThreads / 8) + (threadIdx.x >> 3);
  for (long long u = first; u - (first & 3) < units; u += step) {
    const bool in = u < units;
    const long long uu = in ? u : units - 1;
    const int slab = static_cast<int>(uu % slabs);
    const int is_v = static_cast<int>(uu / slabs % 2);
    const int row = static_cast<int>(uu / slabs / 2);
    const int slot = p.slots[row];
    const T *src = static_cast<const T *>(is_v ? p.v : p.k) + row * (is_v ? p.v_stride : p.k_stride) + slab * 64 + j * 8;
    const uint4 w = *reinterpret_cast<const uint4 *>(src);
    float x[8] = {X::lo(w.x), X::hi(w.x), X::lo(w.y), X::hi(w.y), X::lo(w.z), X::hi(w.z), X::lo(w.w), X::hi(w.w)};
    float hi = x[0], lo = x[0];
    bool fine = true;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      hi = fmaxf(hi, x[i]), lo = fminf(lo, x[i]);
      fine &= isfinite(x[i]);
    }
#pragma unroll
    for (int off = 1; off < 8; off <<= 1) {
      hi = fmaxf(hi, __shfl_xor_sync(0xffffffffu, hi, off));
      lo = fminf(lo, __shfl_xor_sync(0xffffffffu, lo, off));
    }
    fine = ((__ballot_sync(0xffffffffu, fine) >> (threadIdx.x & 24)) & 0xffu) == 0xffu;
    // halves first: max - min may pass the type's range
    const float s = fine ? X::round((0.5f * hi - 0.5f * lo) / 7.5f) : NAN;
    const float z = fine ? X::round(hi - 7.f * s) : NAN;  // 7 s is exact in fp32
    uint32_t codes = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float c = s > 0.f ? fminf(fmaxf(rintf((x[i] - z) / s), -8.f), 7.f) : 0.f;
      codes |= static_cast<uint32_t>(static_cast<int>(c) + 8) << (4 * i);
    }
    if (!in || slot < 0) continue;
    const int block = slot >> p.pool.bs_shift;
    if (block >= p.pool.n_blocks) {
      if (j == 0) set_error(p.err, WF_DEV_ERR_PAGE);
      continue;
    }
    const int pos = slot & (p.pool.bs - 1), at = pos & 15;
    unsigned char *rec = kv4_record(p.pool, block, 0, slab, pos >> 4);
    if (is_v) {
      *reinterpret_cast<uint16_t *>(rec + kv4_val_offset(at, j, 0)) = static_cast<uint16_t>(codes);
      *reinterpret_cast<uint16_t *>(rec + kv4_val_offset(at, j, 1)) = static_cast<uint16_t>(codes >> 16);
    } else {
      *reinterpret_cast<uint32_t *>(rec + at * 32 + j * 4) = codes;
    }
    if (j == 0) *reinterpret_cast<uint32_t *>(rec + kv4_scale_offset(at, is_v)) = X::pack(s, z);
  }
}

template <typename T>
__global__ void __launch_bounds__(kRowThreads) kv4_load_kernel(const StoreParams p) {
  pdl_wait();
  pdl_launch_dependents();
  using X = Kv4Type<T>;
  const int slabs = p.pool.heads * p.pool.groups;
  const long long units = static_cast<long long>(p.n) * slabs * 2;
  const int j = threadIdx.x & 7;
  for (long long u = static_cast<long long>(blockIdx.x) * (kRowThreads / 8) + (threadIdx.x >> 3); u < units;
       u += static_cast<long long>(gridDim.x) * (kRowThreads / 8)) {
    const int slab = static_cast<int>(u % slabs);
    const int is_v = static_cast<int>(u / slabs % 2);
    const int row = static_cast<int>(u / slabs / 2);
    const int slot = p.slots[row];
    uint4 out = {0, 0, 0, 0};
    const int block = slot >> p.pool.bs_shift;
    if (slot >= 0 && block < p.pool.n_blocks) {
      const int pos = slot & (p.pool.bs - 1), at = pos & 15;
      const unsigned char *rec = kv4_record(p.pool, block, 0, slab, pos >> 4);
      uint32_t codes;
      if (is_v)
        codes = *reinterpret_cast<const uint16_t *>(rec + kv4_val_offset(at, j, 0)) |
                static_cast<uint32_t>(*reinterpret_cast<const uint16_t *>(rec + kv4_val_offset(at, j, 1))) << 16;
      else
        codes = *reinterpret_cast<const uint32_t *>(rec + at * 32 + j * 4);
      const uint32_t sz = *reinterpret_cast<const uint32_t *>(rec + kv4_scale_offset(at, is_v));
      const float s = X::lo(sz), z = X::hi(sz);
      float x[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = fmaf(s, static_cast<float>(static_cast<int>(codes >> (4 * i) & 15) - 8), z);
      out = {X::pack(x[0], x[1]), X::pack(x[2], x[3]), X::pack(x[4], x[5]), X::pack(x[6], x[7])};
    } else if (slot >= 0 && j == 0) {
      set_error(p.err, WF_DEV_ERR_PAGE);
    }
    T *dst = static_cast<T *>(is_v ? p.v_out : p.k_out) + row * (is_v ? p.v_stride : p.k_stride) + slab * 64 + j * 8;
    *reinterpret_cast<uint4 *>(dst) = out;
  }
}

// ---------------------------------------------------------- reordering --
struct ReorderParams {
  Kv4Pool pool;
  long long layer_stride, block_bytes;
  int n_layers;
  const int32_t *table_in, *len, *parent, *n_free;
  int32_t *table_out, *free_ids, *n_free_out;
  int stride, n_req, W;
  int32_t *gone, *gone_n, *moves, *n_free_copy;  // scratch
  uint32_t *err;
};
constexpr int kReorderThreads = 256;

// One CTA per request: its table columns (each by one thread, which reads the
// column before it writes it), the ids that no beam holds any more in order,
// and the copies of last blocks that the second kernel makes.
__global__ void __launch_bounds__(kReorderThreads) beam_tables_kernel(const ReorderParams p) {
  pdl_wait();
  pdl_launch_dependents();
  const int W = p.W, req = blockIdx.x, tid = threadIdx.x;
  __shared__ int par[WF_MAX_BEAMS], from[WF_MAX_BEAMS], over_s;
  __shared__ int wsum[kReorderThreads / 32];
  const int32_t *in = p.table_in + static_cast<size_t>(req) * W * p.stride;
  int32_t *out = p.table_out + static_cast<size_t>(req) * W * p.stride;
  int32_t *gone = p.gone + static_cast<size_t>(req) * W * p.stride;
  int len = p.len[static_cast<size_t>(req) * W];
  const int bs = p.pool.bs;
  uint32_t err = 0;
  if (len < 0 || (static_cast<long long>(len) + bs - 1) / bs > p.stride) {
    err |= WF_DEV_ERR_PAGE;
    len = len < 0 ? 0 : p.stride * bs;
  }
  const int full = len / bs, rem = len % bs;
  if (tid < W) {
    int v = p.parent[static_cast<size_t>(req) * W + tid];
    if (v < -1 || v >= W) err |= WF_DEV_ERR_PAGE, v = -1;
    par[tid] = v;
  }
  __syncthreads();
  if (tid == 0) {
    uint32_t has_child = 0, keeps = 0;
    int over = 1;
    for (int w = 0; w < W; ++w) {
      const int v = par[w];
      if (v < 0) continue;
      over = 0;
      if (!(has_child >> v & 1)) keeps |= 1u << w;
      has_child |= 1u << v;
    }
    // the k-th beam that keeps nothing takes the last block of the k-th without children
    uint32_t dead = ~has_child & ((1u << W) - 1);
    for (int w = 0; w < W; ++w) {
      if (keeps >> w & 1) {
        from[w] = par[w];
      } else {
        from[w] = __ffs(dead) - 1;
        dead &= dead - 1;
      }
    }
    over_s = over;
    if (req == 0) *p.n_free_copy = *p.n_free;
  }
  __syncthreads();
  const bool over = over_s;
  // copies: (source, destination) of each child that takes another beam's block
  if (tid < W) {
    int src = -1, dst = -1;
    if (rem && par[tid] >= 0 && from[tid] != par[tid]) {
      src = in[par[tid] * p.stride + full];
      dst = in[from[tid] * p.stride + full];
      if (src < 0 || src >= p.pool.n_blocks || dst < 0 || dst >= p.pool.n_blocks) err |= WF_DEV_ERR_PAGE, src = dst = -1;
    }
    int32_t *m = p.moves + (static_cast<size_t>(req) * W + tid) * 4;
    m[0] = src, m[1] = dst, m[2] = (rem + 15) / 16, m[3] = 0;
  }
  __syncthreads();
  int base = 0;
  const int cols = full + (rem ? 1 : 0);
  for (int c0 = 0; c0 < cols; c0 += kReorderThreads) {
    const int c = c0 + tid;
    int old[WF_MAX_BEAMS], now[WF_MAX_BEAMS];
    uint32_t dead = 0;
    if (c < cols) {
#pragma unroll
      for (int w = 0; w < WF_MAX_BEAMS; ++w)
        if (w < W) old[w] = in[static_cast<size_t>(w) * p.stride + c];
      for (int w = 0; w < W; ++w) {
        int id = -1;
        const int f = c < full ? par[w] : (over ? -1 : from[w]);
#pragma unroll
        for (int q = 0; q < WF_MAX_BEAMS; ++q)
          if (q == f) id = old[q];
#pragma unroll
        for (int q = 0; q < WF_MAX_BEAMS; ++q)
          if (q == w) now[q] = id;
        out[static_cast<size_t>(w) * p.stride + c] = id;
      }
#pragma unroll
      for (int w = 0; w < WF_MAX_BEAMS; ++w) {
        if (w >= W || old[w] < 0) continue;
        bool held = false;
#pragma unroll
        for (int q = 0; q < WF_MAX_BEAMS; ++q)
          if (q < W) held |= now[q] == old[w] || (q < w && old[q] == old[w]);
        if (!held) dead |= 1u << w;
      }
    }
    int cnt = __popc(dead), scan = cnt;
    const int lane = tid & 31, wp = tid >> 5;
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
      const int v = __shfl_up_sync(0xffffffffu, scan, off);
      if (lane >= off) scan += v;
    }
    if (lane == 31) wsum[wp] = scan;
    __syncthreads();
    int total = 0, before = 0;
    for (int i = 0; i < kReorderThreads / 32; ++i) {
      if (i < wp) before += wsum[i];
      total += wsum[i];
    }
    int at = base + before + scan - cnt;
#pragma unroll
    for (int w = 0; w < WF_MAX_BEAMS; ++w)
      if (dead >> w & 1) gone[at++] = old[w];
    base += total;
    __syncthreads();
  }
  if (tid == 0) p.gone_n[req] = base;
  if (err) set_error(p.err, err);
}

// grid (n_req * W, layers): the copies of last blocks, 16 positions at a time;
// in layer 0 the first CTA of a request also pushes its freed ids.
__global__ void __launch_bounds__(kReorderThreads) beam_moves_kernel(const ReorderParams p) {
  pdl_wait();
  pdl_launch_dependents();
  const int req = blockIdx.x / p.W;
  const int32_t *m = p.moves + static_cast<size_t>(blockIdx.x) * 4;
  if (m[0] >= 0) {
    const int chunk = m[2] * (kKv4Rec / 16);  // 16-byte pieces of a slab that are in use
    const int slabs = p.pool.heads * p.pool.groups, per = (p.pool.bs >> 4) * (kKv4Rec / 16);
    unsigned char *layer = p.pool.base + static_cast<long long>(blockIdx.y) * p.layer_stride;
    const uint4 *src = reinterpret_cast<const uint4 *>(layer + m[0] * p.block_bytes);
    uint4 *dst = reinterpret_cast<uint4 *>(layer + m[1] * p.block_bytes);
    for (int i = threadIdx.x; i < slabs * chunk; i += kReorderThreads) {
      const int at = i / chunk * per + i % chunk;
      dst[at] = src[at];
    }
  }
  if (blockIdx.y != 0 || blockIdx.x % p.W != 0) return;
  __shared__ int sums[2][kReorderThreads / 32];
  int before = 0, total = 0;
  for (int i = threadIdx.x; i < p.n_req; i += kReorderThreads) {
    const int v = p.gone_n[i];
    total += v;
    if (i < req) before += v;
  }
#pragma unroll
  for (int off = 16; off; off >>= 1) {
    before += __shfl_xor_sync(0xffffffffu, before, off);
    total += __shfl_xor_sync(0xffffffffu, total, off);
  }
  if ((threadIdx.x & 31) == 0) sums[0][threadIdx.x >> 5] = before, sums[1][threadIdx.x >> 5] = total;
  __syncthreads();
  before = total = 0;
  for (int i = 0; i < kReorderThreads / 32; ++i) before += sums[0][i], total += sums[1][i];
  int nf = *p.n_free_copy;
  const bool bad = nf < 0 || static_cast<long long>(nf) + total > p.pool.n_blocks;
  if (bad) {  // more ids than the stack holds: none is pushed
    if (threadIdx.x == 0) set_error(p.err, WF_DEV_ERR_PAGE);
  } else {
    const int32_t *gone = p.gone + static_cast<size_t>(req) * p.W * p.stride;
    for (int i = threadIdx.x; i < p.gone_n[req]; i += kReorderThreads) p.free_ids[nf + before + i] = gone[i];
  }
  if (req == 0 && threadIdx.x == 0) *p.n_free_out = bad ? nf : nf + total;
}

static int sm_count() {
  static const int n = [] {
    int dev = 0, v = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&v, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess)
      return 0;
    return v;
  }();
  return n;
}

}  // namespace wf

using namespace wf;

extern "C" {

size_t wf_kv4_block_bytes(int32_t block_size, int32_t n_kv_heads, int32_t head_dim) {
  return kv4_shape_ok(block_size, n_kv_heads, head_dim) ? kv4_block_bytes(block_size, n_kv_heads, head_dim) : 0;
}

wf_status wf_page_plan(const int32_t *d_old_len, const int32_t *d_new_len, int32_t n, int32_t block_size,
                       const int32_t *d_free, int32_t n_blocks, const int32_t *d_n_free, int32_t *d_table,
                       int32_t table_stride, int32_t *d_offsets, int32_t *d_slots, int32_t slots_cap, int32_t *d_len,
                       int32_t *d_n_free_out, uint32_t *d_err, void *stream) {
  if (!d_old_len || !d_new_len || !d_free || !d_n_free || !d_table || !d_offsets || !d_len || !d_n_free_out ||
      (!d_slots && slots_cap > 0) || n <= 0 || n_blocks <= 0 || table_stride <= 0 || slots_cap < 0)
    return WF_ERR_INVALID;
  if (d_len == d_old_len || d_len == d_new_len || d_n_free_out == d_n_free) return WF_ERR_INVALID;
  if (block_size != 16 && block_size != 32 && block_size != 64) return WF_ERR_UNSUPPORTED;
  if (static_cast<int64_t>(n_blocks) * block_size > INT32_MAX || static_cast<int64_t>(table_stride) * block_size > INT32_MAX ||
      n > (1 << 22))
    return WF_ERR_INVALID;
  const int sms = sm_count();
  if (!sms) return WF_ERR_CUDA;
  PlanParams p = {d_old_len, d_new_len, d_free,     d_n_free,     d_table,   d_offsets, d_slots, d_len,
                  d_n_free_out, n,      block_size == 16 ? 4 : (block_size == 32 ? 5 : 6), n_blocks, table_stride, slots_cap, d_err};
  const int grid = std::max(std::min(n, 4 * sms), (n + kPlanOwned - 1) / kPlanOwned);
  void *args[] = {&p};
  return launch_pdl(reinterpret_cast<const void *>(page_plan_kernel), grid, kPlanThreads, 0, args,
                    static_cast<cudaStream_t>(stream)) == cudaSuccess
             ? WF_OK
             : WF_ERR_CUDA;
}

static wf_status rows_check(const wf_kv4_pool *pool, int32_t layer, const void *k, int64_t ks, const void *v, int64_t vs,
                            const int32_t *slots, int32_t n, StoreParams *p) {
  const wf_status st = kv4_pool_check(pool, layer, &p->pool, nullptr);
  if (st != WF_OK) return st;
  const int64_t d = static_cast<int64_t>(pool->n_kv_heads) * pool->head_dim;
  if (!k || !v || !slots || n < 0 || !aligned16(k) || !aligned16(v) || ks % 8 || vs % 8 || ks < d || vs < d)
    return WF_ERR_INVALID;
  p->k_stride = ks;
  p->v_stride = vs;
  p->slots = slots;
  p->n = n;
  return WF_OK;
}
static wf_status rows_launch(const void *fn, StoreParams *p, void *stream) {
  if (p->n == 0) return WF_OK;
  const int sms = sm_count();
  if (!sms) return WF_ERR_CUDA;
  const long long units = static_cast<long long>(p->n) * p->pool.heads * p->pool.groups * 2;
  const long long want = (units + kRowThreads / 8 - 1) / (kRowThreads / 8);
  void *args[] = {p};
  return launch_pdl(fn, static_cast<unsigned>(std::min<long long>(want, 32LL * sms)), kRowThreads, 0, args,
                    static_cast<cudaStream_t>(stream)) == cudaSuccess
             ? WF_OK
             : WF_ERR_CUDA;
}

wf_status wf_kv4_store(const wf_kv4_pool *pool, int32_t layer, const void *d_k, int64_t k_stride, const void *d_v,
                       int64_t v_stride, const int32_t *d_slots, int32_t n, uint32_t *d_err, void *stream) {
  StoreParams p = {};
  const wf_status st = rows_check(pool, layer, d_k, k_stride, d_v, v_stride, d_slots, n, &p);
  if (st != WF_OK) return st;
  p.k = d_k, p.v = d_v, p.err = d_err;
  return rows_launch(pool->dtype == WF_F16 ? reinterpret_cast<const void *>(kv4_store_kernel<__half>)
                                           : reinterpret_cast<const void *>(kv4_store_kernel<__nv_bfloat16>),
                     &p, stream);
}

wf_status wf_kv4_load(const wf_kv4_pool *pool, int32_t layer, const int32_t *d_slots, int32_t n, void *d_k, int64_t k_stride,
                      void *d_v, int64_t v_stride, uint32_t *d_err, void *stream) {
  StoreParams p = {};
  const wf_status st = rows_check(pool, layer, d_k, k_stride, d_v, v_stride, d_slots, n, &p);
  if (st != WF_OK) return st;
  p.k_out = d_k, p.v_out = d_v, p.err = d_err;
  return rows_launch(pool->dtype == WF_F16 ? reinterpret_cast<const void *>(kv4_load_kernel<__half>)
                                           : reinterpret_cast<const void *>(kv4_load_kernel<__nv_bfloat16>),
                     &p, stream);
}

// scratch: freed ids [n_req][beams * stride], their counts [n_req], copies
// [n_req * beams][4], the free count
size_t wf_beam_reorder_scratch_bytes(int32_t n_req, int32_t beams, int32_t table_stride) {
  if (n_req <= 0 || beams <= 0 || beams > WF_MAX_BEAMS || table_stride <= 0) return 0;
  const size_t rows = static_cast<size_t>(n_req) * beams;
  return (rows * table_stride + n_req + rows * 4 + 1) * sizeof(int32_t);
}

wf_status wf_beam_reorder(const wf_kv4_pool *pool, const int32_t *d_table_in, int32_t *d_table_out, int32_t table_stride,
                          const int32_t *d_len, const int32_t *d_parent, int32_t n_req, int32_t beams, int32_t *d_free,
                          const int32_t *d_n_free, int32_t *d_n_free_out, void *d_scratch, size_t scratch_bytes,
                          uint32_t *d_err, void *stream) {
  ReorderParams p = {};
  int64_t stride = 0;
  const wf_status st = kv4_pool_check(pool, 0, &p.pool, &stride);
  if (st != WF_OK) return st;
  if (!d_table_in || !d_table_out || !d_len || !d_parent || !d_free || !d_n_free || !d_n_free_out || !d_scratch || n_req <= 0 ||
      beams <= 0 || table_stride <= 0 || (reinterpret_cast<uintptr_t>(d_scratch) & 3))
    return WF_ERR_INVALID;
  if (beams > WF_MAX_BEAMS || pool->n_layers > 65535) return WF_ERR_UNSUPPORTED;
  if (static_cast<int64_t>(table_stride) * pool->block_size > INT32_MAX || static_cast<int64_t>(n_req) * beams > INT32_MAX)
    return WF_ERR_INVALID;
  if (scratch_bytes < wf_beam_reorder_scratch_bytes(n_req, beams, table_stride)) return WF_ERR_CAPACITY;
  const size_t rows = static_cast<size_t>(n_req) * beams;
  p.layer_stride = stride;
  p.block_bytes = static_cast<long long>(kv4_block_bytes(pool->block_size, pool->n_kv_heads, pool->head_dim));
  p.n_layers = pool->n_layers;
  p.table_in = d_table_in, p.table_out = d_table_out, p.stride = table_stride;
  p.len = d_len, p.parent = d_parent, p.n_req = n_req, p.W = beams;
  p.free_ids = d_free, p.n_free = d_n_free, p.n_free_out = d_n_free_out;
  p.gone = static_cast<int32_t *>(d_scratch);
  p.gone_n = p.gone + rows * table_stride;
  p.moves = p.gone_n + n_req;
  p.n_free_copy = p.moves + rows * 4;
  p.err = d_err;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  void *args[] = {&p};
  if (launch_pdl(reinterpret_cast<const void *>(beam_tables_kernel), n_req, kReorderThreads, 0, args, s) != cudaSuccess ||
      launch_pdl(reinterpret_cast<const void *>(beam_moves_kernel), dim3(static_cast<unsigned>(rows), p.n_layers), kReorderThreads, 0,
                 args, s) != cudaSuccess)
    return WF_ERR_CUDA;
  return WF_OK;
}

}  // extern "C"
