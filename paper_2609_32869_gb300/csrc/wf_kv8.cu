// Rows into the paged 8-bit cache and back.
//
// A record's 16 positions of a head share a power of two, so a row that is
// appended may change it for the positions before it: the record is read,
// scaled and rounded again, and written whole.  e4m3 codes under a larger power
// of two stay exact but for those that fall below the smallest normal one.
#include <algorithm>

#include "wf_device.cuh"
#include "wf_kv8.cuh"

namespace wf {

constexpr int kK8Warps = 4;

struct Kv8RowParams {
  Kv8Pool pool;
  const void *k, *v;
  void *k_out, *v_out;
  long long k_stride, v_stride;
  const int32_t *slots;
  int n, rows, heads;  // rows and heads of a CTA
  uint32_t *err;
};

// The slots of a CTA's first 32 rows, a lane each (-1 past the last), and as bits
// those of its own rows that open a run.  Rows of a record that follow one
// another are one run, rows that are skipped between them or not (up to
// kK8Skips in a row); `ascending`: rows directly behind one another, as far as
// their positions ascend.
constexpr int kK8Skips = 31;
struct Kv8Rows {
  int slot;
  uint32_t openers;
};
__device__ __forceinline__ Kv8Rows kv8_rows(const Kv8RowParams &p, int row0, int lane, bool ascending) {
  Kv8Rows r;
  r.slot = row0 + lane < p.n ? p.slots[row0 + lane] : -1;
  const int back = row0 - 32 + lane >= 0 ? p.slots[row0 - 32 + lane] : -1;
  int before, apart = 1;
  if (ascending) {
    const int first = __shfl_sync(0xffffffffu, back, 31), up = __shfl_up_sync(0xffffffffu, r.slot, 1);
    before = lane == 0 ? first : up;
  } else {  // the nearest that is not skipped
    const uint32_t here = __ballot_sync(0xffffffffu, r.slot >= 0) & ((1u << lane) - 1), there = __ballot_sync(0xffffffffu, back >= 0);
    const int at = 31 - __clz(here ? here : there ? there : 1u);
    const int near = __shfl_sync(0xffffffffu, r.slot, at), far = __shfl_sync(0xffffffffu, back, at);
    before = here ? near : far, apart = (here ? 0 : 32) + lane - at;
  }
  const bool mine = lane < p.rows && row0 + lane < p.n;
  const bool opens = r.slot < 0 ? ascending : before < 0 || apart > kK8Skips + 1 || before >> 4 != r.slot >> 4 || (ascending && before >= r.slot);
  r.openers = __ballot_sync(0xffffffffu, mine && opens);
  return r;
}
// Bit n (from 0) of those that are set.
__device__ __forceinline__ int nth_bit(uint32_t bits, int n) {
  for (; n > 0; --n) bits &= bits - 1;
  return __ffs(bits) - 1;
}

// The positions of the run of rows that row `first` of the CTA opens: of lane
// l < 16 the row of position l (-1: none).
struct Kv8Run {
  int slot;      // the first row's
  int row;
  uint32_t has;  // positions with a row
};
__device__ __forceinline__ Kv8Run kv8_run(const Kv8RowParams &p, const Kv8Rows &rows, int row0, int first, int lane, bool ascending) {
  Kv8Run r;
  r.slot = __shfl_sync(0xffffffffu, rows.slot, first);
  r.row = -1;
  int at = row0 + first, slot = __shfl_sync(0xffffffffu, rows.slot, (lane + first) & 31), most = 32 - first, latest = at;
  for (;;) {  // (again only for more rows than a record has positions, or where rows are skipped)
    const bool same = slot >= 0 && slot >> 4 == r.slot >> 4;
    bool in = lane < most && at + lane < p.n && (same || (slot < 0 && !ascending));
    if (ascending) {
      const int before = __shfl_up_sync(0xffffffffu, slot, 1);
      in = in && (lane == 0 || before < slot);
    }
    const uint32_t out = ~__ballot_sync(0xffffffffu, in);
    const int count = out ? __ffs(out) - 1 : 32;
    uint32_t which = __ballot_sync(0xffffffffu, same && lane < count);
    if (which == 0 || at + __ffs(which) - 1 - latest > kK8Skips + 1) break;
    latest = at + 31 - __clz(which);
    const int start = r.slot & 15;
    if (at == row0 + first && __all_sync(0xffffffffu, lane >= count || slot == r.slot + lane)) {
      if (lane >= start && lane - start < count) r.row = at + lane - start;
    } else {
      for (; which; which &= which - 1) {
        const int c = __ffs(which) - 1;
        if ((__shfl_sync(0xffffffffu, slot, c) & 15) == lane) r.row = at + c;
      }
    }
    if (count < most || ascending) break;
    at += most, most = 32;
    slot = at + lane < p.n ? p.slots[at + lane] : -1;
  }
  r.has = __ballot_sync(0xffffffffu, lane < 16 && r.row >= 0);
  return r;
}

template <typename T>
struct Kv8Limits;
template <>
struct Kv8Limits<__nv_bfloat16> {
  static constexpr uint32_t kInf = 0x7f80;
};
template <>
struct Kv8Limits<__half> {
  static constexpr uint32_t kInf = 0x7c00;
};

// The larger of two pairs of 16-bit magnitudes.
__device__ __forceinline__ uint32_t max_u16x2(uint32_t a, uint32_t b) { return __vmaxu2(a, b); }

// The least e with max |x| <= 448 * 2^e: 448 = 1.75 * 2^8.
__device__ __forceinline__ int kv8_exponent(float most) {
  const uint32_t u = __float_as_uint(most);
  const int e = static_cast<int>(u >> 23) - 135 + ((u & 0x7fffffu) > 0x600000u);
  return most == 0.f ? kKv8Low : min(max(e, kKv8Low), kKv8High);
}

// The power of two of a record's values, from the rows that a warp's lanes hold; what
// is not finite becomes NaN and does not count.
template <typename T, int G>
__device__ __forceinline__ int kv8_most(uint4 (&w)[G][4]) {
  uint32_t most2 = 0;
#pragma unroll
  for (int g = 0; g < G; ++g)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t m = 0x7fff7fffu;
      most2 = max_u16x2(max_u16x2(max_u16x2(w[g][i].x & m, w[g][i].y & m), max_u16x2(w[g][i].z & m, w[g][i].w & m)), most2);
    }
  uint32_t most = __reduce_max_sync(0xffffffffu, max(most2 & 0xffff, most2 >> 16));
  if (most >= Kv8Limits<T>::kInf) {
    most = 0;
#pragma unroll
    for (int g = 0; g < G; ++g)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        uint32_t *u = reinterpret_cast<uint32_t *>(&w[g][i]);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const uint32_t lo = u[j] & 0x7fff, hi = u[j] >> 16 & 0x7fff;
          if (lo < Kv8Limits<T>::kInf) most = max(most, lo); else u[j] |= 0x7fff;
          if (hi < Kv8Limits<T>::kInf) most = max(most, hi); else u[j] |= 0x7fff0000u;
        }
      }
    most = __reduce_max_sync(0xffffffffu, most);
  }
  return kv8_exponent(Type16<T>::lo(most));
}

// One warp per record and head.  Lane 4 r + t holds the dims 8r .. 8r + 7 of
// every group for the positions 2t, 2t + 1, 2t + 8, 2t + 9: its 32 bytes of value
// codes, and pieces of 8 bytes of the key codes.  Every load, of rows and of
// what a record keeps, is on its way before the first is used.
//   48000 rows of 20 heads x 64, bf16, records of their own: 63 us, 5.9 TB/s, by
//     HBM (read back in as long); with a record's loads one after another 70
//     (fp16 keeps 28 bytes a thread in memory at six CTAs an SM)
template <typename T, int G>
__global__ void __launch_bounds__(kK8Warps * 32, G == 1 ? 6 : 3) kv8_store_kernel(const Kv8RowParams p) {
  using X = Type16<T>;
  pdl_wait();
  pdl_launch_dependents();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, r = lane >> 2, t = lane & 3;
  const int row0 = blockIdx.x * p.rows, head0 = blockIdx.y * p.heads, heads = min(p.heads, p.pool.heads - head0);
  const Kv8Rows rows = kv8_rows(p, row0, lane, false);
  const int units = __popc(rows.openers) * heads;
  for (int unit = warp; unit < units; unit += kK8Warps) {
    const int head = head0 + unit % heads;
    const Kv8Run run = kv8_run(p, rows, row0, nth_bit(rows.openers, unit / heads), lane, false);
    const int block = run.slot >> p.pool.bs_shift;
    if (block >= p.pool.n_blocks) {
      if (lane == 0) set_error(p.err, WF_DEV_ERR_PAGE);
      continue;
    }
    unsigned char *rec = kv8_record(p.pool, block, head, (run.slot & (p.pool.bs - 1)) >> 4);
    const uint32_t kept = (1u << (__ffs(run.has) - 1)) - 1;
    uint4 w[2][G][4], had_v[G][2];
    uint2 had_k[G][4];
    uint2 held = make_uint2(0, 0);
    bool keeps[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int pos = 2 * t + i % 2 + i / 2 * 8;
      const long long row = __shfl_sync(0xffffffffu, run.row, pos);
      keeps[i] = kept >> pos & 1;
#pragma unroll
      for (int g = 0; g < G; ++g) {
        w[0][g][i] = w[1][g][i] = make_uint4(0, 0, 0, 0);
        if (row >= 0) {
          w[0][g][i] = *reinterpret_cast<const uint4 *>(static_cast<const T *>(p.k) + row * p.k_stride + head * (G * 64) + g * 64 + r * 8);
          w[1][g][i] = *reinterpret_cast<const uint4 *>(static_cast<const T *>(p.v) + row * p.v_stride + head * (G * 64) + g * 64 + r * 8);
        }
        if (keeps[i]) had_k[g][i] = *reinterpret_cast<const uint2 *>(rec + g * kKv8Group + pos * 64 + r * 8);
      }
    }
    if (kept) {
#pragma unroll
      for (int g = 0; g < G; ++g)
#pragma unroll
        for (int h = 0; h < 2; ++h) had_v[g][h] = *reinterpret_cast<const uint4 *>(rec + g * kKv8Group + 1024 + h * 512 + lane * 16);
      held = *reinterpret_cast<const uint2 *>(rec + G * kKv8Group);
    }
    float scales[2];
    // keys, then values
#pragma unroll
    for (int is_v = 0; is_v < 2; ++is_v) {
      int e = kv8_most<T, G>(w[is_v]);
      float back = 1.f;
      if (kept) {
        const int old = min(max(static_cast<int>((is_v ? held.y : held.x) >> 23 & 255) - 127, kKv8Low), kKv8High);
        e = max(e, old);
        back = two_to(old - e);
      }
      const float scale = two_to(-e);
      scales[is_v] = two_to(e);
#pragma unroll
      for (int g = 0; g < G; ++g) {
        float x[4][8];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint32_t *u = reinterpret_cast<const uint32_t *>(&w[is_v][g][i]);
#pragma unroll
          for (int j = 0; j < 4; ++j) x[i][2 * j] = X::lo(u[j]) * scale, x[i][2 * j + 1] = X::hi(u[j]) * scale;
        }
        if (!is_v) {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            if (keeps[i]) {
#pragma unroll
              for (int j = 0; j < 4; ++j) {
                const float2 f = codes_to_f32((j < 2 ? had_k[g][i].x : had_k[g][i].y) >> (j % 2 * 16));
                x[i][2 * j] = f.x * back, x[i][2 * j + 1] = f.y * back;
              }
            }
            const int pos = 2 * t + i % 2 + i / 2 * 8;
            *reinterpret_cast<uint2 *>(rec + g * kKv8Group + pos * 64 + r * 8) =
                make_uint2(f32_to_codes(x[i][0], x[i][1]) | f32_to_codes(x[i][2], x[i][3]) << 16,
                           f32_to_codes(x[i][4], x[i][5]) | f32_to_codes(x[i][6], x[i][7]) << 16);
          }
        } else {
          uint4 *at = reinterpret_cast<uint4 *>(rec + g * kKv8Group + 1024 + lane * 16);
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            uint32_t c[4];
            if (kept) {
              c[0] = had_v[g][h].x, c[1] = had_v[g][h].y, c[2] = had_v[g][h].z, c[3] = had_v[g][h].w;
#pragma unroll
              for (int j = 0; j < 8; ++j) {  // 16 bits: [odd dim][a]
                const int dim = j % 2 * 4 + 2 * h + j / 4, i = j / 2 % 2 * 2;
                const float2 f = codes_to_f32(c[j / 2] >> (j % 2 * 16));
                if (keeps[i]) x[i][dim] = f.x * back;
                if (keeps[i + 1]) x[i + 1][dim] = f.y * back;
              }
            }
#pragma unroll
            for (int w4 = 0; w4 < 4; ++w4) {
              const int dim = 2 * h + w4 / 2, i = w4 % 2 * 2;
              c[w4] = f32_to_codes(x[i][dim], x[i + 1][dim]) | f32_to_codes(x[i][dim + 4], x[i + 1][dim + 4]) << 16;
            }
            at[h * 32] = make_uint4(c[0], c[1], c[2], c[3]);
          }
        }
      }
    }
    __syncwarp();  // every lane has read the old scales
    if (lane == 0) *reinterpret_cast<float4 *>(rec + G * kKv8Group) = make_float4(scales[0], scales[1], 0.f, 0.f);
  }
}

template <typename T, int G>
__global__ void __launch_bounds__(kK8Warps * 32) kv8_load_kernel(const Kv8RowParams p) {
  using X = Type16<T>;
  pdl_wait();
  pdl_launch_dependents();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, r = lane >> 2, t = lane & 3;
  const int row0 = blockIdx.x * p.rows, head0 = blockIdx.y * p.heads, heads = min(p.heads, p.pool.heads - head0);
  const Kv8Rows rows = kv8_rows(p, row0, lane, true);
  const int units = __popc(rows.openers) * heads;
  for (int unit = warp; unit < units; unit += kK8Warps) {
    const int head = head0 + unit % heads, nth = nth_bit(rows.openers, unit / heads);
    const long long first = row0 + nth;
    T *k = static_cast<T *>(p.k_out) + head * (G * 64) + r * 8, *v = static_cast<T *>(p.v_out) + head * (G * 64) + r * 8;
    const int slot = __shfl_sync(0xffffffffu, rows.slot, nth), block = slot >> p.pool.bs_shift;
    const bool none = slot < 0, out = !none && block >= p.pool.n_blocks;
    if (out && lane == 0) set_error(p.err, WF_DEV_ERR_PAGE);
    if (none) {  // a row of its own
#pragma unroll
      for (int g = 0; g < G; ++g)
        if (t < 2) *reinterpret_cast<uint4 *>((t ? v : k) + first * (t ? p.v_stride : p.k_stride) + g * 64) = make_uint4(0, 0, 0, 0);
      continue;
    }
    const Kv8Run run = kv8_run(p, rows, row0, nth, lane, true);
    const unsigned char *rec = kv8_record(p.pool, out ? 0 : block, head, (slot & (p.pool.bs - 1)) >> 4);
    const float2 scale = *reinterpret_cast<const float2 *>(rec + G * kKv8Group);
#pragma unroll
    for (int g = 0; g < G; ++g) {
      const uint4 va = *reinterpret_cast<const uint4 *>(rec + g * kKv8Group + 1024 + lane * 16);
      const uint4 vb = *reinterpret_cast<const uint4 *>(rec + g * kKv8Group + 1536 + lane * 16);
      const uint32_t c[2][4] = {{va.x, va.y, va.z, va.w}, {vb.x, vb.y, vb.z, vb.w}};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int pos = 2 * t + i % 2 + i / 2 * 8;
        const long long row = __shfl_sync(0xffffffffu, run.row, pos);
        if (row < 0) continue;
        const uint2 kc = *reinterpret_cast<const uint2 *>(rec + g * kKv8Group + pos * 64 + r * 8);
        uint32_t ko[4], vo[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float2 f = codes_to_f32((j < 2 ? kc.x : kc.y) >> (j % 2 * 16));
          ko[j] = X::pack(f.x * scale.x, f.y * scale.x);
          // dims 2j and 2j + 1: piece j % 2, words of the even and the odd dim
          const int a = j / 2 + i / 2 * 2, shift = a % 2 * 16 + i % 2 * 8;
          const float2 e = codes_to_f32(c[j % 2][a / 2] >> shift & 0xff), o = codes_to_f32(c[j % 2][2 + a / 2] >> shift & 0xff);
          vo[j] = X::pack(e.x * scale.y, o.x * scale.y);
        }
        const uint4 kw = out ? make_uint4(0, 0, 0, 0) : make_uint4(ko[0], ko[1], ko[2], ko[3]);
        const uint4 vw = out ? make_uint4(0, 0, 0, 0) : make_uint4(vo[0], vo[1], vo[2], vo[3]);
        *reinterpret_cast<uint4 *>(k + row * p.k_stride + g * 64) = kw;
        *reinterpret_cast<uint4 *>(v + row * p.v_stride + g * 64) = vw;
      }
    }
    __syncwarp();
  }
}

}  // namespace wf

using namespace wf;

static wf_status kv8_rows(const wf_kv8_pool *pool, int32_t layer, const void *k, int64_t k_stride, const void *v, int64_t v_stride,
                          const int32_t *d_slots, int32_t n, Kv8RowParams *p) {
  const wf_status st = kv8_pool_check(pool, layer, &p->pool);
  if (st != WF_OK) return st;
  const int64_t d = static_cast<int64_t>(pool->n_kv_heads) * pool->head_dim;
  if (!k || !v || !d_slots || n < 0 || !aligned16(k) || !aligned16(v) || k_stride % 8 || v_stride % 8 || k_stride < d || v_stride < d)
    return WF_ERR_INVALID;
  if (n > INT32_MAX - 64) return WF_ERR_UNSUPPORTED;
  p->k_stride = k_stride, p->v_stride = v_stride, p->slots = d_slots, p->n = n;
  return WF_OK;
}

static wf_status kv8_rows_launch(const void *fn, Kv8RowParams *p, void *stream) {
  if (p->n == 0) return WF_OK;
  // A warp takes about one record and head while there are SMs for it: of rows
  // that are each a record's only one (few of them, a decode step) four a CTA
  // and head, of a prompt's 16, a record or two; then up to eight heads a CTA.
  // 80 rows with 680 read back, 20 heads: 8.2 us; with eight heads from the start 14.
  const int64_t tiles = (static_cast<int64_t>(p->n) + 15) / 16;
  p->rows = static_cast<int64_t>(p->n) * p->pool.heads <= kSms * 64 ? 4 : 16;
  p->heads = static_cast<int>(std::max<int64_t>(1, std::min<int64_t>({tiles * p->pool.heads / (kSms * 16), 8, p->pool.heads})));
  const dim3 grid((p->n + p->rows - 1) / p->rows, (p->pool.heads + p->heads - 1) / p->heads);
  void *args[] = {p};
  return launch_pdl(fn, grid, kK8Warps * 32, 0, args, static_cast<cudaStream_t>(stream)) == cudaSuccess ? WF_OK : WF_ERR_CUDA;
}

#define WF_KV8_KERNEL(NAME)                                                                                                          \
  (pool->dtype == WF_F16                                                                                                             \
       ? (pool->head_dim == 64 ? reinterpret_cast<const void *>(NAME<__half, 1>) : reinterpret_cast<const void *>(NAME<__half, 2>)) \
       : (pool->head_dim == 64 ? reinterpret_cast<const void *>(NAME<__nv_bfloat16, 1>)                                             \
                               : reinterpret_cast<const void *>(NAME<__nv_bfloat16, 2>)))

extern "C" {

size_t wf_kv8_block_bytes(int32_t block_size, int32_t n_kv_heads, int32_t head_dim) {
  return kv8_shape_ok(block_size, n_kv_heads, head_dim) ? kv8_block_bytes(block_size, n_kv_heads, head_dim) : 0;
}

wf_status wf_kv8_store(const wf_kv8_pool *pool, int32_t layer, const void *d_k, int64_t k_stride, const void *d_v, int64_t v_stride,
                       const int32_t *d_slots, int32_t n, uint32_t *d_err, void *stream) {
  Kv8RowParams p = {};
  const wf_status st = kv8_rows(pool, layer, d_k, k_stride, d_v, v_stride, d_slots, n, &p);
  if (st != WF_OK) return st;
  p.k = d_k, p.v = d_v, p.err = d_err;
  return kv8_rows_launch(WF_KV8_KERNEL(kv8_store_kernel), &p, stream);
}

wf_status wf_kv8_load(const wf_kv8_pool *pool, int32_t layer, const int32_t *d_slots, int32_t n, void *d_k, int64_t k_stride, void *d_v,
                      int64_t v_stride, uint32_t *d_err, void *stream) {
  Kv8RowParams p = {};
  const wf_status st = kv8_rows(pool, layer, d_k, k_stride, d_v, v_stride, d_slots, n, &p);
  if (st != WF_OK) return st;
  p.k_out = d_k, p.v_out = d_v, p.err = d_err;
  return kv8_rows_launch(WF_KV8_KERNEL(kv8_load_kernel), &p, stream);
}

}  // extern "C"
