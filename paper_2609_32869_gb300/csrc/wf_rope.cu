// Rotary positions of queries and keys, and the way back of their gradients.
//
// Pair i of a row at position p turns by the angle p f_i.  f_i / 2 pi is held as
// a fraction of 2^64, so that p f_i mod a whole turn is one wrapping 64-bit
// product; its upper 32 bits give the quarter and, within an eighth of a turn
// on either side of it, a remainder that fp32 holds to 2^-28 of a turn.
#include <algorithm>
#include <cmath>

#include "wf_device.cuh"
#include "wf_ops.cuh"

namespace wf {

constexpr int kRopeThreads = 256;
constexpr int kRopePairs = 512;  // of a CTA's rows, cos and sin in shared memory

struct RopeParams {
  const void *q, *k;
  void *q_out, *k_out;
  long long q_stride, k_stride, q_out_stride, k_out_stride;
  const int32_t *pos;
  int n, hq, heads;                            // heads: of queries and keys
  int rows, units, turned, slots, per_y;       // of a CTA: rows; units of a head, those that turn, and unit columns; heads at a time and of a grid row
  int adjoint, q_copy, k_copy;                 // whether the dims that do not turn are written
  wf_rope_table table;
};

// A vector of VEC elements in memory.
template <typename T, int VEC>
struct alignas(sizeof(T) * VEC) RopeVec {
  T v[VEC];
};
__device__ __forceinline__ float rope_up(float x) { return x; }
__device__ __forceinline__ float rope_up(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float rope_up(__half x) { return __half2float(x); }
__device__ __forceinline__ void rope_down(float x, float &y) { y = x; }
__device__ __forceinline__ void rope_down(float x, __nv_bfloat16 &y) { y = __float2bfloat16_rn(x); }
__device__ __forceinline__ void rope_down(float x, __half &y) { y = __float2half_rn(x); }

// Whole 16 bytes pass as a stream: they are read once, and what is written is
// more than L2 holds or, of few rows, stays in it all the same (2% of a large call).
template <typename V>
__device__ __forceinline__ V rope_load(const V *p) {
  if constexpr (sizeof(V) == 16) {
    const uint4 u = __ldcs(reinterpret_cast<const uint4 *>(p));
    return *reinterpret_cast<const V *>(&u);
  } else {
    return *p;
  }
}
template <typename V>
__device__ __forceinline__ void rope_store(V *p, const V &v) {
  if constexpr (sizeof(V) == 16)
    __stcs(reinterpret_cast<uint4 *>(p), *reinterpret_cast<const uint4 *>(&v));
  else
    *p = v;
}

// gain cos and gain sin of pos * turns.
__device__ __forceinline__ float2 rope_angle(int pos, uint64_t turns, float gain) {
  const uint32_t at = static_cast<uint32_t>((static_cast<uint64_t>(static_cast<int64_t>(pos)) * turns) >> 32);
  const uint32_t quarter = (at + 0x20000000u) >> 30;
  const float x = static_cast<float>(static_cast<int32_t>(at - (quarter << 30))) * 0x1p-31f;  // half turns
  float s, c;
  sincospif(x, &s, &c);
  s *= gain, c *= gain;
  const float cs = quarter & 1 ? s : c, sn = quarter & 1 ? c : s;
  return make_float2(quarter == 1 || quarter == 2 ? -cs : cs, quarter >= 2 ? -sn : sn);
}

// A unit is VEC pairs of a head, two vectors: the same dims of both halves, or,
// where pairs are neighbours, vectors `turned` apart, so that a warp's accesses
// are without gaps; or two vectors of dims that do not turn.  A thread keeps its
// row's cos and sin of one unit in registers and takes that unit of several
// heads, the next one's loads in flight; a CTA works out each (row, pair)'s angle once.
//   16384 rows of 40 heads x 128, bf16, neighbours: 61 us, 5.5 TB/s; at three CTAs
//     an SM (76 registers instead of 64) 68, with two units ahead 71 to 83
//   6001 rows of 40 heads x 64, fp32, 32 dims turn: 20.7 us, 5.9 TB/s; with one unit ahead 22.7
//   80 rows of 40 heads x 64, bf16: 5.7 us, the call and two dependent reads
//   (at 64 registers the 16-bit ones keep 12 to 40 bytes of a thread's addresses in memory)
template <typename T, int VEC, bool kHalf>
__global__ void __launch_bounds__(kRopeThreads, 4) rope_kernel(const __grid_constant__ RopeParams p) {
  using V = RopeVec<T, VEC>;
  constexpr int kAhead = VEC == 8 ? 1 : 2;  // units on their way
  __shared__ float2 turn[kRopePairs];
  pdl_wait();
  pdl_launch_dependents();
  const int pairs = p.table.rot_dim / 2, dim = p.table.head_dim, rot = p.table.rot_dim;
  const long long row0 = static_cast<long long>(blockIdx.x) * p.rows;
  const int rows = static_cast<int>(min(static_cast<long long>(p.rows), p.n - row0));
  const int columns = blockDim.x / (p.rows * p.slots);
  const int col = threadIdx.x % columns, slot = threadIdx.x / columns % p.slots, r = threadIdx.x / (columns * p.slots);
  const bool live = r < rows;
  const long long row = row0 + (live ? r : 0);
  const T *q = static_cast<const T *>(p.q) + row * p.q_stride, *k = static_cast<const T *>(p.k) + row * p.k_stride;
  T *q_out = static_cast<T *>(p.q_out) + row * p.q_out_stride, *k_out = static_cast<T *>(p.k_out) + row * p.k_out_stride;
  const int first = blockIdx.y * p.per_y + slot, last = min(p.heads, (static_cast<int>(blockIdx.y) + 1) * p.per_y);
  V x[kAhead] = {}, y[kAhead] = {};
  int a = 0, b = 0;
  bool two = false;
  const auto unit = [&](int u) {
    const bool turns = u < p.turned;
    const int i = turns ? u : u - p.turned, apart = turns ? p.turned : p.units - p.turned, from = turns ? 0 : rot;
    a = from + i * VEC;
    b = turns && kHalf ? a + pairs : from + (i + apart) * VEC;
    if (VEC == 1 && !kHalf && turns) a = 2 * i, b = 2 * i + 1;
    two = b + VEC <= dim;  // (dims that do not turn may be an odd number of vectors)
  };
  const auto load = [&](int h, int s) {
    const T *src = h < p.hq ? q + static_cast<long long>(h) * dim : k + static_cast<long long>(h - p.hq) * dim;
    x[s] = rope_load(reinterpret_cast<const V *>(src + a));
    if (two) y[s] = rope_load(reinterpret_cast<const V *>(src + b));
  };
  const auto start = [&]() {
#pragma unroll
    for (int s = 0; s < kAhead; ++s)
      if (first + s * p.slots < last) load(first + s * p.slots, s);
  };
  unit(col);
  if (live) start();  // on their way while the angles are worked out
  for (int i = threadIdx.x; i < rows * pairs; i += blockDim.x) {
    const int ri = i / pairs;
    float2 t = rope_angle(p.pos[row0 + ri], p.table.turns[i - ri * pairs], p.table.gain);
    if (p.adjoint) t.y = -t.y;
    turn[i] = t;
  }
  __syncthreads();
  if (!live) return;
  for (int u = col; u < p.units; u += columns) {
    const bool turns = u < p.turned;
    float2 cs[VEC];
    if (turns) {
#pragma unroll
      for (int e = 0; e < VEC; ++e)
        cs[e] = turn[r * pairs + (kHalf || VEC == 1 ? u * VEC + e : (2 * e < VEC ? u : u + p.turned) * (VEC / 2) + e % ((VEC + 1) / 2))];
    }
    if (u != col) {
      unit(u);
      start();
    }
    for (int h0 = first; h0 < last; h0 += kAhead * p.slots) {
#pragma unroll
      for (int s = 0; s < kAhead; ++s) {
        const int h = h0 + s * p.slots;
        if (h >= last) break;
        const V cx = x[s], cy = y[s];
        if (h + kAhead * p.slots < last) load(h + kAhead * p.slots, s);
        T *dst = h < p.hq ? q_out + static_cast<long long>(h) * dim : k_out + static_cast<long long>(h - p.hq) * dim;
        V ox = cx, oy = cy;
        if (turns) {
#pragma unroll
          for (int e = 0; e < VEC; ++e) {
            // elements e of both vectors, or 2e and 2e + 1 of the two in a row
            const T &i0 = kHalf || VEC == 1 ? cx.v[e] : (2 * e < VEC ? cx.v[2 * e % VEC] : cy.v[2 * e % VEC]);
            const T &i1 = kHalf || VEC == 1 ? cy.v[e] : (2 * e < VEC ? cx.v[(2 * e + 1) % VEC] : cy.v[(2 * e + 1) % VEC]);
            T &o0 = kHalf || VEC == 1 ? ox.v[e] : (2 * e < VEC ? ox.v[2 * e % VEC] : oy.v[2 * e % VEC]);
            T &o1 = kHalf || VEC == 1 ? oy.v[e] : (2 * e < VEC ? ox.v[(2 * e + 1) % VEC] : oy.v[(2 * e + 1) % VEC]);
            const float f0 = rope_up(i0), f1 = rope_up(i1);
            rope_down(fmaf(f0, cs[e].x, -f1 * cs[e].y), o0);
            rope_down(fmaf(f0, cs[e].y, f1 * cs[e].x), o1);
          }
        } else if (!(h < p.hq ? p.q_copy : p.k_copy)) {
          continue;
        }
        rope_store(reinterpret_cast<V *>(dst + a), ox);
        if (two) rope_store(reinterpret_cast<V *>(dst + b), oy);
      }
    }
  }
}

}  // namespace wf

using namespace wf;

template <typename T>
static const void *rope_fn(int vec, bool half) {
  constexpr int kMost = 16 / sizeof(T);
  if (vec == kMost) return half ? reinterpret_cast<const void *>(rope_kernel<T, kMost, true>) : reinterpret_cast<const void *>(rope_kernel<T, kMost, false>);
  if (vec == 4) return half ? reinterpret_cast<const void *>(rope_kernel<T, 4, true>) : reinterpret_cast<const void *>(rope_kernel<T, 4, false>);
  if (vec == 2) return half ? reinterpret_cast<const void *>(rope_kernel<T, 2, true>) : reinterpret_cast<const void *>(rope_kernel<T, 2, false>);
  return half ? reinterpret_cast<const void *>(rope_kernel<T, 1, true>) : reinterpret_cast<const void *>(rope_kernel<T, 1, false>);
}

static bool rope_table_ok(const wf_rope_table *t) {
  return t && t->head_dim >= 2 && t->head_dim <= 4096 && t->rot_dim >= 2 && t->rot_dim <= 2 * WF_ROPE_MAX_PAIRS && t->rot_dim <= t->head_dim &&
         t->rot_dim % 2 == 0 && (t->layout == WF_ROPE_HALF || t->layout == WF_ROPE_INTERLEAVED) && t->gain > 0.f && std::isfinite(t->gain);
}

extern "C" {

wf_status wf_rope_init(const wf_rope_spec *s, wf_rope_table *out) {
  if (!s || !out) return WF_ERR_INVALID;
  wf_rope_table t = {};
  t.head_dim = s->head_dim, t.rot_dim = s->rot_dim, t.layout = s->layout, t.gain = static_cast<float>(s->gain);
  if (s->head_dim > 4096 || s->rot_dim > 2 * WF_ROPE_MAX_PAIRS) return WF_ERR_UNSUPPORTED;
  if (!rope_table_ok(&t) || !(s->base > 1) || !std::isfinite(s->base) || s->scaling < WF_ROPE_PLAIN || s->scaling > WF_ROPE_PARTS)
    return WF_ERR_INVALID;
  if (s->scaling != WF_ROPE_PLAIN && (!(s->factor >= 1) || !std::isfinite(s->factor))) return WF_ERR_INVALID;
  const bool by_turns = s->scaling == WF_ROPE_WAVES || s->scaling == WF_ROPE_PARTS;
  if (by_turns && (!(s->low > 0) || !(s->high > s->low) || !std::isfinite(s->high) || !(s->trained_len > 0) || !std::isfinite(s->trained_len)))
    return WF_ERR_INVALID;
  constexpr double kTwoPi = 6.283185307179586476925286766559;
  const int rot = s->rot_dim;
  const double base = s->scaling == WF_ROPE_BASE && rot > 2 ? s->base * std::pow(s->factor, static_cast<double>(rot) / (rot - 2)) : s->base;
  double a = 0, b = 1;
  if (s->scaling == WF_ROPE_PARTS) {
    const auto pair = [&](double n) { return rot * std::log(s->trained_len / (kTwoPi * n)) / (2 * std::log(s->base)); };
    a = std::max(std::floor(pair(s->high)), 0.0), b = std::min(std::ceil(pair(s->low)), rot - 1.0);
  }
  for (int i = 0; i < rot / 2; ++i) {
    double f = std::pow(base, -2.0 * i / rot);
    if (s->scaling == WF_ROPE_LINEAR) f /= s->factor;
    if (s->scaling == WF_ROPE_WAVES) {
      const double w = std::min(std::max((f * s->trained_len / kTwoPi - s->low) / (s->high - s->low), 0.0), 1.0);
      f = w * f + (1 - w) * f / s->factor;
    }
    if (s->scaling == WF_ROPE_PARTS) {
      const double w = std::min(std::max((i - a) / std::max(b - a, 0.001), 0.0), 1.0);
      f = w * f / s->factor + (1 - w) * f;
    }
    t.turns[i] = static_cast<uint64_t>(std::ldexp(f / kTwoPi, 64));  // f is at most 1: below 2^62
  }
  *out = t;
  return WF_OK;
}

wf_status wf_rope(const wf_rope_table *table, const void *d_q, int64_t q_stride, int32_t n_heads, const void *d_k, int64_t k_stride,
                  int32_t n_kv_heads, const int32_t *d_pos, int32_t n, int32_t dtype, int32_t adjoint, void *d_q_out, int64_t q_out_stride,
                  void *d_k_out, int64_t k_out_stride, void *stream) {
  if (!rope_table_ok(table) || !d_q || !d_q_out || !d_pos || n < 0 || n_heads <= 0 || n_kv_heads < 0) return WF_ERR_INVALID;
  if (dtype != WF_BF16 && dtype != WF_F16 && dtype != WF_F32) return WF_ERR_UNSUPPORTED;
  const int size = dtype == WF_F32 ? 4 : 2;
  const int64_t dim = table->head_dim, q_row = dim * n_heads, k_row = dim * n_kv_heads;
  if (q_stride < q_row || q_out_stride < q_row) return WF_ERR_INVALID;
  if (n_kv_heads && (!d_k || !d_k_out || k_stride < k_row || k_out_stride < k_row)) return WF_ERR_INVALID;
  if ((d_q == d_q_out && q_stride != q_out_stride) || (n_kv_heads && d_k == d_k_out && k_stride != k_out_stride)) return WF_ERR_INVALID;
  if (static_cast<int64_t>(n_heads) + n_kv_heads > 65535) return WF_ERR_UNSUPPORTED;
  uintptr_t bits = reinterpret_cast<uintptr_t>(d_q) | reinterpret_cast<uintptr_t>(d_q_out);
  int64_t strides = q_stride | q_out_stride;
  if (n_kv_heads) bits |= reinterpret_cast<uintptr_t>(d_k) | reinterpret_cast<uintptr_t>(d_k_out), strides |= k_stride | k_out_stride;
  if (bits % size) return WF_ERR_INVALID;
  if (n == 0) return WF_OK;
  const bool half = table->layout == WF_ROPE_HALF;
  const int rot = table->rot_dim;
  int vec = 16 / size;  // as wide as addresses, strides and the dims' parts allow
  while (vec > 1 && (bits % (vec * size) || strides % vec || dim % vec || rot % (2 * vec))) vec /= 2;
  RopeParams p = {};
  p.q = d_q, p.k = d_k, p.q_out = d_q_out, p.k_out = d_k_out;
  p.q_stride = q_stride, p.k_stride = k_stride, p.q_out_stride = q_out_stride, p.k_out_stride = k_out_stride;
  p.pos = d_pos, p.n = n, p.hq = n_heads, p.heads = n_heads + n_kv_heads, p.adjoint = adjoint != 0;
  p.q_copy = d_q != d_q_out, p.k_copy = d_k != d_k_out, p.table = *table;
  p.turned = rot / (2 * vec);
  const bool copies = p.q_copy || (n_kv_heads && p.k_copy);
  p.units = p.turned + (copies ? static_cast<int>((dim - rot) / vec + 1) / 2 : 0);
  const int columns = std::min(p.units, kRopeThreads);
  // Rows of a CTA: rounds of four CTAs an SM, each as long as its rows' bytes and about
  // 12 KB more for a CTA's start; as few of that as can be, of at least one whole round.
  // (16384 rows of 40 heads, bf16: 128 dims with 4 rows, 7 rounds, 61 us, 8 rows, 4 rounds, 63;
  // 64 dims with 4 rows 37.1, with 8 34.0)
  const int64_t row_bytes = static_cast<int64_t>(p.units) * 2 * vec * size * p.heads;
  constexpr int kRound = kSms * 4;
  p.rows = 1;
  int64_t least = INT64_MAX;
  for (int rows = 1; rows <= 8 && rows * (rot / 2) <= kRopePairs && rows * columns <= kRopeThreads && (rows == 1 || n / rows >= kRound); rows *= 2) {
    const int64_t ctas = (static_cast<int64_t>(n) + rows - 1) / rows, cost = (ctas + kRound - 1) / kRound * (rows * row_bytes + 12288);
    if (cost <= least) least = cost, p.rows = rows;
  }
  p.slots = std::max(1, std::min(p.heads, kRopeThreads / (p.rows * columns)));
  // Few rows: a grid row for every `slots` heads, so that a thread takes one.
  p.per_y = n <= kSms * 4 ? p.slots : p.heads;
  const dim3 grid(static_cast<unsigned>((static_cast<int64_t>(n) + p.rows - 1) / p.rows), (p.heads + p.per_y - 1) / p.per_y);
  const void *fn = dtype == WF_F32 ? rope_fn<float>(vec, half) : dtype == WF_F16 ? rope_fn<__half>(vec, half) : rope_fn<__nv_bfloat16>(vec, half);
  void *args[] = {&p};
  return launch_pdl(fn, grid, p.rows * columns * p.slots, 0, args, static_cast<cudaStream_t>(stream)) == cudaSuccess ? WF_OK : WF_ERR_CUDA;
}

}  // extern "C"
