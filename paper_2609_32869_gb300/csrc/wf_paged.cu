// The paged 4-bit cache around its attention: block tables and slot maps from
// request lengths, rows into and out of the cache, and the reordering of the
// beams' tables after a selection.
#include <algorithm>
#include <type_traits>

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
constexpr int kPlanRequests = 1 << 16;  // every CTA reads all lengths: n^2 / 64 reads
constexpr int kPlanSlots = INT32_MAX - (1 << 20);  // a grid's step past the last slot is still an int

// Inclusive scan over the CTA of two counts at a time, and their totals.
__device__ __forceinline__ void block_scan2(long long &a, long long &b, long long (*sm)[2], long long &ta, long long &tb) {
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
#pragma unroll
  for (int off = 1; off < 32; off <<= 1) {
    const long long pa = __shfl_up_sync(0xffffffffu, a, off), pb = __shfl_up_sync(0xffffffffu, b, off);
    if (lane >= off) a += pa, b += pb;
  }
  if (lane == 31) sm[w][0] = a, sm[w][1] = b;
  __syncthreads();
  ta = tb = 0;
#pragma unroll
  for (int i = 0; i < kPlanThreads / 32; ++i) {
    if (i < w) a += sm[i][0], b += sm[i][1];
    ta += sm[i][0], tb += sm[i][1];
  }
}

// Every CTA scans all the lengths, a run of requests a thread, and keeps the
// prefixes of the requests it owns, i = blockIdx mod gridDim; then it fills
// those requests' table columns and slots.  Counts only grow along the
// requests, so the granted ones are a prefix.  Bound by its chain of reads
// (lengths, ids, slots) and the launch: 4.8 us for one token each of 80
// requests, 7.2 us for 512 prompts of up to 4096 tokens (by passes of 256
// requests 9.9).
__global__ void __launch_bounds__(kPlanThreads) page_plan_kernel(const PlanParams p) {
  pdl_wait();
  pdl_launch_dependents();
  __shared__ long long sm[2][kPlanThreads / 32][2];
  __shared__ int own_block[kPlanOwned], own_tok[kPlanOwned], own_ok[kPlanOwned];
  const int bs = 1 << p.bs_shift;
  int nf = *p.n_free;
  uint32_t err = 0;
  if (nf < 0 || nf > p.n_blocks) nf = 0, err = WF_DEV_ERR_PAGE;
  const auto need = [&](int i, long long &nb, long long &nt) {
    const int a = p.old_len[i], b = p.new_len[i];
    const bool valid = a >= 0 && b >= a && (static_cast<long long>(b) + bs - 1) >> p.bs_shift <= p.stride;
    nt = valid ? b - a : 0;
    nb = valid ? ((static_cast<long long>(b) + bs - 1) >> p.bs_shift) - ((static_cast<long long>(a) + bs - 1) >> p.bs_shift) : 0;
    return valid;
  };
  const int run = (p.n + kPlanThreads - 1) / kPlanThreads, i0 = min(static_cast<int>(threadIdx.x) * run, p.n), i1 = min(i0 + run, p.n);
  long long my_b = 0, my_t = 0, all_b, all_t;
#pragma unroll 4
  for (int i = i0; i < i1; ++i) {
    long long nb, nt;
    need(i, nb, nt);
    my_b += nb, my_t += nt;
  }
  long long cb = my_b, ct = my_t;
  block_scan2(cb, ct, sm[0], all_b, all_t);
  cb -= my_b, ct -= my_t;
  long long grant_b = 0, grant_t = 0;  // of the granted ones
#pragma unroll 2
  for (int i = i0; i < i1; ++i) {
    long long nb, nt;
    const bool valid = need(i, nb, nt);
    cb += nb, ct += nt;
    const bool ok = valid && cb <= nf && ct <= p.cap;
    if (!ok) err |= valid ? WF_DEV_ERR_CAPACITY : WF_DEV_ERR_PAGE;
    if (ok) grant_b = cb, grant_t = ct;
    if (i % gridDim.x == blockIdx.x) {
      const int k = i / gridDim.x;
      own_block[k] = ok ? static_cast<int>(cb - nb) : 0;
      own_tok[k] = static_cast<int>(min(ct - nt, static_cast<long long>(p.cap)));
      own_ok[k] = ok;
    }
  }
  if (all_b <= nf && all_t <= p.cap) {
    grant_b = all_b, grant_t = all_t;
    __syncthreads();
  } else {  // the largest granted counts
#pragma unroll
    for (int off = 16; off; off >>= 1) {
      grant_b = max(grant_b, __shfl_xor_sync(0xffffffffu, grant_b, off));
      grant_t = max(grant_t, __shfl_xor_sync(0xffffffffu, grant_t, off));
    }
    if ((threadIdx.x & 31) == 0) sm[1][threadIdx.x >> 5][0] = grant_b, sm[1][threadIdx.x >> 5][1] = grant_t;
    __syncthreads();
    for (int w = 0; w < kPlanThreads / 32; ++w) grant_b = max(grant_b, sm[1][w][0]), grant_t = max(grant_t, sm[1][w][1]);
  }
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
    for (int t0 = threadIdx.x; t0 < b - a; t0 += 8 * kPlanThreads) {
      int id[8];  // eight reads in flight
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        const int c = (a + min(t0 + u * kPlanThreads, b - a - 1)) >> p.bs_shift;
        id[u] = c < c0 ? part : ids[-(c - c0)];
      }
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        const int t = t0 + u * kPlanThreads;
        if (t >= b - a) break;
        const bool in = id[u] >= 0 && id[u] < p.n_blocks;
        p.slots[at + t] = in ? (id[u] << p.bs_shift) + ((a + t) & (bs - 1)) : -1;
        if (!in) set_error(p.err, WF_DEV_ERR_PAGE);
      }
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
constexpr int kRowWarps = kRowThreads / 32;

// A warp's unit is one group of 16 rows, keys and values.  Where 16
// consecutive rows fill a record (a prefill's do, but seldom from a multiple
// of 16 rows on), the warp of their first row takes them as a whole: the record
// is put together in shared memory and written, or read, 16 bytes a lane.  All
// other rows go one by one, to the same places.
// 48000 rows of 20 heads x 64: in 66 us, bound by issue (67% of the slots; 880
// instructions for 16 rows of a head, keys and values) at 4.5 TB/s; out 47 us,
// bound by HBM at 6.3 TB/s.
struct RowUnit {
  int slab;
  int whole;        // first row of a record that begins in this unit's rows; -1: none
  uint32_t single;  // of the unit's 16 rows, those outside whole records
};
__device__ __forceinline__ RowUnit row_unit(const StoreParams &p, long long unit, int slabs, int lane, int &slot) {
  RowUnit r;
  const int tile = static_cast<int>(unit / slabs);
  r.slab = static_cast<int>(unit - static_cast<long long>(tile) * slabs);
  // lane j holds the slots of rows 16 (tile - 1) + j and 16 (tile + 1) + j
  const int r0 = (tile - 1) * 16 + lane, r1 = r0 + 32;
  const int s0 = r0 >= 0 && r0 < p.n ? p.slots[r0] : -2, s1 = r1 < p.n ? p.slots[r1] : -2;
  const int up0 = __shfl_up_sync(0xffffffffu, s0, 1), up1 = __shfl_up_sync(0xffffffffu, s1, 1), last0 = __shfl_sync(0xffffffffu, s0, 31);
  // bit j: row 16 (tile - 1) + j goes on from the one before it
  const unsigned long long next =
      __ballot_sync(0xffffffffu, lane > 0 && s0 == up0 + 1) | static_cast<unsigned long long>(__ballot_sync(0xffffffffu, s1 == (lane ? up1 : last0) + 1)) << 32;
  const unsigned long long first = __ballot_sync(0xffffffffu, s0 >= 0 && (s0 & 15) == 0);
  // a record starts at bit j: its slot is a multiple of 16 and 15 rows go on
  const auto starts = [&](int j) { return j >= 0 && (first >> j & 1) && (next >> (j + 1) & 0x7fff) == 0x7fff; };
  const int j = lane & 15;
  const int mine = __shfl_sync(0xffffffffu, s0, 16 + j);  // of row 16 tile + j
  const uint32_t begins = __ballot_sync(0xffffffffu, lane < 16 && starts(16 + j)) & 0xffff;
  r.single = __ballot_sync(0xffffffffu, lane < 16 && mine >= 0 && !starts(16 + j - (mine & 15))) & 0xffff;
  r.whole = begins ? tile * 16 + __ffs(begins) - 1 : -1;
  slot = mine;
  return r;
}

// Larger and smaller of each half, NaN if either is.
template <typename T>
using Pair16 = typename std::conditional<std::is_same<T, __half>::value, __half2, __nv_bfloat162>::type;
template <typename T>
__device__ __forceinline__ uint32_t max2_nan(uint32_t a, uint32_t b) {
  const Pair16<T> m = __hmax2_nan(*reinterpret_cast<const Pair16<T> *>(&a), *reinterpret_cast<const Pair16<T> *>(&b));
  return *reinterpret_cast<const uint32_t *>(&m);
}
template <typename T>
__device__ __forceinline__ uint32_t min2_nan(uint32_t a, uint32_t b) {
  const Pair16<T> m = __hmin2_nan(*reinterpret_cast<const Pair16<T> *>(&a), *reinterpret_cast<const Pair16<T> *>(&b));
  return *reinterpret_cast<const uint32_t *>(&m);
}

// Eight values for each of 8 lanes' 8 rows: lane j gets row j's over the lanes.
template <typename F>
__device__ __forceinline__ uint32_t rows_over_lanes(const uint32_t (&v)[8], int j, F op) {
  uint32_t a[4], b[2];
#pragma unroll
  for (int q = 0; q < 4; ++q) a[q] = op(j & 4 ? v[q + 4] : v[q], __shfl_xor_sync(0xffffffffu, j & 4 ? v[q] : v[q + 4], 4));
#pragma unroll
  for (int q = 0; q < 2; ++q) b[q] = op(j & 2 ? a[q + 2] : a[q], __shfl_xor_sync(0xffffffffu, j & 2 ? a[q] : a[q + 2], 2));
  return op(j & 1 ? b[1] : b[0], __shfl_xor_sync(0xffffffffu, j & 1 ? b[0] : b[1], 1));
}

// Quantises one group of 8 rows held by 8 lanes, row c's values 8j .. 8j + 7
// in lane j's w[c]: code = clamp(rint((x - z) / s), -8, 7) + 8, the quotient
// rounded to fp32.  Lane j works out row j's (s, z).  A quotient is the
// numerator times the rounded reciprocal, corrected once by its exact remainder,
// which rounds it correctly (P. Markstein, IBM J. Res. Dev. 34 (1990) 111); it
// has to, for exact halves are common among 16-bit values.  Rows where a
// quotient needs the clamp or s is far from 1 are divided one by one.  All
// lanes call.
template <typename T>
__device__ __forceinline__ void quantise_rows(const uint4 (&w)[8], int lane, uint32_t (&codes)[8], uint32_t (&sz)[8]) {
  using X = Kv4Type<T>;
  const int j = lane & 7;
  // (maximum, -minimum), which are values of the 16-bit type
  uint32_t ends[8];
#pragma unroll
  for (int c = 0; c < 8; ++c) {
    const uint32_t hi = max2_nan<T>(max2_nan<T>(w[c].x, w[c].y), max2_nan<T>(w[c].z, w[c].w));
    const uint32_t lo = min2_nan<T>(min2_nan<T>(w[c].x, w[c].y), min2_nan<T>(w[c].z, w[c].w)) ^ 0x80008000u;
    ends[c] = max2_nan<T>(__byte_perm(hi, lo, 0x5410), __byte_perm(hi, lo, 0x7632));
  }
  const uint32_t end = rows_over_lanes(ends, j, max2_nan<T>);
  const float top = X::lo(end), low = -X::hi(end);
  const bool fine = isfinite(top) && isfinite(low);
  // halves first: max - min may pass the type's range
  const float s = fine ? X::round((0.5f * top - 0.5f * low) / 7.5f) : NAN;
  const float z = fine ? X::round(top - 7.f * s) : NAN;  // 7 s is exact in fp32
  const bool none = !(s > 0.f);  // all codes 8
  const float inv = none ? 0.f : 1.f / s;
  const bool plain = none || (s > 1e-20f && s < 1e20f && (top - z) * inv < 7.49f && (low - z) * inv > -8.49f);
  const uint32_t pair = X::pack(s, z);
  const unsigned slow = __ballot_sync(0xffffffffu, !plain), flat = __ballot_sync(0xffffffffu, none);
#pragma unroll
  for (int c = 0; c < 8; ++c) {
    const int from = (lane & 24) + c;
    sz[c] = __shfl_sync(0xffffffffu, pair, from);
    const float r = __shfl_sync(0xffffffffu, inv, from);
    const bool zero = flat >> from & 1;
    const float zc = zero ? 0.f : X::hi(sz[c]);
    const float2 mz = {-zc, -zc}, rr = {r, r}, magic = {12582920.f, 12582920.f};  // 1.5 * 2^23 + 8
    const uint32_t raw[4] = {w[c].x, w[c].y, w[c].z, w[c].w};
    const float minus_s = -X::lo(sz[c]);
    const float2 ms = {minus_s, minus_s};
    uint32_t sum = 0;  // the codes sit in the low bits of magic's; its own share is taken off below
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 d = add2(make_float2(X::lo(raw[i]), X::hi(raw[i])), mz), t = mul2(d, rr);
      const float2 f = add2(fma2(fma2(t, ms, d), rr, t), magic);
      sum += __float_as_uint(f.x) * (1u << (8 * i));
      sum += __float_as_uint(f.y) * (1u << (8 * i + 4));
    }
    codes[c] = zero ? 0x88888888u : sum - 0x4b400000u * 0x11111111u;
    if (slow >> from & 1) {
      uint32_t exact = 0;
#pragma unroll 1
      for (int i = 0; i < 8; ++i) {
        const uint32_t u = i < 2 ? raw[0] : i < 4 ? raw[1] : i < 6 ? raw[2] : raw[3];
        const float v = i & 1 ? X::hi(u) : X::lo(u);
        exact |= static_cast<uint32_t>(static_cast<int>(fminf(fmaxf(rintf((zc - v) / minus_s), -8.f), 7.f)) + 8) << (4 * i);
      }
      codes[c] = exact;
    }
  }
}

// 8 codes against (s, z), rounded once: s (c - 8) has at most 15 bits, and fp32
// holds the sum that the fused operation rounds unless the two span more than
// its 24.
__device__ __forceinline__ uint4 dequantise8(uint32_t w, uint32_t sz, __nv_bfloat16) {
  uint32_t r[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t u = and_or(w >> (4 * i), 0x000f000fu, 0x43004300u), eight = 0x43084308u;  // 128 + c, 136
    const uint32_t s2 = __byte_perm(sz, 0, 0x1010), z2 = __byte_perm(sz, 0, 0x3232);
    const __nv_bfloat162 c = __hsub2(*reinterpret_cast<const __nv_bfloat162 *>(&u), *reinterpret_cast<const __nv_bfloat162 *>(&eight));
    const __nv_bfloat162 v = __hfma2(c, *reinterpret_cast<const __nv_bfloat162 *>(&s2), *reinterpret_cast<const __nv_bfloat162 *>(&z2));
    r[i] = *reinterpret_cast<const uint32_t *>(&v);
  }
  return make_uint4(__byte_perm(r[0], r[1], 0x5410), __byte_perm(r[2], r[3], 0x5410), __byte_perm(r[0], r[1], 0x7632), __byte_perm(r[2], r[3], 0x7632));
}
__device__ __forceinline__ uint4 dequantise8(uint32_t w, uint32_t sz, __half) {
  uint32_t r[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t u = and_or(w >> (4 * i), 0x000f000fu, 0x64006400u), eight = 0x64086408u;  // 1024 + c, 1032
    const uint32_t s2 = __byte_perm(sz, 0, 0x1010), z2 = __byte_perm(sz, 0, 0x3232);
    const __half2 c = __hsub2(*reinterpret_cast<const __half2 *>(&u), *reinterpret_cast<const __half2 *>(&eight));
    const __half2 v = __hfma2(c, *reinterpret_cast<const __half2 *>(&s2), *reinterpret_cast<const __half2 *>(&z2));
    r[i] = *reinterpret_cast<const uint32_t *>(&v);
  }
  return make_uint4(__byte_perm(r[0], r[1], 0x5410), __byte_perm(r[2], r[3], 0x5410), __byte_perm(r[0], r[1], 0x7632), __byte_perm(r[2], r[3], 0x7632));
}

// The places of a row's 8 codes from dim 8 j on in a record.
__device__ __forceinline__ void put_codes(unsigned char *rec, int at, int j, int is_v, uint32_t codes) {
  if (is_v) {
    *reinterpret_cast<uint16_t *>(rec + kv4_val_offset(at, j, 0)) = static_cast<uint16_t>(codes);
    *reinterpret_cast<uint16_t *>(rec + kv4_val_offset(at, j, 1)) = static_cast<uint16_t>(codes >> 16);
  } else {
    *reinterpret_cast<uint32_t *>(rec + at * 32 + j * 4) = codes;
  }
}
__device__ __forceinline__ uint32_t get_codes(const unsigned char *rec, int at, int j, int is_v) {
  if (is_v)
    return *reinterpret_cast<const uint16_t *>(rec + kv4_val_offset(at, j, 0)) |
           static_cast<uint32_t>(*reinterpret_cast<const uint16_t *>(rec + kv4_val_offset(at, j, 1))) << 16;
  return *reinterpret_cast<const uint32_t *>(rec + at * 32 + j * 4);
}

template <typename T>
__global__ void __launch_bounds__(kRowThreads, 4) kv4_store_kernel(const StoreParams p) {
  __shared__ __align__(16) unsigned char records[kRowWarps][kKv4Rec];
  pdl_wait();
  pdl_launch_dependents();
  const int lane = threadIdx.x & 31, j = lane & 7, sub = lane >> 3;
  unsigned char *rec = records[threadIdx.x >> 5];
  const int slabs = p.pool.heads * p.pool.groups;
  const long long units = (static_cast<long long>(p.n) + 15) / 16 * slabs;
  for (long long unit = static_cast<long long>(blockIdx.x) * kRowWarps + (threadIdx.x >> 5); unit < units;
       unit += static_cast<long long>(gridDim.x) * kRowWarps) {
    int slot;
    const RowUnit u = row_unit(p, unit, slabs, lane, slot);
    const int tile = static_cast<int>(unit / slabs);
    const T *k = static_cast<const T *>(p.k) + u.slab * 64 + j * 8, *v = static_cast<const T *>(p.v) + u.slab * 64 + j * 8;
    if (u.whole >= 0) {
      const int at = p.slots[u.whole], block = at >> p.pool.bs_shift;
      uint4 w[8];
      uint32_t codes[8], sz[8];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const long long row = u.whole + i * 4 + sub;
        w[i] = *reinterpret_cast<const uint4 *>(k + row * p.k_stride);
        w[4 + i] = *reinterpret_cast<const uint4 *>(v + row * p.v_stride);
      }
      quantise_rows<T>(w, lane, codes, sz);
      __syncwarp();
#pragma unroll
      for (int c = 0; c < 8; ++c) {
        const int r = (c & 3) * 4 + sub;
        put_codes(rec, r, j, c >> 2, codes[c]);
        if (j == 0) *reinterpret_cast<uint32_t *>(rec + kv4_scale_offset(r, c >> 2)) = sz[c];
      }
      __syncwarp();
      if (block < p.pool.n_blocks) {
        uint4 *dst = reinterpret_cast<uint4 *>(kv4_record(p.pool, block, 0, u.slab, (at & (p.pool.bs - 1)) >> 4));
#pragma unroll
        for (int i = 0; i < 3; ++i)
          if (i * 32 + lane < kKv4Rec / 16) dst[i * 32 + lane] = reinterpret_cast<const uint4 *>(rec)[i * 32 + lane];
      } else if (lane == 0) {
        set_error(p.err, WF_DEV_ERR_PAGE);
      }
    }
    if (u.single) {
      uint4 w[8];
      uint32_t codes[8], sz[8];
      int at[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int r = i * 4 + sub;
        at[i] = __shfl_sync(0xffffffffu, slot, r);
        if (!(u.single >> r & 1)) at[i] = -1;
        if (at[i] >= 0 && at[i] >> p.pool.bs_shift >= p.pool.n_blocks) {
          if (j == 0) set_error(p.err, WF_DEV_ERR_PAGE);
          at[i] = -1;
        }
        w[i] = w[4 + i] = make_uint4(0, 0, 0, 0);
        if (at[i] >= 0) {
          const long long row = static_cast<long long>(tile) * 16 + r;
          w[i] = *reinterpret_cast<const uint4 *>(k + row * p.k_stride);
          w[4 + i] = *reinterpret_cast<const uint4 *>(v + row * p.v_stride);
        }
      }
      quantise_rows<T>(w, lane, codes, sz);
#pragma unroll
      for (int c = 0; c < 8; ++c) {
        if (at[c & 3] < 0) continue;
        const int pos = at[c & 3] & (p.pool.bs - 1);
        unsigned char *dst = kv4_record(p.pool, at[c & 3] >> p.pool.bs_shift, 0, u.slab, pos >> 4);
        put_codes(dst, pos & 15, j, c >> 2, codes[c]);
        if (j == 0) *reinterpret_cast<uint32_t *>(dst + kv4_scale_offset(pos & 15, c >> 2)) = sz[c];
      }
    }
  }
}

template <typename T>
__global__ void __launch_bounds__(kRowThreads) kv4_load_kernel(const StoreParams p) {
  __shared__ __align__(16) unsigned char records[kRowWarps][kKv4Rec];
  pdl_wait();
  pdl_launch_dependents();
  const int lane = threadIdx.x & 31, j = lane & 7, sub = lane >> 3;
  unsigned char *rec = records[threadIdx.x >> 5];
  const int slabs = p.pool.heads * p.pool.groups;
  const long long units = (static_cast<long long>(p.n) + 15) / 16 * slabs;
  for (long long unit = static_cast<long long>(blockIdx.x) * kRowWarps + (threadIdx.x >> 5); unit < units;
       unit += static_cast<long long>(gridDim.x) * kRowWarps) {
    int slot;
    const RowUnit u = row_unit(p, unit, slabs, lane, slot);
    const int tile = static_cast<int>(unit / slabs);
    T *k = static_cast<T *>(p.k_out) + u.slab * 64 + j * 8, *v = static_cast<T *>(p.v_out) + u.slab * 64 + j * 8;
    if (u.whole >= 0) {
      const int at = p.slots[u.whole], block = at >> p.pool.bs_shift;
      const bool in = block < p.pool.n_blocks;
      if (!in && lane == 0) set_error(p.err, WF_DEV_ERR_PAGE);
      __syncwarp();
      const uint4 *src = reinterpret_cast<const uint4 *>(kv4_record(p.pool, in ? block : 0, 0, u.slab, (at & (p.pool.bs - 1)) >> 4));
#pragma unroll
      for (int i = 0; i < 3; ++i)
        if (i * 32 + lane < kKv4Rec / 16) reinterpret_cast<uint4 *>(rec)[i * 32 + lane] = src[i * 32 + lane];
      __syncwarp();
#pragma unroll
      for (int is_v = 0; is_v < 2; ++is_v)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int r = i * 4 + sub;
          uint4 x = dequantise8(get_codes(rec, r, j, is_v), *reinterpret_cast<const uint32_t *>(rec + kv4_scale_offset(r, is_v)), T());
          if (!in) x = make_uint4(0, 0, 0, 0);
          *reinterpret_cast<uint4 *>((is_v ? v : k) + (u.whole + r) * (is_v ? p.v_stride : p.k_stride)) = x;
        }
    }
    // rows outside whole records, and those without a slot, which read as zeros
    const uint32_t rest = u.single | (__ballot_sync(0xffffffffu, lane < 16 && tile * 16 + lane < p.n && slot < 0) & 0xffff);
    if (rest) {
#pragma unroll
      for (int is_v = 0; is_v < 2; ++is_v)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int r = i * 4 + sub, at = __shfl_sync(0xffffffffu, slot, r);
          if (!(rest >> r & 1)) continue;
          uint4 x = {0, 0, 0, 0};
          if (at >= 0 && at >> p.pool.bs_shift < p.pool.n_blocks) {
            const int pos = at & (p.pool.bs - 1);
            const unsigned char *src = kv4_record(p.pool, at >> p.pool.bs_shift, 0, u.slab, pos >> 4);
            x = dequantise8(get_codes(src, pos & 15, j, is_v), *reinterpret_cast<const uint32_t *>(src + kv4_scale_offset(pos & 15, is_v)), T());
          } else if (at >= 0 && j == 0) {
            set_error(p.err, WF_DEV_ERR_PAGE);
          }
          *reinterpret_cast<uint4 *>((is_v ? v : k) + (static_cast<long long>(tile) * 16 + r) * (is_v ? p.v_stride : p.k_stride)) = x;
        }
    }
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
  int32_t *moves, *gone, *gone_n, *n_free_copy;  // scratch
  uint32_t *err;
};
constexpr int kReorderThreads = 256;

// One CTA per request: its table columns (each by one thread, which reads the
// column before it writes it), the ids that no beam holds any more in order,
// and the copies of last blocks that the second kernel makes.  MAXW: 4, 8 or
// 16, the least that holds the beams; a column's comparisons grow with its
// square.  Bound by its chain of reads (parents, lengths, columns) and, with
// the second kernel, by two launches: 11.7 to 12.6 us for one request's 5 beams.
template <int MAXW>
__global__ void __launch_bounds__(kReorderThreads) beam_tables_kernel(const ReorderParams p) {
  pdl_wait();
  pdl_launch_dependents();
  const int W = p.W, req = blockIdx.x, tid = threadIdx.x, lane = tid & 31, wp = tid >> 5;
  __shared__ int par_s[MAXW], from_s[MAXW], spare[MAXW];
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
  const int full = len >> p.pool.bs_shift, rem = len & (bs - 1), cols = full + (rem ? 1 : 0);
  if (wp == 0) {
    int v = -1;
    if (lane < W) {
      v = p.parent[static_cast<size_t>(req) * W + lane];
      if (v < -1 || v >= W) err |= WF_DEV_ERR_PAGE, v = -1;
    }
    // a parent's first child keeps its last block; the k-th other beam takes that of the k-th without children
    const unsigned same = __match_any_sync(0xffffffffu, v);
    const bool keeps = v >= 0 && (same & ((1u << lane) - 1)) == 0;
    const unsigned parents = __reduce_or_sync(0xffffffffu, v >= 0 ? 1u << v : 0u), all = (1u << W) - 1;
    const unsigned dead = ~parents & all, takers = __ballot_sync(0xffffffffu, lane < W && !keeps);
    if (dead >> lane & 1) spare[__popc(dead & ((1u << lane) - 1))] = lane;
    __syncwarp();
    if (lane < W) {
      const int from = keeps ? v : spare[__popc(takers & ((1u << lane) - 1))];
      par_s[lane] = v, from_s[lane] = from;
      int src = -1, dst = -1;
      if (rem && v >= 0 && from != v) {
        src = in[v * p.stride + full];
        dst = in[from * p.stride + full];
        if (src < 0 || src >= p.pool.n_blocks || dst < 0 || dst >= p.pool.n_blocks) err |= WF_DEV_ERR_PAGE, src = dst = -1;
      }
      *reinterpret_cast<int4 *>(p.moves + (static_cast<size_t>(req) * W + lane) * 4) = make_int4(src, dst, (rem + 15) / 16, 0);
    }
    if (req == 0 && lane == 0) *p.n_free_copy = *p.n_free;
  }
  __syncthreads();  // (the copies' entries are read before any is written)
  int par[MAXW], from[MAXW];
  bool over = true;
#pragma unroll
  for (int w = 0; w < MAXW; ++w) {
    par[w] = w < W ? par_s[w] : -1, from[w] = w < W ? from_s[w] : -1;
    over = over && par[w] < 0;
  }
  int base = 0;
  for (int c0 = 0; c0 < cols; c0 += kReorderThreads) {
    const int c = c0 + tid;
    int old[MAXW], now[MAXW];
    uint32_t dead = 0;
    if (c < cols) {
#pragma unroll
      for (int w = 0; w < MAXW; ++w) old[w] = w < W ? in[static_cast<size_t>(w) * p.stride + c] : -1;
#pragma unroll
      for (int w = 0; w < MAXW; ++w) {
        const int f = c < full ? par[w] : (over ? -1 : from[w]);
        now[w] = -1;
#pragma unroll
        for (int q = 0; q < MAXW; ++q) now[w] = q == f ? old[q] : now[w];
        if (w < W) out[static_cast<size_t>(w) * p.stride + c] = now[w];
      }
#pragma unroll
      for (int w = 0; w < MAXW; ++w) {
        if (old[w] >= p.pool.n_blocks) err |= WF_DEV_ERR_PAGE;  // no block of the pool: not one to push
        bool held = old[w] < 0 || old[w] >= p.pool.n_blocks;
#pragma unroll
        for (int q = 0; q < MAXW; ++q) held |= now[q] == old[w] || (q < w && old[q] == old[w]);
        if (!held) dead |= 1u << w;
      }
    }
    const int cnt = __popc(dead);
    int scan = cnt;
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
      const int v = __shfl_up_sync(0xffffffffu, scan, off);
      if (lane >= off) scan += v;
    }
    if (lane == 31) wsum[wp] = scan;
    __syncthreads();
    int total = 0, before = 0;
#pragma unroll
    for (int i = 0; i < kReorderThreads / 32; ++i) {
      if (i < wp) before += wsum[i];
      total += wsum[i];
    }
    int at = base + before + scan - cnt;
#pragma unroll
    for (int w = 0; w < MAXW; ++w)
      if (dead >> w & 1) gone[at++] = old[w];
    base += total;
    __syncthreads();
  }
  if (tid == 0) p.gone_n[req] = base;
  if (err) set_error(p.err, err);
}

// grid (n_req * W, layers): the copies of last blocks, 16 positions at a time;
// in layer 0 the first CTA of a request also pushes its freed ids.  16 requests
// x 5 beams move 41 MB in 32 layers; with the first kernel 12.7 to 14.1 us
// (with one read in flight a thread instead of six 1.7 more).
__global__ void __launch_bounds__(kReorderThreads) beam_moves_kernel(const ReorderParams p) {
  pdl_wait();
  pdl_launch_dependents();
  const int req = blockIdx.x / p.W;
  const int4 m = *reinterpret_cast<const int4 *>(p.moves + static_cast<size_t>(blockIdx.x) * 4);
  if (m.x >= 0) {
    const int chunk = m.z * (kKv4Rec / 16);  // 16-byte pieces of a slab that are in use
    const int slabs = p.pool.heads * p.pool.groups, per = (p.pool.bs >> 4) * (kKv4Rec / 16);
    unsigned char *layer = p.pool.base + static_cast<long long>(blockIdx.y) * p.layer_stride;
    const uint4 *src = reinterpret_cast<const uint4 *>(layer + m.x * p.block_bytes);
    uint4 *dst = reinterpret_cast<uint4 *>(layer + m.y * p.block_bytes);
    constexpr int kAhead = 6;  // reads in flight
    for (int i0 = threadIdx.x; i0 < slabs * chunk; i0 += kAhead * kReorderThreads) {
      uint4 v[kAhead];
      int at[kAhead];
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        const int i = min(i0 + u * kReorderThreads, slabs * chunk - 1), slab = i / chunk;
        at[u] = slab * per + i - slab * chunk;
        v[u] = src[at[u]];
      }
#pragma unroll
      for (int u = 0; u < kAhead; ++u)
        if (i0 + u * kReorderThreads < slabs * chunk) dst[at[u]] = v[u];
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
  static PerDevice count;
  const int dev = current_device();
  return count.get(dev, [&] {
    int v = 0;
    return cudaDeviceGetAttribute(&v, cudaDevAttrMultiProcessorCount, dev) == cudaSuccess ? v : 0;
  });
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
  if (static_cast<int64_t>(n_blocks) * block_size > INT32_MAX || static_cast<int64_t>(table_stride) * block_size > INT32_MAX)
    return WF_ERR_INVALID;
  if (n > kPlanRequests || slots_cap > kPlanSlots) return WF_ERR_UNSUPPORTED;
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
  const long long units = (static_cast<long long>(p->n) + 15) / 16 * p->pool.heads * p->pool.groups;
  const long long want = (units + kRowWarps - 1) / kRowWarps;
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

// scratch: copies [n_req * beams][4], freed ids [n_req][beams * stride], their
// counts [n_req], the free count
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
      beams <= 0 || table_stride <= 0 || !aligned16(d_scratch))
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
  p.moves = static_cast<int32_t *>(d_scratch);
  p.gone = p.moves + rows * 4;
  p.gone_n = p.gone + rows * table_stride;
  p.n_free_copy = p.gone_n + n_req;
  p.err = d_err;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  void *args[] = {&p};
  const void *tables = beams <= 4   ? reinterpret_cast<const void *>(beam_tables_kernel<4>)
                       : beams <= 8 ? reinterpret_cast<const void *>(beam_tables_kernel<8>)
                                    : reinterpret_cast<const void *>(beam_tables_kernel<16>);
  if (launch_pdl(tables, n_req, kReorderThreads, 0, args, s) != cudaSuccess ||
      launch_pdl(reinterpret_cast<const void *>(beam_moves_kernel), dim3(static_cast<unsigned>(rows), p.n_layers), kReorderThreads, 0,
                 args, s) != cudaSuccess)
    return WF_ERR_CUDA;
  return WF_OK;
}

}  // extern "C"
