// The 8-bit cache's record format.
#pragma once
#include <cuda_fp8.h>

#include "wf_ops.cuh"

namespace wf {

// A record: 16 positions of a head.  Of every group of 64 dims
//   key codes    [position][dim]
//   value codes  [dims % 4 >= 2 = h][lane][odd dim][a][odd position]: lane
//                4 r + t of a warp finds in two 16-byte pieces of its own the
//                dims 8r .. 8r + 7 of the positions 2t, 2t + 1 (a = 0: dims below
//                8r + 4, a = 1: the others), 2t + 8 and 2t + 9 (a = 2, 3), two
//                positions of the same dim beside each other
// and then 2^e of the keys and of the values in fp32 and 8 bytes of zeros.
constexpr int kKv8Group = 2048;  // bytes of 64 dims
constexpr int kKv8Low = -60, kKv8High = 36;  // e

struct Kv8Pool {  // a checked wf_kv8_pool at one layer
  unsigned char *base;
  int n_blocks, bs, bs_shift, heads, groups;  // groups of 64 dims of a head
};

__host__ __device__ __forceinline__ int kv8_record_bytes(int groups) { return groups * kKv8Group + 16; }

inline bool kv8_shape_ok(int32_t bs, int32_t heads, int32_t dim) {
  return (bs == 16 || bs == 32 || bs == 64) && heads > 0 && heads <= 4096 && (dim == 64 || dim == 128);
}
inline size_t kv8_block_bytes(int bs, int heads, int dim) {
  return static_cast<size_t>(heads) * (bs / 16) * kv8_record_bytes(dim / 64);
}
// Host checks of a pool and a layer of it; fills `out`.
inline wf_status kv8_pool_check(const wf_kv8_pool *p, int32_t layer, Kv8Pool *out) {
  if (!p || !p->d_base || (reinterpret_cast<uintptr_t>(p->d_base) & 15) || p->n_layers <= 0 || p->n_blocks <= 0 || layer < 0 ||
      layer >= p->n_layers)
    return WF_ERR_INVALID;
  if (!kv8_shape_ok(p->block_size, p->n_kv_heads, p->head_dim) || (p->dtype != WF_BF16 && p->dtype != WF_F16)) return WF_ERR_UNSUPPORTED;
  if (static_cast<int64_t>(p->n_blocks) * p->block_size > INT32_MAX) return WF_ERR_INVALID;
  const int64_t need = static_cast<int64_t>(kv8_block_bytes(p->block_size, p->n_kv_heads, p->head_dim)) * p->n_blocks;
  const int64_t stride = p->layer_stride ? p->layer_stride : need;
  if (stride < need || (stride & 15)) return WF_ERR_INVALID;
  out->base = static_cast<unsigned char *>(p->d_base) + stride * layer;
  out->n_blocks = p->n_blocks;
  out->bs = p->block_size;
  out->bs_shift = p->block_size == 16 ? 4 : (p->block_size == 32 ? 5 : 6);
  out->heads = p->n_kv_heads;
  out->groups = p->head_dim / 64;
  return WF_OK;
}

// Record of the 16 positions `tile` of a block, head `h`.
__device__ __forceinline__ unsigned char *kv8_record(const Kv8Pool &p, int block, int h, int tile) {
  return p.base + ((static_cast<long long>(block) * p.heads + h) * (p.bs >> 4) + tile) * kv8_record_bytes(p.groups);
}

// Two codes as a pair of fp16, which holds them exactly.
__device__ __forceinline__ uint32_t codes_to_f16(uint32_t two) {
  uint32_t d;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(d) : "h"(static_cast<unsigned short>(two)));
  return d;
}
__device__ __forceinline__ float2 codes_to_f32(uint32_t two) {
  const uint32_t h = codes_to_f16(two);
  return __half22float2(*reinterpret_cast<const __half2 *>(&h));
}
// x in the low byte, y in the next: nearest even, magnitudes above 448 as 448, NaN as NaN.
__device__ __forceinline__ uint32_t f32_to_codes(float x, float y) {
  unsigned short d;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(d) : "f"(y), "f"(x));
  return d;
}
__device__ __forceinline__ float two_to(int e) { return __int_as_float((e + 127) << 23); }  // -126 <= e <= 127

}  // namespace wf
