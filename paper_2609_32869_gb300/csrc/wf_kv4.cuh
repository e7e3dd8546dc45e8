// The 4-bit cache's record format and the helpers its kernels share.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "../../include/wf.h"
#include "wf_internal.h"
#include "wf_per_device.h"

namespace wf {

// SMs that a call's work is cut for.  A constant: the scratch sizes depend on
// the cut and are asked for without a device.
constexpr int kSms = 152;

// A record: 16 positions of one group of 64 values, keys and values.
//   key codes    [position][32 bytes], dims 2b and 2b + 1 in byte b (low nibble first)
//   value codes  [dims / 8 = r][position pair t][positions 8.. = u][dims / 4 % 2 = h][odd position][2 bytes]:
//                lane 4 r + t of a warp finds the positions 2t, 2t + 1, 2t + 8,
//                2t + 9 of the dims 8r .. 8r + 7 in 16 bytes of its own, two
//                positions of the same dim 16 bits apart
//   (s, z)       [position % 8][keys, values][position / 8]
constexpr int kKv4Rec = WF_KV4_RECORD;
constexpr int kKv4ValOff = 512;
constexpr int kKv4ScaleOff = 1024;

__host__ __device__ __forceinline__ int kv4_val_offset(int pos, int r, int h) {
  return kKv4ValOff + (r * 4 + ((pos & 7) >> 1)) * 16 + (pos >> 3) * 8 + h * 4 + (pos & 1) * 2;
}
__host__ __device__ __forceinline__ int kv4_scale_offset(int pos, int is_value) {
  return kKv4ScaleOff + (pos & 7) * 16 + is_value * 8 + (pos >> 3) * 4;
}

struct Kv4Pool {  // a checked wf_kv4_pool at one layer
  unsigned char *base;
  int n_blocks, bs, bs_shift, heads, groups;  // groups: of a head
};

inline bool kv4_shape_ok(int32_t bs, int32_t heads, int32_t dim) {
  return (bs == 16 || bs == 32 || bs == 64) && heads > 0 && heads <= 4096 && (dim == 64 || dim == 128);
}
inline size_t kv4_block_bytes(int bs, int heads, int dim) {
  return static_cast<size_t>(heads) * (dim / WF_KV4_GROUP) * (bs / 16) * kKv4Rec;
}
// Host checks of a pool and a layer of it; fills `out`.
inline wf_status kv4_pool_check(const wf_kv4_pool *p, int32_t layer, Kv4Pool *out, int64_t *layer_stride) {
  if (!p || !p->d_base || (reinterpret_cast<uintptr_t>(p->d_base) & 15) || p->n_layers <= 0 || p->n_blocks <= 0 ||
      layer < 0 || layer >= p->n_layers)
    return WF_ERR_INVALID;
  if (!kv4_shape_ok(p->block_size, p->n_kv_heads, p->head_dim) || (p->dtype != WF_BF16 && p->dtype != WF_F16))
    return WF_ERR_UNSUPPORTED;
  if (static_cast<int64_t>(p->n_blocks) * p->block_size > INT32_MAX) return WF_ERR_INVALID;
  const int64_t need = static_cast<int64_t>(kv4_block_bytes(p->block_size, p->n_kv_heads, p->head_dim)) * p->n_blocks;
  const int64_t stride = p->layer_stride ? p->layer_stride : need;
  if (stride < need || (stride & 15)) return WF_ERR_INVALID;
  out->base = static_cast<unsigned char *>(p->d_base) + stride * layer;
  out->n_blocks = p->n_blocks;
  out->bs = p->block_size;
  out->bs_shift = p->block_size == 16 ? 4 : (p->block_size == 32 ? 5 : 6);
  out->heads = p->n_kv_heads;
  out->groups = p->head_dim / WF_KV4_GROUP;
  if (layer_stride) *layer_stride = stride;
  return WF_OK;
}

// Record of 16-position tile `tile` of a block, head `h`, group `g`.
__device__ __forceinline__ unsigned char *kv4_record(const Kv4Pool &p, int block, int h, int g, int tile) {
  const long long slab = static_cast<long long>(block) * (p.heads * p.groups) + h * p.groups + g;
  return p.base + (slab * (p.bs >> 4) + tile) * kKv4Rec;
}

inline cudaError_t launch_pdl(const void *fn, dim3 grid, dim3 block, size_t smem, void **args, cudaStream_t s,
                              int cluster_y = 1) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = block;
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = 1;
  attr[1].val.clusterDim.y = cluster_y;
  attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = cluster_y > 1 ? 2 : 1;
  return cudaLaunchKernelExC(&cfg, fn, args);
}

// The device that a call runs on; -1 where there is none.
inline int current_device() {
  int dev = -1;
  return cudaGetDevice(&dev) == cudaSuccess ? dev : -1;
}
inline bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// Two fp32 operations in one instruction.
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
  float2 d;
  asm("add.rn.f32x2 %0, %1, %2;"
      : "=l"(*reinterpret_cast<unsigned long long *>(&d))
      : "l"(*reinterpret_cast<const unsigned long long *>(&a)), "l"(*reinterpret_cast<const unsigned long long *>(&b)));
  return d;
}
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
  float2 d;
  asm("fma.rn.f32x2 %0, %1, %2, %3;"
      : "=l"(*reinterpret_cast<unsigned long long *>(&d))
      : "l"(*reinterpret_cast<const unsigned long long *>(&a)), "l"(*reinterpret_cast<const unsigned long long *>(&b)),
        "l"(*reinterpret_cast<const unsigned long long *>(&c)));
  return d;
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
  float2 d;
  asm("mul.rn.f32x2 %0, %1, %2;"
      : "=l"(*reinterpret_cast<unsigned long long *>(&d))
      : "l"(*reinterpret_cast<const unsigned long long *>(&a)), "l"(*reinterpret_cast<const unsigned long long *>(&b)));
  return d;
}

__device__ __forceinline__ float max3(float a, float b, float c) {
  float d;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}

// (w & mask) | magic in one instruction, which the compiler makes two of.
__device__ __forceinline__ uint32_t and_or(uint32_t w, uint32_t mask, uint32_t magic) {
  uint32_t d;
  asm("lop3.b32 %0, %1, %2, %3, 0xea;" : "=r"(d) : "r"(w), "r"(mask), "r"(magic));
  return d;
}

// The largest of a warp's values (no NaN, unless all are).
__device__ __forceinline__ float warp_max(float v) {
  float m;
  asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(m) : "f"(v));
  return m;
}

template <typename T>
struct Kv4Type;
template <>
struct Kv4Type<__nv_bfloat16> {
  static __device__ __forceinline__ float lo(uint32_t w) { return __uint_as_float(w << 16); }
  static __device__ __forceinline__ float hi(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }
  static __device__ __forceinline__ uint32_t pack(float a, float b) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t *>(&v);
  }
  static __device__ __forceinline__ float round(float v) { return __bfloat162float(__float2bfloat16_rn(v)); }
};
template <>
struct Kv4Type<__half> {
  static __device__ __forceinline__ float lo(uint32_t w) {
    return __half2float(__ushort_as_half(static_cast<unsigned short>(w & 0xffff)));
  }
  static __device__ __forceinline__ float hi(uint32_t w) {
    return __half2float(__ushort_as_half(static_cast<unsigned short>(w >> 16)));
  }
  static __device__ __forceinline__ uint32_t pack(float a, float b) {
    const __half2 v = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t *>(&v);
  }
  static __device__ __forceinline__ float round(float v) { return __half2float(__float2half_rn(v)); }
};

}  // namespace wf
