// The 4-bit cache's record format.
#pragma once
#include "wf_ops.cuh"

namespace wf {

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

template <typename T>
using Kv4Type = Type16<T>;

}  // namespace wf
