// Attention over the paged 8-bit cache (softmax(scale q K^T) V).
#include <algorithm>
#include <climits>

#include "wf_device.cuh"
#include "wf_kv8.cuh"

namespace wf {

struct Kv8AttnParams {
  Kv8Pool pool;
  const void *q;
  void *out;
  long long q_stride, out_stride;
  const int32_t *table, *len;
  int table_stride, n_seq, rps, n_heads, causal, max_len;
  float scale;
  uint32_t *err;
};

// A warp per query row and head, a position at a time.
template <typename T, int G>
__global__ void __launch_bounds__(128) kv8_attention_kernel(const Kv8AttnParams p) {
  using X = Type16<T>;
  pdl_wait();
  pdl_launch_dependents();
  const int lane = threadIdx.x & 31;
  const long long unit = static_cast<long long>(blockIdx.x) * 4 + (threadIdx.x >> 5);
  if (unit >= static_cast<long long>(p.n_seq) * p.rps * p.n_heads) return;
  const int h = static_cast<int>(unit % p.n_heads), kh = h / (p.n_heads / p.pool.heads);
  const long long row = unit / p.n_heads;
  const int seq = static_cast<int>(row / p.rps), j = static_cast<int>(row % p.rps);
  const int raw = p.len[seq], len = min(max(raw, 0), p.max_len);
  if (raw != len && lane == 0) set_error(p.err, raw < 0 ? WF_DEV_ERR_PAGE : WF_DEV_ERR_CAPACITY);
  const int limit = p.causal ? len - (p.rps - 1 - j) : len;
  // lane l holds the dims 2 l and 2 l + 1 of every group
  float2 q[G], o[G] = {};
#pragma unroll
  for (int g = 0; g < G; ++g) {
    const uint32_t w = *reinterpret_cast<const uint32_t *>(static_cast<const T *>(p.q) + row * p.q_stride + h * (G * 64) + g * 64 + lane * 2);
    q[g] = make_float2(X::lo(w), X::hi(w));
  }
  float m = -INFINITY, l = 0.f;
  const int32_t *table = p.table + static_cast<long long>(seq) * p.table_stride;
  for (int pos = 0; pos < limit; ++pos) {
    const int block = table[pos >> p.pool.bs_shift];
    if (static_cast<uint32_t>(block) >= static_cast<uint32_t>(p.pool.n_blocks)) {
      if (lane == 0) set_error(p.err, WF_DEV_ERR_PAGE);
      continue;
    }
    const unsigned char *rec = kv8_record(p.pool, block, kh, (pos & (p.pool.bs - 1)) >> 4);
    const float2 sc = *reinterpret_cast<const float2 *>(rec + G * kKv8Group);
    float x = 0.f;
    float2 v[G];
#pragma unroll
    for (int g = 0; g < G; ++g) {
      const unsigned char *at = rec + g * kKv8Group;
      const float2 k = codes_to_f32(*reinterpret_cast<const unsigned short *>(at + pos % 16 * 64 + lane * 2));
      x += q[g].x * k.x + q[g].y * k.y;
      const unsigned char *va = at + 1024 + lane % 2 * 512 + lane / 4 * 64 + pos / 2 % 4 * 16 + pos / 8 % 2 * 4 + lane / 2 % 2 * 2 + pos % 2;
      v[g] = codes_to_f32(va[0] | va[8] << 8);
    }
    x = warp_sum(x) * (sc.x * p.scale);
    const float next = fmaxf(m, x), keep = m == -INFINITY ? 0.f : __expf(m - next), w = x == -INFINITY ? 0.f : __expf(x - next);
    l = l * keep + w;
    m = next;
#pragma unroll
    for (int g = 0; g < G; ++g) o[g].x = o[g].x * keep + w * sc.y * v[g].x, o[g].y = o[g].y * keep + w * sc.y * v[g].y;
  }
  const float inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
  for (int g = 0; g < G; ++g)
    *reinterpret_cast<uint32_t *>(static_cast<T *>(p.out) + row * p.out_stride + h * (G * 64) + g * 64 + lane * 2) = X::pack(o[g].x * inv, o[g].y * inv);
}

}  // namespace wf

using namespace wf;

constexpr int kK8Longest = INT_MAX - 1023;  // a step past the last position is still an int

extern "C" {

size_t wf_kv8_attention_scratch_bytes(int32_t n_seq, int32_t rps, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim, int32_t max_len) {
  return 0;
}

wf_status wf_kv8_attention(const wf_kv8_pool *pool, int32_t layer, const void *d_q, int64_t q_stride, const int32_t *d_table,
                           int32_t table_stride, const int32_t *d_len, int32_t n_seq, int32_t rps, int32_t n_heads, int32_t causal,
                           float scale, int32_t max_len, void *d_out, int64_t out_stride, void *d_scratch, size_t scratch_bytes,
                           uint32_t *d_err, void *stream) {
  Kv8AttnParams p = {};
  const wf_status st = kv8_pool_check(pool, layer, &p.pool);
  if (st != WF_OK) return st;
  const int64_t d = static_cast<int64_t>(n_heads) * pool->head_dim;
  if (!d_q || !d_table || !d_len || !d_out || n_seq <= 0 || rps <= 0 || n_heads <= 0 || n_heads % pool->n_kv_heads || max_len <= 0 ||
      table_stride < 0 || !aligned16(d_q) || !aligned16(d_out) || q_stride % 8 || out_stride % 8 || q_stride < d || out_stride < d ||
      !(scale == scale))
    return WF_ERR_INVALID;
  // every position up to max_len needs a table column (stride 0: one row that the caller made long enough)
  if (table_stride && static_cast<int64_t>(table_stride) * pool->block_size < max_len) return WF_ERR_INVALID;
  const int64_t rows = static_cast<int64_t>(rps) * (n_heads / pool->n_kv_heads);
  if (static_cast<int64_t>(n_seq) * pool->n_kv_heads > INT32_MAX || rows > 65535 * 8LL || n_heads / pool->n_kv_heads > 4096 ||
      max_len > kK8Longest)
    return WF_ERR_UNSUPPORTED;
  p.q = d_q, p.out = d_out, p.q_stride = q_stride, p.out_stride = out_stride;
  p.table = d_table, p.len = d_len, p.table_stride = table_stride;
  p.n_seq = n_seq, p.rps = rps, p.n_heads = n_heads, p.causal = causal != 0, p.max_len = max_len, p.scale = scale, p.err = d_err;
  using B = __nv_bfloat16;
  const bool wide = pool->head_dim == 128;
  const void *fn = pool->dtype == WF_F16 ? (wide ? reinterpret_cast<const void *>(kv8_attention_kernel<__half, 2>) : reinterpret_cast<const void *>(kv8_attention_kernel<__half, 1>))
                                         : (wide ? reinterpret_cast<const void *>(kv8_attention_kernel<B, 2>) : reinterpret_cast<const void *>(kv8_attention_kernel<B, 1>));
  const int64_t units = static_cast<int64_t>(n_seq) * rps * n_heads;
  if ((units + 3) / 4 > INT32_MAX) return WF_ERR_UNSUPPORTED;
  void *args[] = {&p};
  return launch_pdl(fn, static_cast<unsigned>((units + 3) / 4), 128, 0, args, static_cast<cudaStream_t>(stream)) == cudaSuccess ? WF_OK : WF_ERR_CUDA;
}

}  // extern "C"
