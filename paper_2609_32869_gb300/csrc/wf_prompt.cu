// Attention of whole prompts, packed one after another (softmax(scale q K^T) V).
#include <algorithm>
#include <climits>
#include <cmath>

#include "wf_device.cuh"
#include "wf_ops.cuh"

namespace wf {

struct PromptParams {
  const void *q, *k, *v;
  void *out;
  float *lse;
  long long q_stride, k_stride, v_stride, out_stride;
  const int32_t *q_start, *k_start;
  int n_seq, n_q, n_k, max_k, n_heads, group, causal;
  float scale;
  uint32_t *err;
};

// A warp per query row and head, a key at a time.
template <typename T, int G>
__global__ void __launch_bounds__(128) prompt_attention_kernel(const PromptParams p) {
  using X = Type16<T>;
  pdl_wait();
  pdl_launch_dependents();
  const int lane = threadIdx.x & 31;
  const long long unit = static_cast<long long>(blockIdx.x) * 4 + (threadIdx.x >> 5);
  if (unit >= static_cast<long long>(p.n_q) * p.n_heads) return;
  const int h = static_cast<int>(unit % p.n_heads), kh = h / p.group, row = static_cast<int>(unit / p.n_heads);
  int seq = -1, q0 = 0, q1 = 0;
  for (int i = 0; i < p.n_seq; ++i) {
    const int a = p.q_start[i], b = p.q_start[i + 1];
    if (row >= a && row < b) {
      seq = i, q0 = a, q1 = b;
      break;
    }
  }
  if (seq < 0) return;
  const int k0 = min(max(p.k_start[seq], 0), p.n_k), k1 = min(max(p.k_start[seq + 1], k0), p.n_k);
  const int keys = min(k1 - k0, p.max_k), limit = p.causal ? keys - (q1 - 1 - row) : keys;
  float2 q[G], o[G] = {};
#pragma unroll
  for (int g = 0; g < G; ++g) {
    const uint32_t w = *reinterpret_cast<const uint32_t *>(static_cast<const T *>(p.q) + row * p.q_stride + h * (G * 64) + g * 64 + lane * 2);
    q[g] = make_float2(X::lo(w), X::hi(w));
  }
  float m = -INFINITY, l = 0.f;
  for (int pos = 0; pos < limit; ++pos) {
    const T *k = static_cast<const T *>(p.k) + (k0 + pos) * p.k_stride + kh * (G * 64) + lane * 2;
    const T *v = static_cast<const T *>(p.v) + (k0 + pos) * p.v_stride + kh * (G * 64) + lane * 2;
    float x = 0.f;
    uint32_t w[G];
#pragma unroll
    for (int g = 0; g < G; ++g) {
      const uint32_t u = *reinterpret_cast<const uint32_t *>(k + g * 64);
      w[g] = *reinterpret_cast<const uint32_t *>(v + g * 64);
      x += q[g].x * X::lo(u) + q[g].y * X::hi(u);
    }
    x = warp_sum(x) * p.scale;
    const float next = fmaxf(m, x), keep = m == -INFINITY ? 0.f : __expf(m - next), f = next == -INFINITY ? 0.f : __expf(x - next);
    l = l * keep + f;
    m = next;
#pragma unroll
    for (int g = 0; g < G; ++g) o[g].x = o[g].x * keep + f * X::lo(w[g]), o[g].y = o[g].y * keep + f * X::hi(w[g]);
  }
  const float inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
  for (int g = 0; g < G; ++g)
    *reinterpret_cast<uint32_t *>(static_cast<T *>(p.out) + row * p.out_stride + h * (G * 64) + g * 64 + lane * 2) = X::pack(o[g].x * inv, o[g].y * inv);
  if (p.lse && lane == 0) p.lse[static_cast<long long>(row) * p.n_heads + h] = l == 0.f ? -INFINITY : m + logf(l);
}

}  // namespace wf

using namespace wf;

extern "C" {

size_t wf_prompt_attention_scratch_bytes(int32_t n_seq, int32_t n_q, int32_t max_k, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim) {
  return 0;
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
  PromptParams p = {};
  p.q = d_q, p.k = d_k, p.v = d_v, p.out = d_out, p.lse = d_lse;
  p.q_stride = q_stride, p.k_stride = k_stride, p.v_stride = v_stride, p.out_stride = out_stride;
  p.q_start = d_q_start, p.k_start = d_k_start, p.n_seq = n_seq, p.n_q = n_q, p.n_k = n_k, p.max_k = max_k;
  p.n_heads = n_heads, p.group = n_heads / n_kv_heads, p.causal = causal != 0, p.scale = scale, p.err = d_err;
  using B = __nv_bfloat16;
  const void *fn = dtype == WF_F16 ? (head_dim == 128 ? reinterpret_cast<const void *>(prompt_attention_kernel<__half, 2>) : reinterpret_cast<const void *>(prompt_attention_kernel<__half, 1>))
                                   : (head_dim == 128 ? reinterpret_cast<const void *>(prompt_attention_kernel<B, 2>) : reinterpret_cast<const void *>(prompt_attention_kernel<B, 1>));
  const int64_t units = static_cast<int64_t>(n_q) * n_heads;
  if ((units + 3) / 4 > INT32_MAX) return WF_ERR_UNSUPPORTED;
  void *args[] = {&p};
  return launch_pdl(fn, static_cast<unsigned>((units + 3) / 4), 128, 0, args, static_cast<cudaStream_t>(stream)) == cudaSuccess ? WF_OK : WF_ERR_CUDA;
}

}  // extern "C"
