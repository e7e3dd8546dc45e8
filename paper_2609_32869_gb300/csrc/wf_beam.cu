// Beam search's selection over beams and vocabulary.
//
// Within a row the order of the scores, score + ((logit - max) - log(sum)), is
// the order of the logits,
// so the vocabulary is read once: each CTA takes a chunk of a row, keeps the
// chunk's running maximum and sum of exponentials and its 2 beams largest
// logits.  A second kernel joins the chunks of a request's rows, turns the
// survivors into scores and ranks them.
#include <algorithm>

#include "wf_device.cuh"
#include "wf_kv4.cuh"

namespace wf {

struct SelectParams {
  const void *logits;
  long long ld;
  const float *scores;
  const uint8_t *suppress;
  int n_req, W, V, eos, chunks;
  int32_t *token, *parent;
  float *score;
  int32_t *fin_parent;
  float *fin_score;
  // scratch: per (row, chunk) the maximum and the sum, and 2W keys
  unsigned long long *keys;  // [rows][chunks][2W]
  double *sum;               // [rows][chunks]
  float *max;                // [rows][chunks]
};
constexpr int kSelThreads = 256;
constexpr int kSelPer = 16;                         // logits of a thread
constexpr int kSelChunk = kSelThreads * kSelPer;    // of a CTA

// (value descending, index ascending) as one descending unsigned key; 0 is
// below every key of a value above -inf.
__device__ __forceinline__ unsigned long long order_key(float v, uint32_t idx) {
  const uint32_t b = __float_as_uint(v + 0.f);  // -0 as 0
  const uint32_t o = (b & 0x80000000u) ? ~b : (b | 0x80000000u);
  return static_cast<unsigned long long>(o) << 32 | (0xffffffffu - idx);
}
__device__ __forceinline__ float key_value(unsigned long long k) {
  const uint32_t o = static_cast<uint32_t>(k >> 32);
  return __uint_as_float((o & 0x80000000u) ? (o & 0x7fffffffu) : ~o);
}
__device__ __forceinline__ uint32_t key_index(unsigned long long k) { return 0xffffffffu - static_cast<uint32_t>(k); }
__device__ __forceinline__ unsigned long long warp_max(unsigned long long k) {
#pragma unroll
  for (int off = 16; off; off >>= 1) {
    const unsigned long long v = __shfl_xor_sync(0xffffffffu, k, off);
    k = v > k ? v : k;
  }
  return k;
}
__device__ __forceinline__ float as_float(float v) { return v; }
__device__ __forceinline__ float as_float(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float as_float(__half v) { return __half2float(v); }

template <typename T>
__global__ void __launch_bounds__(kSelThreads) beam_chunk_kernel(const SelectParams p) {
  pdl_wait();
  pdl_launch_dependents();
  const int chunk = blockIdx.x, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const long long row = blockIdx.y + static_cast<long long>(blockIdx.z) * 65535;
  if (row >= static_cast<long long>(p.n_req) * p.W) return;
  const T *src = static_cast<const T *>(p.logits) + row * p.ld;
  __shared__ float sm_m[kSelThreads / 32];
  __shared__ double sm_s[kSelThreads / 32];
  __shared__ unsigned long long sm_k[2][kSelThreads / 32];
  float x[kSelPer];
  float m = -INFINITY;
#pragma unroll
  for (int i = 0; i < kSelPer; ++i) {
    const int id = chunk * kSelChunk + i * kSelThreads + tid;
    x[i] = id < p.V ? as_float(src[id]) : -INFINITY;
    if (x[i] != x[i] || (id < p.V && p.suppress && p.suppress[id])) x[i] = -INFINITY;
    m = fmaxf(m, x[i]);
  }
#pragma unroll
  for (int off = 16; off; off >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, off));
  if (lane == 0) sm_m[warp] = m;
  __syncthreads();
  for (int w = 0; w < kSelThreads / 32; ++w) m = fmaxf(m, sm_m[w]);
  float part = 0.f;
#pragma unroll
  for (int i = 0; i < kSelPer; ++i) part += x[i] == -INFINITY ? 0.f : expf(x[i] - m);
  double s = part;
#pragma unroll
  for (int off = 16; off; off >>= 1) s += __shfl_xor_sync(0xffffffffu, s, off);
  if (lane == 0) sm_s[warp] = s;
  // the 2W largest, one at a time
  unsigned long long best = 0;
#pragma unroll
  for (int i = 0; i < kSelPer; ++i) {
    const unsigned long long k = x[i] == -INFINITY ? 0 : order_key(x[i], chunk * kSelChunk + i * kSelThreads + tid);
    best = k > best ? k : best;
  }
  unsigned long long *out = p.keys + (row * p.chunks + chunk) * (2 * p.W);
  for (int k = 0; k < 2 * p.W; ++k) {
    const unsigned long long mine = warp_max(best);
    if (lane == 0) sm_k[k & 1][warp] = mine;
    __syncthreads();
    unsigned long long top = 0;
    for (int w = 0; w < kSelThreads / 32; ++w) top = sm_k[k & 1][w] > top ? sm_k[k & 1][w] : top;
    if (tid == 0) out[k] = top;
    if (top == best && top) {
      best = 0;
#pragma unroll
      for (int i = 0; i < kSelPer; ++i) {
        const unsigned long long q = x[i] == -INFINITY ? 0 : order_key(x[i], chunk * kSelChunk + i * kSelThreads + tid);
        if (q < top && q > best) best = q;
      }
    }
  }
  if (tid == 0) {
    double total = 0;
    for (int w = 0; w < kSelThreads / 32; ++w) total += sm_s[w];
    p.sum[row * p.chunks + chunk] = total;
    p.max[row * p.chunks + chunk] = m;
  }
}

// One CTA per request, one warp per beam.
__global__ void __launch_bounds__(WF_MAX_BEAMS * 32) beam_join_kernel(const SelectParams p) {
  pdl_wait();
  pdl_launch_dependents();
  const int W = p.W, K = 2 * W, req = blockIdx.x, lane = threadIdx.x & 31, beam = threadIdx.x >> 5;
  __shared__ unsigned long long cand[WF_MAX_BEAMS][2 * WF_MAX_BEAMS];  // (score, place) by beam, best first
  __shared__ int32_t tok[WF_MAX_BEAMS][2 * WF_MAX_BEAMS];
  const long long row = static_cast<long long>(req) * W + beam;
  const float *cm = p.max + row * p.chunks;
  const double *cs = p.sum + row * p.chunks;
  float m = -INFINITY;
  for (int c = lane; c < p.chunks; c += 32) m = fmaxf(m, cm[c]);
#pragma unroll
  for (int off = 16; off; off >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, off));
  double s = 0;
  for (int c = lane; c < p.chunks; c += 32)
    if (cm[c] != -INFINITY) s += cs[c] * exp(static_cast<double>(cm[c]) - static_cast<double>(m));
#pragma unroll
  for (int off = 16; off; off >>= 1) s += __shfl_xor_sync(0xffffffffu, s, off);
  const float log_sum = static_cast<float>(log(s));
  const float base = p.scores[row];
  // the row's best: each lane walks the sorted lists of its chunks
  const unsigned long long *keys = p.keys + row * p.chunks * K;
  unsigned long long floor_key = ~0ull;
  for (int k = 0; k < K; ++k) {
    unsigned long long best = 0;
    for (int c = lane; c < p.chunks; c += 32)
      for (int i = 0; i < K; ++i) {
        const unsigned long long v = keys[c * K + i];
        if (v < floor_key) {
          best = v > best ? v : best;
          break;
        }
      }
    best = warp_max(best);
    if (lane == 0) {
      float total = best ? base + ((key_value(best) - m) - log_sum) : -INFINITY;
      const bool live = total > -INFINITY;  // not NaN either
      cand[beam][k] = live ? order_key(total, beam * K + k) : 0;
      tok[beam][k] = live ? static_cast<int32_t>(key_index(best)) : -1;
    }
    floor_key = best;
  }
  __syncthreads();
  if (beam != 0) return;
  // the request's best: lane w walks beam w's list
  int at = 0, n_go = 0, n_fin = 0;
  const size_t o = static_cast<size_t>(req) * W;
  for (int k = 0; k < K; ++k) {
    const unsigned long long mine = lane < W && at < K ? cand[lane][at] : 0;
    const unsigned long long best = warp_max(mine);
    if (!best) break;
    if (mine == best) ++at;
    const uint32_t place = key_index(best);
    const int b = place / K, t = tok[b][place % K];
    const float v = key_value(best);
    if (t == p.eos) {
      if (k < W) {
        if (lane == 0) p.fin_parent[o + n_fin] = b, p.fin_score[o + n_fin] = v;
        ++n_fin;
      }
    } else if (n_go < W) {
      if (lane == 0) p.token[o + n_go] = t, p.parent[o + n_go] = b, p.score[o + n_go] = v;
      ++n_go;
    }
  }
  if (lane < W) {
    if (lane >= n_go) p.token[o + lane] = -1, p.parent[o + lane] = lane, p.score[o + lane] = -INFINITY;
    if (lane >= n_fin) p.fin_parent[o + lane] = -1, p.fin_score[o + lane] = -INFINITY;
  }
}

}  // namespace wf

using namespace wf;

static int select_chunks(int V) { return (V + kSelChunk - 1) / kSelChunk; }

extern "C" {

size_t wf_beam_select_scratch_bytes(int32_t n_req, int32_t beams, int32_t vocab) {
  if (n_req <= 0 || beams <= 0 || beams > WF_MAX_BEAMS || vocab < 2 * beams) return 0;
  return static_cast<size_t>(n_req) * beams * select_chunks(vocab) * (2 * beams * 8 + 16);
}

wf_status wf_beam_select(const void *d_logits, int32_t dtype, int64_t ld, const float *d_scores, const uint8_t *d_suppress,
                         int32_t n_req, int32_t beams, int32_t vocab, int32_t eos, int32_t *d_token, int32_t *d_parent,
                         float *d_score, int32_t *d_fin_parent, float *d_fin_score, void *d_scratch, size_t scratch_bytes,
                         void *stream) {
  if (!d_logits || !d_scores || !d_token || !d_parent || !d_score || !d_fin_parent || !d_fin_score || !d_scratch || n_req <= 0 ||
      beams <= 0 || vocab <= 0 || ld < vocab || (reinterpret_cast<uintptr_t>(d_scratch) & 7))
    return WF_ERR_INVALID;
  if (dtype < WF_BF16 || dtype > WF_F32 || beams > WF_MAX_BEAMS || vocab < 2 * beams) return WF_ERR_UNSUPPORTED;
  const long long rows = static_cast<long long>(n_req) * beams;
  if (rows > INT32_MAX) return WF_ERR_INVALID;
  if (scratch_bytes < wf_beam_select_scratch_bytes(n_req, beams, vocab)) return WF_ERR_CAPACITY;
  SelectParams p = {};
  p.logits = d_logits, p.ld = ld, p.scores = d_scores, p.suppress = d_suppress;
  p.n_req = n_req, p.W = beams, p.V = vocab, p.eos = eos < 0 ? -2 : eos, p.chunks = select_chunks(vocab);
  p.token = d_token, p.parent = d_parent, p.score = d_score, p.fin_parent = d_fin_parent, p.fin_score = d_fin_score;
  p.keys = static_cast<unsigned long long *>(d_scratch);
  p.sum = reinterpret_cast<double *>(p.keys + rows * p.chunks * 2 * beams);
  p.max = reinterpret_cast<float *>(p.sum + rows * p.chunks);
  const void *fn = dtype == WF_F32 ? reinterpret_cast<const void *>(beam_chunk_kernel<float>)
                   : dtype == WF_F16 ? reinterpret_cast<const void *>(beam_chunk_kernel<__half>)
                                     : reinterpret_cast<const void *>(beam_chunk_kernel<__nv_bfloat16>);
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  void *args[] = {&p};
  const dim3 grid(p.chunks, static_cast<unsigned>(std::min<long long>(rows, 65535)), static_cast<unsigned>((rows + 65534) / 65535));
  if (launch_pdl(fn, grid, kSelThreads, 0, args, s) != cudaSuccess ||
      launch_pdl(reinterpret_cast<const void *>(beam_join_kernel), n_req, beams * 32, 0, args, s) != cudaSuccess)
    return WF_ERR_CUDA;
  return WF_OK;
}

}  // extern "C"
