// The attention weight that every cached key gathers from the rows of a pass (sm_103a):
// with p the softmax of q . k * scale over the keys a row sees (as in the verify
// attention),
//     out[b][g][n] = decay * in[b][g][n] + sum over rows i < committed[b] and the query
//                    heads h of KV head g of p[b][i][h][n]
// where a key appended with these rows (n >= len[b] - R) brings no weight with it.
//
// The plainest form: a CTA a (KV head, scene), first each row's maximum and sum, then
// each key's weights.
#include "common.cuh"

#include <math.h>

SD_DEFINE_ERROR_ACCESSOR(sd_take_error_weights)

namespace {

constexpr int kThreads = 256;

template <int D>
__device__ float dot(const float* q, const __nv_bfloat16* k) {
  float x = 0.f;
  for (int j = 0; j < D; j += 2) {
    const uint32_t w = __ldcg(reinterpret_cast<const unsigned int*>(k + j));
    x = fmaf(q[j], sd_bf16_lo(w), fmaf(q[j + 1], sd_bf16_hi(w), x));
  }
  return x;
}

template <int D>
__global__ void __launch_bounds__(kThreads) key_weights_kernel(const __nv_bfloat16* q, const __nv_bfloat16* k,
                                                               const int32_t* len, const int32_t* committed,
                                                               const float* in, float decay, float* out, int R, int Hq,
                                                               int Hkv, int cap, float scale_log2) {
  sd_pdl_enter();
  const int kvh = blockIdx.x, b = blockIdx.y, G = Hq / Hkv;
  const int n = __ldcg(len + b);
  const int rows = committed ? __ldcg(committed + b) : R;
  if (n < R || n > cap || rows < 0 || rows > R) {
    if (threadIdx.x == 0) sd_set_error(n < R || n > cap ? SD_DEVERR_LENGTH : SD_DEVERR_ROLLBACK);
    return;
  }
  __shared__ float qs[D];
  __shared__ float red[kThreads];
  const long long plane = static_cast<long long>(b) * Hkv + kvh;
  k += plane * cap * D;
  in = in ? in + plane * cap : nullptr;
  out += plane * cap;
  for (int t = threadIdx.x; t < n; t += kThreads) out[t] = in && t < n - R ? decay * __ldcg(in + t) : 0.f;
  for (int p = 0; p < rows * G; ++p) {
    const int i = p / G, h = kvh * G + p % G, seen = n - R + i + 1;
    __syncthreads();
    if (threadIdx.x < D)
      qs[threadIdx.x] = sd_ldcg_bf16(q + ((static_cast<long long>(b) * R + i) * Hq + h) * D + threadIdx.x) * scale_log2;
    __syncthreads();
    float m = -INFINITY;
    for (int t = threadIdx.x; t < seen; t += kThreads) m = fmaxf(m, dot<D>(qs, k + static_cast<long long>(t) * D));
    red[threadIdx.x] = m;
    __syncthreads();
    for (int w = 0; w < kThreads; ++w) m = fmaxf(m, red[w]);
    __syncthreads();
    float l = 0.f;
    for (int t = threadIdx.x; t < seen; t += kThreads) l += exp2f(dot<D>(qs, k + static_cast<long long>(t) * D) - m);
    red[threadIdx.x] = l;
    __syncthreads();
    l = 0.f;
    for (int w = 0; w < kThreads; ++w) l += red[w];
    for (int t = threadIdx.x; t < seen; t += kThreads)
      out[t] += exp2f(dot<D>(qs, k + static_cast<long long>(t) * D) - m) / l;
  }
}

}  // namespace

extern "C" sd_status sd_attention_weights(const void* q, const sd_kv_cache* cache, int R, int Hq, float scale,
                                          const int32_t* committed, const float* weights_in, float decay,
                                          float* weights, sd_stream_t stream) {
  if (!cache) return SD_ERR_INVALID_ARG;
  const int B = cache->batch, Hkv = cache->n_kv_heads, D = cache->head_dim, cap = cache->capacity;
  if (B < 0 || R <= 0 || Hq <= 0 || Hkv <= 0 || cap <= 0 || Hq % Hkv) return SD_ERR_INVALID_ARG;
  if (D != 64 && D != 128) return SD_ERR_UNSUPPORTED;
  if (B > 65535 || Hkv > 65535 || static_cast<long long>(Hq / Hkv) * R > (1 << 24)) return SD_ERR_UNSUPPORTED;
  if (!(scale >= 0.f) || !isfinite(scale) || !isfinite(decay)) return SD_ERR_INVALID_ARG;
  if (B == 0) return SD_OK;
  if (!q || !cache->k || !cache->len || !weights) return SD_ERR_INVALID_ARG;
  if (!sd_aligned16(q) || !sd_aligned16(cache->k) || !sd_aligned16(weights) || !sd_aligned16(weights_in))
    return SD_ERR_INVALID_ARG;
  const double sc = scale > 0.f ? scale : 1.0 / sqrt(static_cast<double>(D));
  const float scale_log2 = static_cast<float>(sc * 1.4426950408889634);
  if (sd_launch_pdl(D == 64 ? key_weights_kernel<64> : key_weights_kernel<128>, dim3(Hkv, B), dim3(kThreads), 0,
                    reinterpret_cast<cudaStream_t>(stream), static_cast<const __nv_bfloat16*>(q),
                    static_cast<const __nv_bfloat16*>(cache->k), static_cast<const int32_t*>(cache->len), committed,
                    weights_in, decay, weights, R, Hq, Hkv, cap, scale_log2) != cudaSuccess) {
    (void)cudaGetLastError();
    return SD_ERR_CUDA;
  }
  return SD_OK;
}
