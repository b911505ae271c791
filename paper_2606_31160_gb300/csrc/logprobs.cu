// Log probabilities of given tokens with the entropy and the top alternatives of their
// rows (sm_103a). With x = (z - max z) / T over a row's vocabulary, S = sum e^x and
// W = sum x e^x:
//     log p(t) = x_t - ln S,    entropy = ln S - W / S,
//     alternatives: the top_n largest logits, equal ones by the lowest index.
//
// The plainest form: a CTA a row; the alternatives one by one, each the largest below
// the one before it.
#include "common.cuh"

#include <math.h>

SD_DEFINE_ERROR_ACCESSOR(sd_take_error_logprobs)

namespace {

constexpr int kThreads = 256;

// (value, lowest index first) as one integer that orders descending preference upward.
__device__ __forceinline__ uint64_t key_of(float z, int i) {
  const uint32_t u = __float_as_uint(z + 0.f);
  const uint32_t o = u & 0x80000000u ? ~u : u | 0x80000000u;
  return (static_cast<uint64_t>(o) << 32) | static_cast<uint32_t>(~i);
}

template <bool kBf16>
__device__ __forceinline__ float load(const void* z, long long i) {
  return kBf16 ? sd_ldcg_bf16(static_cast<const __nv_bfloat16*>(z) + i) : __ldcg(static_cast<const float*>(z) + i);
}

template <bool kBf16>
__global__ void __launch_bounds__(kThreads) logprobs_kernel(const void* z, long long stride, int V, const int32_t* tokens,
                                                            float inv_t, int top_n, float* logprob, float* entropy,
                                                            int32_t* top_ids, float* top_logprobs) {
  sd_pdl_enter();
  __shared__ double reds[kThreads], redw[kThreads];
  __shared__ uint64_t redk[kThreads];
  const long long row = blockIdx.x, base = row * stride;
  const int t = threadIdx.x;
  auto best_below = [&](uint64_t limit) {
    uint64_t k = 0;
    for (int i = t; i < V; i += kThreads) {
      const uint64_t x = key_of(load<kBf16>(z, base + i), i);
      if (x < limit && x > k) k = x;
    }
    __syncthreads();
    redk[t] = k;
    __syncthreads();
    for (int w = 0; w < kThreads; ++w) k = max(k, redk[w]);
    return k;
  };
  uint64_t k = best_below(~0ull);
  const float m = load<kBf16>(z, base + static_cast<int>(~static_cast<uint32_t>(k)));
  double S = 0, W = 0;
  for (int i = t; i < V; i += kThreads) {
    const float x = (load<kBf16>(z, base + i) - m) * inv_t, e = expf(x);
    S += e;
    W += e > 0.f ? e * x : 0.f;
  }
  reds[t] = S;
  redw[t] = W;
  __syncthreads();
  S = W = 0;
  for (int w = 0; w < kThreads; ++w) S += reds[w], W += redw[w];
  const double ln = m == -INFINITY ? NAN : log(S);
  if (t == 0) {
    if (entropy) entropy[row] = static_cast<float>(ln - W / S);
    const int tok = __ldcg(tokens + row);
    float lp = 0.f;
    if (tok >= 0 && tok < V) lp = static_cast<float>((load<kBf16>(z, base + tok) - m) * inv_t - ln);
    else if (tok != -1) sd_set_error(SD_DEVERR_TOKEN_RANGE), lp = NAN;
    logprob[row] = lp;
  }
  for (int j = 0; j < top_n; ++j) {
    if (j > 0) k = best_below(k);
    if (t == 0) {
      const int i = static_cast<int>(~static_cast<uint32_t>(k));
      top_ids[row * top_n + j] = i;
      top_logprobs[row * top_n + j] = static_cast<float>((load<kBf16>(z, base + i) - m) * inv_t - ln);
    }
  }
}

}  // namespace

extern "C" sd_status sd_token_logprobs(const void* logits, sd_dtype dtype, int rows, int V, long long row_stride,
                                       const int32_t* tokens, float temperature, int top_n, float* logprob,
                                       float* entropy, int32_t* top_ids, float* top_logprobs, sd_stream_t stream) {
  if (rows < 0 || V <= 0 || row_stride < V) return SD_ERR_INVALID_ARG;
  if (dtype != SD_BF16 && dtype != SD_F32) return SD_ERR_INVALID_ARG;
  if (!(temperature > 0.f) || !isfinite(temperature) || !isfinite(1.f / temperature)) return SD_ERR_INVALID_ARG;
  if (top_n < 0 || top_n > V) return SD_ERR_INVALID_ARG;
  if (top_n > 32) return SD_ERR_UNSUPPORTED;
  if (rows == 0) return SD_OK;
  if (!logits || !tokens || !logprob || (top_n > 0 && (!top_ids || !top_logprobs))) return SD_ERR_INVALID_ARG;
  if (!sd_aligned16(logits)) return SD_ERR_INVALID_ARG;
  if (sd_launch_pdl(dtype == SD_BF16 ? logprobs_kernel<true> : logprobs_kernel<false>, dim3(rows), dim3(kThreads), 0,
                    reinterpret_cast<cudaStream_t>(stream), logits, row_stride, V, tokens, 1.f / temperature, top_n,
                    logprob, entropy, top_ids, top_logprobs) != cudaSuccess) {
    (void)cudaGetLastError();
    return SD_ERR_CUDA;
  }
  return SD_OK;
}
