// Verify attention over the 8-bit KV cache (sm_103a): the rows, masks and results of
// the bf16 verify attention, with key n = k_code[n] * k_scale[n / block] and value
// n = v_code[n] * v_scale[n / block].
//
// The plainest form: a warp a query row, its lanes over the head dim, one pass over the
// row's keys with the running maximum and sum of its softmax.
#include "common.cuh"

#include <math.h>

SD_DEFINE_ERROR_ACCESSOR(sd_take_error_attention_kv8)

namespace {

__device__ __forceinline__ float2 code2(uint32_t w) {
  uint32_t h;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"(static_cast<uint16_t>(w)));
  float lo, hi;
  asm("{\n\t.reg .f16 a, b;\n\tmov.b32 {a, b}, %2;\n\tcvt.f32.f16 %0, a;\n\tcvt.f32.f16 %1, b;\n\t}"
      : "=f"(lo), "=f"(hi)
      : "r"(h));
  return make_float2(lo, hi);
}

// Grid (warps of packed rows, Hkv, B).
template <int D>
__global__ void __launch_bounds__(128) kv8_attention_kernel(const __nv_bfloat16* q, const uint8_t* kc, const uint8_t* vc,
                                                            const float* ks, const float* vs, const int32_t* len,
                                                            __nv_bfloat16* out, int R, int Hq, int Hkv, int cap,
                                                            int block, int nblk, float scale_log2, bool block_mask) {
  sd_pdl_enter();
  constexpr int kPer = D / 32;
  const int G = Hq / Hkv, lane = threadIdx.x & 31;
  const int p = blockIdx.x * 4 + (threadIdx.x >> 5), kvh = blockIdx.y, b = blockIdx.z;
  const int n = __ldcg(len + b);
  if (n < R || n > cap) {
    if (threadIdx.x == 0) sd_set_error(SD_DEVERR_LENGTH);
    return;
  }
  if (p >= G * R) return;
  const int i = p / G, h = kvh * G + (p - i * G);
  const long long row = ((static_cast<long long>(b) * R + i) * Hq + h) * D + lane * kPer;
  float qv[kPer], o[kPer];
  for (int j = 0; j < kPer; ++j) {
    qv[j] = sd_ldcg_bf16(q + row + j);
    o[j] = 0.f;
  }
  const long long plane = static_cast<long long>(b) * Hkv + kvh;
  kc += plane * cap * D + lane * kPer;
  vc += plane * cap * D + lane * kPer;
  ks += plane * nblk;
  vs += plane * nblk;
  const int seen = block_mask ? n : n - R + i + 1;
  float m = -INFINITY, l = 0.f;
  for (int t = 0; t < seen; ++t) {
    float x = 0.f;
    float v[kPer];
    for (int j = 0; j < kPer; j += 2) {
      const float2 kk = code2(__ldcg(reinterpret_cast<const unsigned short*>(kc + static_cast<long long>(t) * D + j)));
      const float2 vv = code2(__ldcg(reinterpret_cast<const unsigned short*>(vc + static_cast<long long>(t) * D + j)));
      x = fmaf(qv[j], kk.x, fmaf(qv[j + 1], kk.y, x));
      v[j] = vv.x;
      v[j + 1] = vv.y;
    }
    for (int s = 16; s > 0; s >>= 1) x += __shfl_xor_sync(0xffffffffu, x, s);
    x *= __ldcg(ks + t / block) * scale_log2;
    const float mn = fmaxf(m, x), f = exp2f(m - mn), e = exp2f(x - mn);
    const float w = e * __ldcg(vs + t / block);
    l = fmaf(l, f, e);
    for (int j = 0; j < kPer; ++j) o[j] = fmaf(o[j], f, w * v[j]);
    m = mn;
  }
  for (int j = 0; j < kPer; ++j) out[row + j] = __float2bfloat16_rn(o[j] / l);
}

}  // namespace

extern "C" sd_status sd_kv8_attention(const void* q, const sd_kv8_cache* cache, void* out, int R, int Hq, float scale,
                                      int flags, sd_stream_t stream) {
  const sd_status s = sd_internal_kv8_check(cache);
  if (s != SD_OK) return s;
  const int B = cache->batch, Hkv = cache->n_kv_heads, D = cache->head_dim;
  if (R <= 0 || Hq <= 0 || Hq % Hkv || (flags & ~SD_ATTN_BLOCK_MASK)) return SD_ERR_INVALID_ARG;
  if (!(scale >= 0.f) || !isfinite(scale)) return SD_ERR_INVALID_ARG;
  if (static_cast<long long>(Hq / Hkv) * R > 128) return SD_ERR_UNSUPPORTED;
  if (B == 0) return SD_OK;
  if (!q || !out || !sd_aligned16(q) || !sd_aligned16(out)) return SD_ERR_INVALID_ARG;
  const double sc = scale > 0.f ? scale : 1.0 / sqrt(static_cast<double>(D));
  const float scale_log2 = static_cast<float>(sc * 1.4426950408889634);
  const int M = Hq / Hkv * R;
  if (sd_launch_pdl(D == 64 ? kv8_attention_kernel<64> : kv8_attention_kernel<128>, dim3((M + 3) / 4, Hkv, B), dim3(128), 0,
                    reinterpret_cast<cudaStream_t>(stream), static_cast<const __nv_bfloat16*>(q),
                    static_cast<const uint8_t*>(cache->k), static_cast<const uint8_t*>(cache->v),
                    static_cast<const float*>(cache->k_scale), static_cast<const float*>(cache->v_scale),
                    static_cast<const int32_t*>(cache->len), static_cast<__nv_bfloat16*>(out), R, Hq, Hkv,
                    cache->capacity, cache->block, (cache->capacity + cache->block - 1) / cache->block, scale_log2,
                    (flags & SD_ATTN_BLOCK_MASK) != 0) != cudaSuccess) {
    (void)cudaGetLastError();
    return SD_ERR_CUDA;
  }
  return SD_OK;
}
