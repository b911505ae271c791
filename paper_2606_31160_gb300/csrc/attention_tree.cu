// Attention of a drafted tree's rows over a paged cache (sm_103a): the simplest form. A
// warp takes one row of one query head and all the keys that it sees, one after the
// other, with a running maximum and sum.
#include "common.cuh"

#include <math.h>

SD_DEFINE_ERROR_ACCESSOR(sd_take_error_attention_tree)

namespace {

constexpr int kMaxRows = 256;

struct TreeArgs {
  const __nv_bfloat16 *q, *k, *v;
  __nv_bfloat16* out;
  const int32_t *table, *len, *parents, *n_new;
  long long q_stride;
  int R, Hq, Hkv, G, n_pages, shift, max_pages;
  float scale;
};

// Grid (rows x heads / 4, scenes), a warp each.
template <int D>
__global__ void __launch_bounds__(128) tree_attention_kernel(const TreeArgs a) {
  constexpr int kPer = D / 32;
  sd_pdl_enter();
  const int b = blockIdx.y, lane = threadIdx.x & 31;
  const int n = __ldcg(a.len + b), m = a.n_new ? __ldcg(a.n_new + b) : a.R;
  if (m < 0 || m > a.R || n < m || n > static_cast<long long>(a.max_pages) << a.shift) {
    if (blockIdx.x == 0 && threadIdx.x == 0) sd_set_error(SD_DEVERR_LENGTH);
    return;
  }
  __shared__ int s_parent[kMaxRows];
  bool ok = true;
  for (int i = threadIdx.x; i < m; i += blockDim.x) {
    const int p = a.parents ? __ldcg(a.parents + static_cast<long long>(b) * a.R + i) : i - 1;
    s_parent[i] = p;
    ok &= p >= -1 && p < i;
  }
  if (!__syncthreads_and(ok)) {
    if (blockIdx.x == 0 && threadIdx.x == 0) sd_set_error(SD_DEVERR_TREE);
    return;
  }
  const int32_t* table = a.table + static_cast<long long>(b) * a.max_pages;
  bool paged = true;
  for (int i = threadIdx.x; i < (n + (1 << a.shift) - 1) >> a.shift; i += blockDim.x) {
    const int id = __ldcg(table + i);
    paged &= id >= 0 && id < a.n_pages;
  }
  paged = __syncthreads_and(paged) != 0;
  if (!paged && blockIdx.x == 0 && threadIdx.x == 0) sd_set_error(SD_DEVERR_PAGE);
  const int item = blockIdx.x * 4 + (threadIdx.x >> 5), i = item / a.Hq, h = item % a.Hq;
  if (i >= m) return;
  const int g = h / a.G, prefix = n - m;
  const long long row = static_cast<long long>(b) * a.R + i;
  float q[kPer], o[kPer], top = -INFINITY, sum = 0.f;
#pragma unroll
  for (int j = 0; j < kPer; ++j) {
    q[j] = sd_ldcg_bf16(a.q + row * a.q_stride + h * D + lane + 32 * j) * a.scale;
    o[j] = 0.f;
  }
  auto key = [&](int at) {
    const long long x =
        (((static_cast<long long>(__ldcg(table + (at >> a.shift))) * a.Hkv + g) << a.shift) + (at & ((1 << a.shift) - 1))) * D + lane;
    float z = 0.f;
#pragma unroll
    for (int j = 0; j < kPer; ++j) z = fmaf(q[j], sd_ldcg_bf16(a.k + x + 32 * j), z);
#pragma unroll
    for (int d = 16; d; d >>= 1) z += __shfl_xor_sync(0xffffffffu, z, d);
    const float now = fmaxf(top, z), ref = now == -INFINITY ? 0.f : now;
    const float f = expf(top - ref), w = expf(z - ref);
    top = now;
    sum = sum * f + w;
#pragma unroll
    for (int j = 0; j < kPer; ++j) o[j] = o[j] * f + w * sd_ldcg_bf16(a.v + x + 32 * j);
  };
  if (paged) {
    for (int at = 0; at < prefix; ++at) key(at);
    for (int j = i; j >= 0; j = s_parent[j]) key(prefix + j);
  }
#pragma unroll
  for (int j = 0; j < kPer; ++j)
    a.out[(row * a.Hq + h) * D + lane + 32 * j] = __float2bfloat16(paged ? o[j] / sum : NAN);
}

}  // namespace

extern "C" size_t sd_tree_attention_workspace(int, int, int, int, int, int) { return 0; }

extern "C" sd_status sd_tree_attention(const void* q, long long q_stride, const sd_paged_cache* cache,
                                       const int32_t* parents, const int32_t* n_new, void* out, int R, int Hq,
                                       float scale, void* workspace, size_t ws_bytes, sd_stream_t stream) {
  const sd_status s = sd_internal_paged_check(cache);
  if (s != SD_OK) return s;
  const int B = cache->batch, Hkv = cache->n_kv_heads, D = cache->head_dim;
  if (R <= 0 || Hq <= 0 || Hq % Hkv) return SD_ERR_INVALID_ARG;
  if (!(scale >= 0.f) || !isfinite(scale)) return SD_ERR_INVALID_ARG;
  if (q_stride < static_cast<long long>(Hq) * D || q_stride % 8) return SD_ERR_INVALID_ARG;
  if (R > kMaxRows) return SD_ERR_UNSUPPORTED;
  if (B == 0) return SD_OK;
  if (!q || !out || !sd_aligned16(q) || !sd_aligned16(out)) return SD_ERR_INVALID_ARG;
  if (workspace && !sd_aligned16(workspace)) return SD_ERR_INVALID_ARG;
  TreeArgs a = {};
  a.q = static_cast<const __nv_bfloat16*>(q);
  a.k = static_cast<const __nv_bfloat16*>(cache->k);
  a.v = static_cast<const __nv_bfloat16*>(cache->v);
  a.out = static_cast<__nv_bfloat16*>(out);
  a.table = cache->table;
  a.len = cache->len;
  a.parents = parents;
  a.n_new = n_new;
  a.q_stride = q_stride;
  a.R = R;
  a.Hq = Hq;
  a.Hkv = Hkv;
  a.G = Hq / Hkv;
  a.n_pages = cache->n_pages;
  a.shift = cache->page == 16 ? 4 : cache->page == 32 ? 5 : cache->page == 64 ? 6 : 7;
  a.max_pages = cache->max_pages;
  a.scale = scale > 0.f ? scale : static_cast<float>(1.0 / sqrt(static_cast<double>(D)));
  if (sd_launch_pdl(D == 64 ? tree_attention_kernel<64> : tree_attention_kernel<128>, dim3((R * Hq + 3) / 4, B), dim3(128), 0,
                    reinterpret_cast<cudaStream_t>(stream), a) != cudaSuccess) {
    (void)cudaGetLastError();
    return SD_ERR_CUDA;
  }
  return SD_OK;
}
