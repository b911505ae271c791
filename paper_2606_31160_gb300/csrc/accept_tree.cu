// Greedy acceptance along a drafted tree (sm_103a).
//
//   star_i = argmax_v logits[b][i][v]   (lowest index among equal maxima)
//   at = 0;  at <- the lowest child c of at with token_c == star_at, while there is one
//   emit star of every row on the walk
//
// The simplest form: a CTA finds one row's maximum; the scene's last CTA (a ticket) walks.
#include "common.cuh"

SD_DEFINE_ERROR_ACCESSOR(sd_take_error_accept_tree)

namespace {

constexpr int kThreads = 256;
constexpr int kMaxRows = 256;

__device__ __forceinline__ uint32_t ordered(float x) {
  const uint32_t u = __float_as_uint(x + 0.f);
  return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}
__device__ __forceinline__ float load_one(const float* p) { return __ldcg(p); }
__device__ __forceinline__ float load_one(const __nv_bfloat16* p) { return sd_ldcg_bf16(p); }

struct AcceptArgs {
  const int32_t *tokens, *parents, *n_new;
  int32_t *n_emit, *path, *out, *argmax;
  unsigned long long* keys;
  uint32_t* ticket;
  long long stride;
  int R, V;
};

// The walk of scene b over its n rows, by one CTA. keys: the rows' maxima.
__device__ void walk(const AcceptArgs& a, int b, int n) {
  __shared__ int s_star[kMaxRows], s_parent[kMaxRows], s_token[kMaxRows];
  const long long row0 = static_cast<long long>(b) * a.R;
  bool tree_ok = true, range_ok = true;
  for (int i = threadIdx.x; i < n; i += kThreads) {
    unsigned long long* key = a.keys + row0 + i;
    s_star[i] = static_cast<int>(0xffffffffu - static_cast<uint32_t>(__ldcg(key)));
    *key = 0ull;  // re-armed for the next call
    const int p = a.parents ? __ldcg(a.parents + row0 + i) : i - 1;
    const int t = i > 0 ? __ldcg(a.tokens + row0 + i) : 0;
    s_parent[i] = p;
    s_token[i] = t;
    tree_ok &= p >= -1 && p < i;
    range_ok &= t >= 0 && t < a.V;
  }
  tree_ok = __syncthreads_and(tree_ok) != 0;
  range_ok = __syncthreads_and(range_ok) != 0;
  if (!tree_ok) {
    if (threadIdx.x == 0) sd_set_error(SD_DEVERR_TREE);
    return;
  }
  if (!range_ok && threadIdx.x == 0) sd_set_error(SD_DEVERR_TOKEN_RANGE);
  for (int i = threadIdx.x; i < n; i += kThreads)
    if (a.argmax) a.argmax[row0 + i] = s_star[i];
  if (threadIdx.x >= 32) return;
  const int lane = threadIdx.x;
  int count = 0, at = n > 0 ? 0 : -1;
  while (at >= 0) {
    if (lane == 0) {
      a.path[row0 + count] = at;
      a.out[row0 + count] = s_star[at];
    }
    ++count;
    int next = -1;
    for (int c0 = (at + 1) & ~31; c0 < n && next < 0; c0 += 32) {  // a child comes after its parent
      const int c = c0 + lane;
      const uint32_t hit = __ballot_sync(0xffffffffu, c < n && s_parent[c] == at && s_token[c] == s_star[at]);
      if (hit) next = c0 + __ffs(hit) - 1;
    }
    at = next;
  }
  for (int i = count + lane; i < a.R; i += 32) a.path[row0 + i] = a.out[row0 + i] = -1;
  if (lane == 0) a.n_emit[b] = count;
}

// Grid (rows, scenes).
template <typename T>
__global__ void __launch_bounds__(kThreads) accept_tree_kernel(const T* logits, const AcceptArgs a) {
  __shared__ unsigned long long s_best[kThreads / 32];
  __shared__ bool s_last;
  sd_pdl_enter();
  const int r = blockIdx.x, b = blockIdx.y;
  const int n = a.n_new ? __ldcg(a.n_new + b) : a.R;
  if (n < 0 || n > a.R) {
    if (r == 0 && threadIdx.x == 0) sd_set_error(SD_DEVERR_LENGTH);
    return;
  }
  if (r >= max(n, 1)) return;
  if (n > 0) {
    const T* row = logits + (static_cast<long long>(b) * a.R + r) * a.stride;
    unsigned long long best = 0;
    for (int v = threadIdx.x; v < a.V; v += kThreads) {
      const float x = load_one(row + v);
      const unsigned long long key =
          (static_cast<unsigned long long>(ordered(x)) << 32) | (0xffffffffu - static_cast<uint32_t>(v));
      if (x == x && key > best) best = key;
    }
    for (int d = 16; d; d >>= 1) best = max(best, __shfl_xor_sync(0xffffffffu, best, d));
    if ((threadIdx.x & 31) == 0) s_best[threadIdx.x >> 5] = best;
    __syncthreads();
    if (threadIdx.x == 0) {
      for (int w = 1; w < kThreads / 32; ++w) best = max(best, s_best[w]);
      if (best == 0) best = 0xffffffffull;  // nothing but NaN: index 0
      a.keys[static_cast<long long>(b) * a.R + r] = best;
    }
  }
  if (threadIdx.x == 0) {
    __threadfence();
    s_last = atomicAdd(&a.ticket[b], 1u) == static_cast<uint32_t>(max(n, 1) - 1);
    if (s_last) a.ticket[b] = 0;
    __threadfence();
  }
  __syncthreads();
  if (s_last) walk(a, b, n);
}

}  // namespace

extern "C" size_t sd_accept_tree_workspace(int B, int R, int V) {
  if (B <= 0 || R <= 0 || V <= 0) return 0;
  return static_cast<size_t>(B) * R * 8 + (static_cast<size_t>(B) * 4 + 15) / 16 * 16;
}

extern "C" sd_status sd_accept_tree(const void* logits, sd_dtype dtype, int B, int R, int V, long long row_stride,
                                    const int32_t* tokens, const int32_t* parents, const int32_t* n_new,
                                    int32_t* n_emit, int32_t* path, int32_t* out, int32_t* argmax, void* ws,
                                    size_t ws_bytes, sd_stream_t stream) {
  if (B < 0 || R <= 0 || V <= 0 || row_stride < V) return SD_ERR_INVALID_ARG;
  if (dtype != SD_BF16 && dtype != SD_F32) return SD_ERR_INVALID_ARG;
  if (R > kMaxRows || B > 65535) return SD_ERR_UNSUPPORTED;
  if (B == 0) return SD_OK;
  if (!logits || !tokens || !n_emit || !path || !out) return SD_ERR_INVALID_ARG;
  if (reinterpret_cast<uintptr_t>(logits) % (dtype == SD_BF16 ? 2 : 4)) return SD_ERR_INVALID_ARG;
  if (!ws || ws_bytes < sd_accept_tree_workspace(B, R, V) || !sd_aligned16(ws)) return SD_ERR_WORKSPACE;
  AcceptArgs a = {};
  a.tokens = tokens;
  a.parents = parents;
  a.n_new = n_new;
  a.n_emit = n_emit;
  a.path = path;
  a.out = out;
  a.argmax = argmax;
  a.keys = static_cast<unsigned long long*>(ws);
  a.ticket = reinterpret_cast<uint32_t*>(static_cast<char*>(ws) + static_cast<size_t>(B) * R * 8);
  a.stride = row_stride;
  a.R = R;
  a.V = V;
  const dim3 grid(R, B);
  const cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  const cudaError_t e =
      dtype == SD_BF16
          ? sd_launch_pdl(accept_tree_kernel<__nv_bfloat16>, grid, dim3(kThreads), 0, st, static_cast<const __nv_bfloat16*>(logits), a)
          : sd_launch_pdl(accept_tree_kernel<float>, grid, dim3(kThreads), 0, st, static_cast<const float*>(logits), a);
  if (e != cudaSuccess) {
    (void)cudaGetLastError();
    return SD_ERR_CUDA;
  }
  return SD_OK;
}
