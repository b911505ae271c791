// Greedy acceptance along a drafted tree (sm_103a).
//
//   star_i = argmax_v logits[b][i][v]   (lowest index among equal maxima)
//   at = 0;  at <- the lowest child c of at with token_c == star_at, while there is one
//   emit star of every row on the walk
//
// One kernel: a CTA scans a segment of one row and raises the row's key by atomicMax; the
// scene's last CTA (a ticket, no spin) walks the tree over the keys and re-arms the
// workspace. The order of the keys is total, so the result does not depend on the order in
// which they come. CTAs of rows that do not count end at once.
// Bound by the logits' bytes where they are many (16 ragged scenes of up to 61 rows x 151936
// fp32, 329 MB: 56 us, 0.88 of a copy's rate); one scene's 26 rows of bf16 (7.9 MB) take 8.7 us:
// the scan, the ticket, the keys, the walk, one after the other.
#include "row_scan.cuh"

#include <algorithm>

SD_DEFINE_ERROR_ACCESSOR(sd_take_error_accept_tree)

namespace {

constexpr int kMaxRows = 256;

struct AcceptArgs {
  const int32_t *tokens, *parents, *n_new;
  int32_t *n_emit, *path, *out, *argmax;
  unsigned long long* keys;
  uint32_t* ticket;
  long long stride;
  int R, V;
};

// The walk of scene b over its n rows, by one CTA; p and t: the parent and token of the
// thread's row.
static_assert(kMaxRows <= kThreads, "a row a thread");
__device__ void walk(const AcceptArgs& a, int b, int n, int p, int t) {
  __shared__ int s_star[kMaxRows], s_parent[kMaxRows], s_token[kMaxRows];
  const long long row0 = static_cast<long long>(b) * a.R;
  bool tree_ok = true, range_ok = true;
  const int i = threadIdx.x;
  if (i < n) {
    unsigned long long* key = a.keys + row0 + i;
    s_star[i] = static_cast<int>(0xffffffffu - static_cast<uint32_t>(__ldcg(key)));
    *key = 0ull;  // re-armed for the next call
    s_parent[i] = p;
    s_token[i] = t;
    tree_ok = p >= -1 && p < i;
    range_ok = t >= 0 && t < a.V;
  }
  tree_ok = __syncthreads_and(tree_ok) != 0;
  range_ok = __syncthreads_and(range_ok) != 0;
  if (!tree_ok) {
    if (threadIdx.x == 0) sd_set_error(SD_DEVERR_TREE);
    return;
  }
  if (!range_ok && threadIdx.x == 0) sd_set_error(SD_DEVERR_TOKEN_RANGE);
  if (i < n && a.argmax) a.argmax[row0 + i] = s_star[i];
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
  for (int c = count + lane; c < a.R; c += 32) a.path[row0 + c] = a.out[row0 + c] = -1;
  if (lane == 0) a.n_emit[b] = count;
}

// Grid (segments, rows, scenes).
template <typename T>
__global__ void __launch_bounds__(kThreads) accept_tree_kernel(const T* logits, int vps, const AcceptArgs a) {
  __shared__ uint32_t s_best[kThreads / 32], s_index;
  __shared__ bool s_last;
  sd_pdl_enter();
  const int r = blockIdx.y, b = blockIdx.z;
  const int n = a.n_new ? __ldcg(a.n_new + b) : a.R;
  if (n < 0 || n > a.R) {
    if (r == 0 && blockIdx.x == 0 && threadIdx.x == 0) sd_set_error(SD_DEVERR_LENGTH);
    return;
  }
  if (r >= max(n, 1)) return;
  const long long at = static_cast<long long>(b) * a.R + r;
  unsigned long long best = 0;
  if (n > 0) best = scan_segment(logits + at * a.stride, a.V, static_cast<int>(blockIdx.x), static_cast<int>(gridDim.x), vps, s_best, &s_index);
  // (the tree travels with the ticket: any CTA may come to walk it)
  const int own = threadIdx.x;
  const long long row0 = static_cast<long long>(b) * a.R;
  const int p = own < n && a.parents ? __ldcg(a.parents + row0 + own) : own - 1;
  const int t = own > 0 && own < n ? __ldcg(a.tokens + row0 + own) : 0;
  if (threadIdx.x == 0) {
    if (n > 0) atomicMax(&a.keys[at], best);
    __threadfence();
    s_last = atomicAdd(&a.ticket[b], 1u) == static_cast<uint32_t>(max(n, 1)) * gridDim.x - 1;
    if (s_last) a.ticket[b] = 0;
    __threadfence();
  }
  __syncthreads();
  if (s_last) walk(a, b, n, p, t);
}

// Vectors a segment: about six CTAs an SM over all rows and at least 16 KB (one step of every
// thread) a segment; where rows do not count the CTAs left would be uneven, so three times as many
// (16 ragged scenes: 57.4 -> 56.1 us; 26 rows that all count 8.7 -> 8.8).
int segment_vectors(int B, int R, int V, int elem_bytes, bool ragged) {
  const long long row = (static_cast<long long>(V) * elem_bytes + 15) / 16;
  const long long ctas = (ragged ? 18LL : 6LL) * sd_num_sms();
  const long long vps = std::max<long long>((row * B * R + ctas - 1) / ctas, kStep * kThreads);
  const long long segs = (row + vps - 1) / vps;
  return static_cast<int>((row + segs - 1) / segs);
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
  const int vps = segment_vectors(B, R, V, dtype == SD_BF16 ? 2 : 4, n_new != nullptr);
  const long long row = (static_cast<long long>(V) * (dtype == SD_BF16 ? 2 : 4) + 15) / 16;
  const dim3 grid(static_cast<unsigned>((row + vps - 1) / vps), R, B);
  const cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  const cudaError_t e =
      dtype == SD_BF16
          ? sd_launch_pdl(accept_tree_kernel<__nv_bfloat16>, grid, dim3(kThreads), 0, st, static_cast<const __nv_bfloat16*>(logits), vps, a)
          : sd_launch_pdl(accept_tree_kernel<float>, grid, dim3(kThreads), 0, st, static_cast<const float*>(logits), vps, a);
  if (e != cudaSuccess) {
    (void)cudaGetLastError();
    return SD_ERR_CUDA;
  }
  return SD_OK;
}
