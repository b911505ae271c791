// Eviction from a KV cache by accumulated attention weight (sm_103a): of a scene's n
// keys a KV head keeps min(n, keep): the first `sinks`, the last `recent`, and of those
// between the ones with the largest weights (among equal weights the lowest index),
// moved in their order to another cache.
//
// The plainest form: a CTA a (KV head, scene). The weight of the last key kept is found
// bit by bit on the weights' order-preserving integers, by counting; then a prefix sum
// over the keys gives each kept one its place.
#include "common.cuh"

SD_DEFINE_ERROR_ACCESSOR(sd_take_error_evict)

namespace {

constexpr int kThreads = 1024;

// An integer that orders as the weight does (-0 as +0; NaN below every number).
__device__ __forceinline__ uint32_t order_of(float w) {
  const uint32_t u = __float_as_uint(w + 0.f);
  if ((u & 0x7fffffffu) > 0x7f800000u) return 0u;
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

__device__ int block_sum(int x, int* red) {
  x = __reduce_add_sync(0xffffffffu, x);
  __syncthreads();
  if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = x;
  __syncthreads();
  return __reduce_add_sync(0xffffffffu, red[threadIdx.x & 31]);
}

__global__ void __launch_bounds__(kThreads) evict_kernel(const sd_kv_cache src, const float* weights, const sd_kv_cache dst,
                                                         int keep, int sinks, int recent, float* weights_out, int32_t* kept) {
  sd_pdl_enter();
  __shared__ int red[32];
  __shared__ int warp_base[33];
  const int h = blockIdx.x, b = blockIdx.y, Hkv = src.n_kv_heads;
  const int n = __ldcg(src.len + b);
  if (n < 0 || n > src.capacity) {
    if (threadIdx.x == 0) sd_set_error(SD_DEVERR_LENGTH);
    return;
  }
  const long long plane = static_cast<long long>(b) * Hkv + h;
  weights += plane * src.capacity;
  const int lo = min(sinks, n), hi = max(lo, n - recent);  // the keys that compete
  const int want = n <= keep ? hi - lo : keep - lo - (n - hi);
  // T: the largest integer that at least `want` of them reach
  uint32_t T = 0;
  if (want < hi - lo)
    for (int bit = 31; bit >= 0; --bit) {
      const uint32_t t = T | (1u << bit);
      int c = 0;
      for (int i = lo + threadIdx.x; i < hi; i += kThreads) c += order_of(__ldcg(weights + i)) >= t;
      if (block_sum(c, red) >= want) T = t;
    }
  int above = 0;
  for (int i = lo + threadIdx.x; i < hi; i += kThreads) above += order_of(__ldcg(weights + i)) > T;
  int ties = want - block_sum(above, red);  // of those equal to T the first `ties`
  const int vec = src.head_dim / 8;
  const uint4* ks = static_cast<const uint4*>(src.k) + plane * src.capacity * vec;
  const uint4* vs = static_cast<const uint4*>(src.v) + plane * src.capacity * vec;
  uint4* kd = static_cast<uint4*>(dst.k) + plane * dst.capacity * vec;
  uint4* vd = static_cast<uint4*>(dst.v) + plane * dst.capacity * vec;
  auto scan = [&](bool flag, int& total) {  // the number of flags before this thread's
    const uint32_t ballot = __ballot_sync(0xffffffffu, flag);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = __popc(ballot);
    __syncthreads();
    if (threadIdx.x == 0) {
      int s = 0;
      for (int w = 0; w < 32; ++w) {
        warp_base[w] = s;
        s += red[w];
      }
      warp_base[32] = s;
    }
    __syncthreads();
    total = warp_base[32];
    return warp_base[threadIdx.x >> 5] + __popc(ballot & ((1u << (threadIdx.x & 31)) - 1));
  };
  int place = 0;
  for (int i0 = 0; i0 < n; i0 += kThreads) {
    const int i = i0 + threadIdx.x;
    const bool in = i < n, fixed = in && (i < lo || i >= hi);
    const uint32_t o = in && !fixed ? order_of(__ldcg(weights + i)) : 0u;
    const bool all = want == hi - lo;
    const bool tie = in && !fixed && o == T;
    int n_ties, n_kept;
    const int t = scan(tie, n_ties);
    const bool k = in && (fixed || all || o > T || (tie && t < ties));
    const int at = place + scan(k, n_kept);
    if (k) {
      for (int c = 0; c < vec; ++c) {
        kd[static_cast<long long>(at) * vec + c] = __ldcg(ks + static_cast<long long>(i) * vec + c);
        vd[static_cast<long long>(at) * vec + c] = __ldcg(vs + static_cast<long long>(i) * vec + c);
      }
      if (weights_out) weights_out[plane * dst.capacity + at] = __ldcg(weights + i);
      if (kept) kept[plane * keep + at] = i;
    }
    ties -= min(ties, n_ties);
    place += n_kept;
  }
  if (kept)
    for (int j = place + threadIdx.x; j < keep; j += kThreads) kept[plane * keep + j] = -1;
  if (h == 0 && threadIdx.x == 0) dst.len[b] = place;
}

// Whether [a, a + na) and [b, b + nb) share a byte.
bool overlap(const void* a, size_t na, const void* b, size_t nb) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return x < y + nb && y < x + na;
}

}  // namespace

extern "C" sd_status sd_kv_evict(const sd_kv_cache* src, const float* weights, int keep, int sinks, int recent,
                                 const sd_kv_cache* dst, float* weights_out, int32_t* kept, sd_stream_t stream) {
  if (!src || !dst) return SD_ERR_INVALID_ARG;
  const int B = src->batch, Hkv = src->n_kv_heads, D = src->head_dim;
  if (B < 0 || Hkv <= 0 || src->capacity <= 0 || dst->capacity <= 0) return SD_ERR_INVALID_ARG;
  if (dst->batch != B || dst->n_kv_heads != Hkv || dst->head_dim != D) return SD_ERR_INVALID_ARG;
  if (D != 64 && D != 128) return SD_ERR_UNSUPPORTED;
  if (B > 65535) return SD_ERR_UNSUPPORTED;
  if (keep <= 0 || keep > dst->capacity || sinks < 0 || recent < 0 || static_cast<long long>(sinks) + recent > keep)
    return SD_ERR_INVALID_ARG;
  if (B == 0) return SD_OK;
  if (!src->k || !src->v || !src->len || !dst->k || !dst->v || !dst->len || !weights) return SD_ERR_INVALID_ARG;
  if (!sd_aligned16(src->k) || !sd_aligned16(src->v) || !sd_aligned16(dst->k) || !sd_aligned16(dst->v))
    return SD_ERR_INVALID_ARG;
  const size_t rows = static_cast<size_t>(B) * Hkv, ns = rows * src->capacity, nd = rows * dst->capacity, row = 2u * D;
  const void* in[3] = {src->k, src->v, weights};
  const size_t in_bytes[3] = {ns * row, ns * row, ns * 4};
  const void* to[4] = {dst->k, dst->v, weights_out, kept};
  const size_t to_bytes[4] = {nd * row, nd * row, weights_out ? nd * 4 : 0, kept ? rows * keep * 4 : 0};
  for (int i = 0; i < 3; ++i)
    for (int j = 0; j < 4; ++j)
      if (to_bytes[j] && overlap(in[i], in_bytes[i], to[j], to_bytes[j])) return SD_ERR_INVALID_ARG;
  if (src->len == dst->len) return SD_ERR_INVALID_ARG;
  if (sd_launch_pdl(evict_kernel, dim3(Hkv, B), dim3(kThreads), 0, reinterpret_cast<cudaStream_t>(stream), *src, weights,
                    *dst, keep, sinks, recent, weights_out, kept) != cudaSuccess) {
    (void)cudaGetLastError();
    return SD_ERR_CUDA;
  }
  return SD_OK;
}
