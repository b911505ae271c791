// The largest value of a segment of one row of logits and its lowest index (sm_103a), for
// the acceptance kernels: running maxima only, the index looked up afterwards.
#pragma once
#include "common.cuh"

namespace {

constexpr int kThreads = 256;
constexpr int kStep = 4;  // 16-byte vectors a thread reads per step

// Order-preserving map of a float to uint32 (-0 as +0); every value, -inf
// included, maps above 0.
__device__ __forceinline__ uint32_t ordered(float x) {
  const uint32_t u = __float_as_uint(x + 0.f);
  return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}

__device__ __forceinline__ __nv_bfloat162 as_pair(uint32_t w) {
  __nv_bfloat162 v;
  memcpy(&v, &w, 4);
  return v;
}

// Largest value of a 16-byte vector, folded into m (NaN loses to any number).
template <typename T>
struct Fold;
template <>
struct Fold<float> {
  float m = -INFINITY;
  __device__ __forceinline__ void add(const uint4& w) {
    m = fmaxf(m, fmaxf(fmaxf(__uint_as_float(w.x), __uint_as_float(w.y)),
                       fmaxf(__uint_as_float(w.z), __uint_as_float(w.w))));
  }
  __device__ __forceinline__ float value() const { return m; }
};
template <>
struct Fold<__nv_bfloat16> {
  uint32_t m = 0xff80ff80u;  // -inf pair
  __device__ __forceinline__ void add(const uint4& w) {
    const __nv_bfloat162 x = __hmax2(__hmax2(as_pair(w.x), as_pair(w.y)), __hmax2(as_pair(w.z), as_pair(w.w)));
    const __nv_bfloat162 y = __hmax2(as_pair(m), x);
    memcpy(&m, &y, 4);
  }
  __device__ __forceinline__ float value() const { return fmaxf(sd_bf16_lo(m), sd_bf16_hi(m)); }
};

// (loads past the read-only path: the kernel is resident while its inputs are written)
__device__ __forceinline__ float load_one(const float* p) { return __ldcg(p); }
__device__ __forceinline__ float load_one(const __nv_bfloat16* p) { return sd_ldcg_bf16(p); }

// First element of a vector that equals best (a value it holds), as its offset.
__device__ __forceinline__ int first_equal(const float*, const uint4& w, float best) {
  const uint32_t x[4] = {w.x, w.y, w.z, w.w};
  int at = 0x7fffffff;
#pragma unroll
  for (int j = 3; j >= 0; --j)
    if (__uint_as_float(x[j]) == best) at = j;
  return at;
}
__device__ __forceinline__ int first_equal(const __nv_bfloat16*, const uint4& w, float best) {
  const uint32_t x[4] = {w.x, w.y, w.z, w.w};
  int at = 0x7fffffff;
#pragma unroll
  for (int j = 3; j >= 0; --j) {
    if (sd_bf16_hi(x[j]) == best) at = 2 * j + 1;
    if (sd_bf16_lo(x[j]) == best) at = 2 * j;
  }
  return at;
}

// The key (ordered value, then lowest index) of segment `seg` of a row's n_seg, whole 16-byte
// vectors vps each; segment 0 also takes the elements before the first 16-byte boundary, the
// last one those after the last. A CTA of kThreads; the same in every thread. s_best:
// kThreads / 32 words, s_index: one.
template <typename T>
__device__ __forceinline__ unsigned long long scan_segment(const T* row, int V, int seg, int n_seg, int vps, uint32_t* s_best,
                                                           uint32_t* s_index_p) {
  constexpr int kPer = 16 / sizeof(T);
  uint32_t& s_index = *s_index_p;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int head = min(V, static_cast<int>((16 - (reinterpret_cast<uintptr_t>(row) & 15)) & 15) / static_cast<int>(sizeof(T)));
  const int n_vec = (V - head) / kPer;
  const uint4* vec = reinterpret_cast<const uint4*>(row + head);
  const int v0 = min(n_vec, seg * vps), v1 = seg == n_seg - 1 ? n_vec : min(n_vec, v0 + vps);
  if (threadIdx.x == 0) s_index = 0xffffffffu;
  // ---- running maximum and the step that raised it (a thread's steps ascend)
  float best = -INFINITY;
  int step = -1;
  for (int v = v0 + static_cast<int>(threadIdx.x); v < v1; v += kStep * kThreads) {
    Fold<T> f;
    if (v + (kStep - 1) * kThreads < v1) {
      uint4 w[kStep];
#pragma unroll
      for (int k = 0; k < kStep; ++k) w[k] = __ldcg(vec + v + k * kThreads);
#pragma unroll
      for (int k = 0; k < kStep; ++k) f.add(w[k]);
    } else {
#pragma unroll
      for (int k = 0; k < kStep; ++k)
        if (v + k * kThreads < v1) f.add(__ldcg(vec + v + k * kThreads));
    }
    const float m = f.value();
    if (m > best) {
      best = m;
      step = v;
    }
  }
  // the single elements at the row's ends, one a thread (fewer than 8 each)
  float single = -INFINITY;
  int single_at = -1;
  if (seg == 0 && static_cast<int>(threadIdx.x) < head) single_at = threadIdx.x;
  if (seg == n_seg - 1 && threadIdx.x >= 32) {
    const int e = head + n_vec * kPer + static_cast<int>(threadIdx.x) - 32;
    if (e < V) single_at = e;
  }
  if (single_at >= 0) single = load_one(row + single_at);
  const float top = fmaxf(best, single);
  const uint32_t wbest = __reduce_max_sync(0xffffffffu, ordered(top == top ? top : -INFINITY));
  if (lane == 0) s_best[warp] = wbest;
  __syncthreads();
  uint32_t bmax = s_best[0];
#pragma unroll
  for (int w = 1; w < kThreads / 32; ++w) bmax = max(bmax, s_best[w]);
  // ---- the lowest index of the segment's maximum (no value above -inf: its start)
  uint32_t at = 0xffffffffu;
  const bool none = bmax == ordered(-INFINITY);
  if (single_at >= 0 && !none && ordered(single) == bmax) at = single_at;
  if (step >= 0 && ordered(best) == bmax) {
#pragma unroll
    for (int k = kStep - 1; k >= 0; --k) {
      const int v = step + k * kThreads;
      if (v >= v1) continue;
      const int e = first_equal(row, __ldcg(vec + v), best);
      if (e != 0x7fffffff) at = min(static_cast<uint32_t>(head + v * kPer + e), at);
    }
  }
  const uint32_t wat = __reduce_min_sync(0xffffffffu, at);
  if (lane == 0 && wat != 0xffffffffu) atomicMin(&s_index, wat);
  __syncthreads();
  const uint32_t idx = s_index != 0xffffffffu ? s_index : static_cast<uint32_t>(seg == 0 ? 0 : min(V - 1, head + v0 * kPer));
  return (static_cast<unsigned long long>(bmax) << 32) | (0xffffffffu - idx);
}

}  // namespace
