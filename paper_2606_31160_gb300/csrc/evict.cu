// Eviction from a KV cache by accumulated attention weight (sm_103a): of a scene's n
// keys a KV head keeps min(n, keep): the first `sinks`, the last `recent`, and of those
// between the ones with the largest weights (among equal weights the lowest index),
// moved in their order to another cache.
//
// Several CTAs a (KV head, scene), each moving its share of the places in dst: they need
// nothing of each other, as each finds the whole selection itself from the weights (4 bytes
// a key against the 512 of a kept row: 16384 keys are 64 KB from L2). The weight of the last
// key kept: integers that order as the weights do are counted by 4096 equal ranges between
// the least and the largest of them; those of the deciding range are listed, and a few
// ranked by counting, more counted by their other bits (over all keys where the list is too
// short). Then a key's place is the number of kept keys before it: a lane marks four keys, a
// warp sums a range of them, and the CTA lists its share from the marks, whose rows it
// copies with four 16-byte loads a thread in flight.
//
// What bounds it. 8 scenes of 16384 keys to 4096, 8 heads: 55.2 us, of which the rows'
// copies are ~42 (268 MB at 6.4 TB/s; with eight loads a thread and stores that stay in L2
// 56.7) and the selection 12 (20 thousand cycles: lengths 3.0, weights and their range 3.3,
// counting 3.0, list 2.3, rank 1.8, marks 2.1, places 5.0), before which no row can be
// copied. It is instructions, not latency: four keys a lane took it from 31 thousand cycles
// (and one scene of 4096 keys from 9.4 to 7.7 us), more loads in flight did not.
#include "common.cuh"

#include <mutex>

SD_DEFINE_ERROR_ACCESSOR(sd_take_error_evict)

namespace {

constexpr int kThreads = 1024;
constexpr int kWarps = kThreads / 32;
constexpr int kBits = 12, kBins = 1 << kBits;
constexpr int kBlock = 128;     // keys a warp looks at at once: four a lane
constexpr int kList = 2048;     // kept keys that a CTA lists, then copies, at a time
constexpr int kRank = 128;      // listed keys that are ranked by counting
constexpr int kKeysMax = 20480; // keys whose integers and marks stay in shared memory; more are read anew each time

// An integer that orders as the weight does (-0 as +0; NaN below every number: 1). 0 is
// no key's, nor is kSure, which stands for the keys that stay whatever their weight.
constexpr uint32_t kSure = 0xffffffffu;
__device__ __forceinline__ uint32_t order_of(float w) {
  const uint32_t u = __float_as_uint(w + 0.f);
  return w != w ? 1u : u ^ (static_cast<uint32_t>(static_cast<int>(u) >> 31) | 0x80000000u);
}

// The sum of x[w], w < n <= 32, by a whole warp.
__device__ __forceinline__ int sum_of(const int* x, int n, int lane) {
  return __reduce_add_sync(0xffffffffu, lane < n ? x[lane] : 0);
}

// Grid (parts, Hkv, B); dynamic shared memory for smem_keys keys.
__global__ void __launch_bounds__(kThreads) evict_kernel(const sd_kv_cache src, const float* weights, const sd_kv_cache dst,
                                                         int keep, int sinks, int recent, float* weights_out, int32_t* kept,
                                                         int smem_keys, int vec_shift) {
  extern __shared__ __align__(16) uint32_t order[];    // [smem_keys], then the marks
  uint8_t* marks = reinterpret_cast<uint8_t*>(order + smem_keys);  // of four keys: which stay, 16 times which tie
  __shared__ __align__(16) int bins[kBins];
  __shared__ __align__(16) int list[kList + 4];
  __shared__ int warp_sum[kWarps];
  __shared__ int warp_kept[kWarps], warp_ties[kWarps];
  __shared__ int s_bin, s_left, s_count;
  __shared__ uint32_t s_T;
  __shared__ uint32_t warp_least[kWarps], warp_most[kWarps];
  sd_pdl_enter();
  const int part = blockIdx.x, parts = gridDim.x, h = blockIdx.y, b = blockIdx.z, Hkv = src.n_kv_heads;
  const int t = threadIdx.x, warp = t >> 5, lane = t & 31;
  const int n = __ldcg(src.len + b);
  if (n < 0 || n > src.capacity) {
    if (t == 0 && part == 0 && h == 0) sd_set_error(SD_DEVERR_LENGTH);
    return;
  }
  const long long plane = static_cast<long long>(b) * Hkv + h;
  weights += plane * src.capacity;
  const int m = min(n, keep);                                   // kept keys
  const int p_lo = static_cast<int>(static_cast<long long>(part) * m / parts);
  const int p_hi = static_cast<int>(static_cast<long long>(part + 1) * m / parts);
  if (part == 0 && h == 0 && t == 0) dst.len[b] = m;
  if (kept && part == 0)
    for (int j = m + t; j < keep; j += kThreads) kept[plane * keep + j] = -1;
  if (p_lo == p_hi) return;
  const int lo = min(sinks, n), hi = max(lo, n - recent);       // the keys that compete
  const int want = m - lo - (n - hi);
  const bool all = n <= keep;                                   // every key stays
  const bool cached = n <= smem_keys;
  const bool aligned = (reinterpret_cast<uintptr_t>(weights) & 15) == 0;
  auto weights4 = [&](int i, float (&w)[4]) {  // of keys i .. i + 3, i a multiple of 4; 0 past the last
    if (aligned && i + 4 <= n) {
      const float4 x = __ldcg(reinterpret_cast<const float4*>(weights + i));
      w[0] = x.x;
      w[1] = x.y;
      w[2] = x.z;
      w[3] = x.w;
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) w[e] = i + e < n ? __ldcg(weights + i + e) : 0.f;
    }
  };
  auto orders4 = [&](int i, const float (&w)[4]) {  // 0 past the last key
    uint32_t o[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] = order_of(w[e]);
    if (i < lo || i + 4 > hi) {
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] = i + e >= n ? 0u : (i + e < lo || i + e >= hi ? kSure : o[e]);
    }
    return make_uint4(o[0], o[1], o[2], o[3]);
  };
  auto order4 = [&](int i) {
    if (cached) return *reinterpret_cast<const uint4*>(order + i);
    float w[4];
    weights4(i, w);
    return orders4(i, w);
  };
  const int n_blocks = (n + kBlock - 1) / kBlock;
  // f(order) of every key
  auto each = [&](auto f) {
    for (int i = 4 * t; i < n; i += 4 * kThreads) {
      const uint4 o = order4(i);
      f(o.x);
      f(o.y);
      f(o.z);
      f(o.w);
    }
  };

  // ---- T: the order of the last competing key kept; `ties` of those equal to it stay
  uint32_t T = 0;
  int ties = 0;
  if (!all) {
    int left = want;  // to be taken among the keys of the range [T, T + 2^shift)
    // every key's integer, the least and the largest of those that compete
    for (int i = t; i < kBins; i += kThreads) bins[i] = 0;
    if (t == 0) s_count = 0;
    uint32_t least = kSure, most = 0;  // less and plus 1: of 0 and kSure neither counts
    constexpr int kU = 4;
    for (int i0 = 4 * t; i0 < n_blocks * kBlock; i0 += kU * 4 * kThreads) {
      float w[kU][4];
#pragma unroll
      for (int u = 0; u < kU; ++u) weights4(i0 + u * 4 * kThreads, w[u]);
#pragma unroll
      for (int u = 0; u < kU; ++u) {
        const int i = i0 + u * 4 * kThreads;
        if (i >= n_blocks * kBlock) break;
        const uint4 o = orders4(i, w[u]);
        if (cached) *reinterpret_cast<uint4*>(order + i) = o;
        least = min(least, min(min(o.x - 1, o.y - 1), min(o.z - 1, o.w - 1)));
        most = max(most, max(max(o.x + 1, o.y + 1), max(o.z + 1, o.w + 1)));
      }
    }
    least = __reduce_min_sync(0xffffffffu, least);
    most = __reduce_max_sync(0xffffffffu, most);
    if (lane == 0) {
      warp_least[warp] = least;
      warp_most[warp] = most;
    }
    __syncthreads();
    // kBins ranges from the least on, each of the smallest power of two that reaches the largest
    T = __reduce_min_sync(0xffffffffu, warp_least[lane]) + 1;
    static_assert(kWarps == 32, "a lane a warp");
    int shift = max(0, 32 - __clz(__reduce_max_sync(0xffffffffu, warp_most[lane]) - 1 - T) - kBits);
    // the bin in which the left-th key lies, the largest digits first: a prefix sum over the
    // bins, four a thread
    auto find = [&](int n_bins) {
      __syncthreads();
      static_assert(kBins == 4 * kThreads, "four bins a thread");
      const int4 c = reinterpret_cast<const int4*>(bins)[t];
      const int sum = (c.x + c.y) + (c.z + c.w);
      int before = sum;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int x = __shfl_up_sync(0xffffffffu, before, o);
        if (lane >= o) before += x;
      }
      if (lane == 31) warp_sum[warp] = before;
      __syncthreads();
      before += sum_of(warp_sum, warp, lane) - sum;
      if (before < left && before + sum >= left) {  // one thread's
        const int c1 = before + c.x, c2 = c1 + c.y, c3 = c2 + c.z;
        const int which = (c1 < left) + (c2 < left) + (c3 < left);
        s_bin = 4 * t + which;
        s_left = left - (which == 0 ? before : which == 1 ? c1 : which == 2 ? c2 : c3);
      }
      __syncthreads();
      T += static_cast<uint32_t>(n_bins - 1 - s_bin) << shift;
      left = s_left;
    };
    if (left > 0) {
      each([&](uint32_t o) {
        if (o - 1 < kSure - 1) atomicAdd(&bins[kBins - 1 - ((o - T) >> shift)], 1);
      });
      find(kBins);
      const int alike = bins[s_bin];  // keys in T's range
      const bool listed = alike <= kList;
      if (listed) {
        // (0 and kSure are further than 2^20 from every weight's integer)
        each([&](uint32_t o) {
          if (o - T < 1u << shift) list[atomicAdd(&s_count, 1)] = static_cast<int>(o);
        });
      }
      if (alike <= kRank) {
        if (t >= alike && t < alike + 3) list[t] = 0;  // (read four at a time)
        __syncthreads();
        if (t < alike) {
          const uint32_t o = static_cast<uint32_t>(list[t]);
          int above = 0, equal = 0;
#pragma unroll 4
          for (int j = 0; j < alike; j += 4) {
            const uint4 x = *reinterpret_cast<const uint4*>(list + j);
            above += (x.x > o) + (x.y > o) + (x.z > o) + (x.w > o);
            equal += (x.x == o) + (x.y == o) + (x.z == o) + (x.w == o);
          }
          if (above < left && above + equal >= left) {  // the threads with that one integer
            s_T = o;
            s_left = left - above;
          }
        }
        __syncthreads();
        T = s_T;
        left = s_left;
      } else {
#pragma unroll 1
        while (shift > 0) {
          const int width = min(kBits, shift), n_bins = 1 << width;
          shift -= width;
          __syncthreads();
          for (int i = t; i < kBins; i += kThreads) bins[i] = 0;
          __syncthreads();
          auto count = [&](uint32_t o) {
            if (o - T < 1u << (shift + width)) atomicAdd(&bins[n_bins - 1 - static_cast<int>((o - T) >> shift)], 1);
          };
          if (listed) {
            for (int i = t; i < alike; i += kThreads) count(static_cast<uint32_t>(list[i]));
          } else {
            each(count);
          }
          find(n_bins);
        }
      }
      ties = left;
    } else {
      T = kSure - 1;  // none of them stays
      __syncthreads();
    }
  }

  // ---- places: each warp's keys, a range of whole blocks
  const int per_warp = (n_blocks + kWarps - 1) / kWarps;
  const int blk_lo = min(n_blocks, warp * per_warp), blk_hi = min(n_blocks, blk_lo + per_warp);
  auto marks_of = [&](int blk) {
    const uint4 o = order4(blk * kBlock + 4 * lane);
    return (o.x > T ? 1u : 0u) | (o.y > T ? 2u : 0u) | (o.z > T ? 4u : 0u) | (o.w > T ? 8u : 0u) |
           (o.x == T ? 16u : 0u) | (o.y == T ? 32u : 0u) | (o.z == T ? 64u : 0u) | (o.w == T ? 128u : 0u);
  };
  auto ones = [](uint32_t x) { return __popc(x & 15u) | __popc(x >> 4) << 16; };  // that stay, and 2^16 times that tie
  if (!all) {
    int stay = 0, tie = 0;
    for (int blk = blk_lo; blk < blk_hi; ++blk) {
      const uint32_t x = marks_of(blk);
      if (cached) marks[blk * 32 + lane] = static_cast<uint8_t>(x);
      stay += __popc(x & 15u);
      tie += __popc(x >> 4);
    }
    stay = __reduce_add_sync(0xffffffffu, static_cast<uint32_t>(stay));
    tie = __reduce_add_sync(0xffffffffu, static_cast<uint32_t>(tie));
    if (lane == 0) {
      warp_kept[warp] = stay;
      warp_ties[warp] = tie;
    }
  }
  __syncthreads();
  const int stay0 = all ? 0 : sum_of(warp_kept, warp, lane), ties0 = all ? 0 : sum_of(warp_ties, warp, lane);
  const int vec = 1 << vec_shift;
  const uint4* ks = static_cast<const uint4*>(src.k) + ((plane * src.capacity) << vec_shift);
  const uint4* vs = static_cast<const uint4*>(src.v) + ((plane * src.capacity) << vec_shift);
  uint4* kd = static_cast<uint4*>(dst.k) + ((plane * dst.capacity) << vec_shift);
  uint4* vd = static_cast<uint4*>(dst.v) + ((plane * dst.capacity) << vec_shift);
#pragma unroll 1
  for (int q_lo = p_lo; q_lo < p_hi; q_lo += kList) {
    const int q_hi = min(p_hi, q_lo + kList);
    __syncthreads();  // the list before is copied
    if (all) {
      for (int j = q_lo + t; j < q_hi; j += kThreads) list[j - q_lo] = j;
    } else {
      int stay = stay0, tie = ties0;
      const bool mine = stay + warp_kept[warp] + min(tie + warp_ties[warp], ties) > q_lo;  // of this warp's keys one at least
      for (int blk = blk_lo; mine && blk < blk_hi && stay + min(tie, ties) < q_hi; ++blk) {
        const uint32_t x = cached ? marks[blk * 32 + lane] : marks_of(blk);
        const int own = ones(x);
        int upto = own;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const int y = __shfl_up_sync(0xffffffffu, upto, o);
          if (lane >= o) upto += y;
        }
        const int sums = __shfl_sync(0xffffffffu, upto, 31), stay1 = stay + (sums & 0xffff), tie1 = tie + (sums >> 16);
        if (stay1 + min(tie1, ties) > q_lo) {
          int at = stay + ((upto - own) & 0xffff) - q_lo, tied = tie + ((upto - own) >> 16);
          const int first = blk * kBlock + 4 * lane;
          // (one store a key, its address chosen: branches were slower)
          const int count = q_hi - q_lo;
          const bool any_tie = sums >> 16 != 0;
          if (!any_tie) at += min(tie, ties);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const bool stays = (x >> e) & 1, ties_here = any_tie && ((x >> (4 + e)) & 1);
            const int place = any_tie ? at + min(tied, ties) : at;
            const bool ok = (stays || (ties_here && tied < ties)) && static_cast<unsigned>(place) < static_cast<unsigned>(count);
            list[ok ? place : kList] = first + e;
            at += stays;
            tied += ties_here;
          }
        }
        stay = stay1;
        tie = tie1;
      }
    }
    __syncthreads();
    const int count = q_hi - q_lo;
    for (int j = t; j < count; j += kThreads) {
      const int i = list[j];
      if (weights_out) weights_out[plane * dst.capacity + q_lo + j] = __ldcg(weights + i);
      if (kept) kept[plane * keep + q_lo + j] = i;
    }
    constexpr int kU = 2;
    const long long to = static_cast<long long>(q_lo) << vec_shift;
    for (int u0 = t; u0 < count << vec_shift; u0 += kU * kThreads) {
      uint4 k[kU], v[kU];
#pragma unroll
      for (int u = 0; u < kU; ++u) {
        const int x = u0 + u * kThreads;
        if (x < count << vec_shift) {
          const long long from = (static_cast<long long>(list[x >> vec_shift]) << vec_shift) + (x & (vec - 1));
          k[u] = __ldcs(ks + from);
          v[u] = __ldcs(vs + from);
        }
      }
#pragma unroll
      for (int u = 0; u < kU; ++u) {
        const int x = u0 + u * kThreads;
        if (x < count << vec_shift) {
          __stcs(kd + to + x, k[u]);
          __stcs(vd + to + x, v[u]);
        }
      }
    }
  }
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
  if (B > 65535 || Hkv > 65535) return SD_ERR_UNSUPPORTED;
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
  // a CTA an SM over all heads, as long as each has 32 rows or more to move. (Two CTAs of half
  // the threads find every selection twice an SM.)
  const long long pairs = static_cast<long long>(B) * Hkv;
  long long parts = sd_num_sms() / pairs;
  if (parts < 1) parts = 1;
  if (parts > (keep + 31) / 32) parts = (keep + 31) / 32;
  const int smem_keys = src->capacity < kKeysMax ? (src->capacity + kBlock - 1) / kBlock * kBlock : kKeysMax;
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) {
    (void)cudaGetLastError();
    return SD_ERR_CUDA;
  }
  // more than 48 KB of shared memory, once per device
  static std::once_flag once[64];
  static bool allowed[64];
  std::call_once(once[dev], [dev] {
    allowed[dev] = cudaFuncSetAttribute(evict_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                        kKeysMax * 4 + kKeysMax / 32 * 8) == cudaSuccess;
    if (!allowed[dev]) (void)cudaGetLastError();
  });
  if (!allowed[dev]) return SD_ERR_CUDA;
  if (sd_launch_pdl(evict_kernel, dim3(static_cast<unsigned>(parts), Hkv, B), dim3(kThreads), smem_keys * 4 + smem_keys / 32 * 8,
                    reinterpret_cast<cudaStream_t>(stream), *src, weights, *dst, keep, sinks, recent, weights_out, kept,
                    smem_keys, D == 64 ? 3 : 4) != cudaSuccess) {
    (void)cudaGetLastError();
    return SD_ERR_CUDA;
  }
  return SD_OK;
}
