// Eviction from a KV cache by accumulated attention weight (sm_103a): of a scene's n
// keys a KV head keeps min(n, keep): the first `sinks`, the last `recent`, and of those
// between the ones with the largest weights (among equal weights the lowest index),
// moved in their order to another cache.
//
// Several CTAs a (KV head, scene), each moving its share of the places in dst: they need
// nothing of each other, as each finds the whole selection itself from the weights (4 bytes
// a key against the 512 of a kept row: 16384 keys are 64 KB from L2). The weight of the last
// key kept: the keys are counted by the leading 11 bits of an integer that orders as the
// weight does; those that share the deciding bits are listed, and a few of them ranked by
// counting, more of them counted by their other bits, in two more passes (over all keys
// where the list is too short: weights within an eighth of each other). Then a key's place is the number of kept keys before it: ballots,
// kept in shared memory, are summed a warp a range of keys, and the CTA lists its share from
// them, whose rows it copies with eight 16-byte loads a thread in flight.
#include "common.cuh"

SD_DEFINE_ERROR_ACCESSOR(sd_take_error_evict)

namespace {

constexpr int kThreads = 1024;
constexpr int kWarps = kThreads / 32;
constexpr int kBins = 2048;
constexpr int kList = 1024;     // kept keys that a CTA lists, then copies, at a time
constexpr int kRank = 64;      // listed keys that are ranked by counting
constexpr int kKeysMax = 20480; // keys whose integers and ballots stay in shared memory; more are read anew each time

// An integer that orders as the weight does (-0 as +0; NaN below every number).
__device__ __forceinline__ uint32_t order_of(float w) {
  const uint32_t u = __float_as_uint(w + 0.f);
  if ((u & 0x7fffffffu) > 0x7f800000u) return 0u;
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// The sum of x[w], w < n <= 32, by a whole warp.
__device__ __forceinline__ int sum_of(const int* x, int n, int lane) {
  return __reduce_add_sync(0xffffffffu, lane < n ? x[lane] : 0);
}

// Grid (parts, Hkv, B); dynamic shared memory for smem_keys keys.
__global__ void __launch_bounds__(kThreads) evict_kernel(const sd_kv_cache src, const float* weights, const sd_kv_cache dst,
                                                         int keep, int sinks, int recent, float* weights_out, int32_t* kept,
                                                         int smem_keys, int vec_shift) {
  extern __shared__ uint32_t order[];                  // [smem_keys], then ballots[smem_keys / 32]
  uint2* ballots = reinterpret_cast<uint2*>(order + smem_keys);  // of 32 keys: which stay, which tie
  __shared__ __align__(16) int bins[kBins];
  __shared__ __align__(16) int list[kList];
  __shared__ int warp_sum[kWarps];
  __shared__ int warp_kept[kWarps], warp_ties[kWarps];
  __shared__ int s_bin, s_left, s_count;
  __shared__ uint32_t s_T;
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
  auto order_at = [&](int i) { return cached ? order[i] : order_of(__ldcg(weights + i)); };

  // ---- T: the order of the last competing key kept; `ties` of those equal to it stay
  uint32_t T = 0;
  int ties = 0;
  if (!all) {
    int left = want;  // to be taken among the keys whose leading bits are T's
    // the bin in which the left-th key lies, the largest digits first: a prefix sum over the
    // bins, two a thread
    auto find = [&](int n_bins, int shift) {
      __syncthreads();
      static_assert(kBins == 2 * kThreads, "two bins a thread");
      const int2 c = reinterpret_cast<const int2*>(bins)[t];
      const int sum = c.x + c.y;
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
        const bool second = before + c.x < left;
        s_bin = 2 * t + second;
        s_left = left - before - (second ? c.x : 0);
      }
      __syncthreads();
      T |= static_cast<uint32_t>(n_bins - 1 - s_bin) << shift;
      left = s_left;
    };
    for (int i = t; i < kBins; i += kThreads) bins[i] = 0;
    if (t == 0) s_count = 0;
    __syncthreads();
    for (int i0 = t; i0 < n; i0 += 4 * kThreads) {
      float w[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) w[u] = i0 + u * kThreads < n ? __ldcg(weights + i0 + u * kThreads) : 0.f;
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int i = i0 + u * kThreads;
        const uint32_t o = order_of(w[u]);
        if (i < n && cached) order[i] = o;
        if (i >= lo && i < hi) atomicAdd(&bins[kBins - 1 - (o >> 21)], 1);
      }
    }
    if (left > 0) {
      find(kBins, 21);
      const int alike = bins[s_bin];  // keys that share T's leading bits
      const bool listed = alike <= kList;
      if (listed) {
        for (int i = lo + t; i < hi; i += kThreads) {
          const uint32_t o = order_at(i);
          if ((o >> 21) == (T >> 21)) list[atomicAdd(&s_count, 1)] = static_cast<int>(o);
        }
      }
      if (alike <= kRank) {
        __syncthreads();
        if (t < alike) {
          const uint32_t o = static_cast<uint32_t>(list[t]);
          int above = 0, equal = 0;
#pragma unroll 8
          for (int j = 0; j < alike; ++j) {
            const uint32_t x = static_cast<uint32_t>(list[j]);
            above += x > o;
            equal += x == o;
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
        for (int pass = 1; pass < 3; ++pass) {
          const int shift = pass == 1 ? 10 : 0, width = pass == 1 ? 11 : 10, n_bins = 1 << width;
          __syncthreads();
          for (int i = t; i < kBins; i += kThreads) bins[i] = 0;
          __syncthreads();
          const int from = listed ? 0 : lo, to = listed ? alike : hi;
          for (int i = from + t; i < to; i += kThreads) {
            const uint32_t o = listed ? static_cast<uint32_t>(list[i]) : order_at(i);
            if ((o >> (shift + width)) == (T >> (shift + width)))
              atomicAdd(&bins[n_bins - 1 - static_cast<int>((o >> shift) & (n_bins - 1))], 1);
          }
          find(n_bins, shift);
        }
      }
      ties = left;
    } else {
      T = 0xffffffffu;  // none of them stays (no key's order is all ones)
      __syncthreads();
    }
  }

  // ---- places: each warp's keys, a range of whole ballots
  const int per_warp = ((n + kWarps - 1) / kWarps + 31) / 32 * 32;
  const int i_lo = warp * per_warp, i_hi = min(n, i_lo + per_warp);
  // a key's kind: 2 stays, 1 ties with the last that stays, 0 goes
  auto kind = [&](int i) {
    if (i >= i_hi) return 0;
    if (all || i < lo || i >= hi) return 2;
    const uint32_t o = order_at(i);
    return o > T ? 2 : (o == T ? 1 : 0);
  };
  auto ballots_at = [&](int i0) {
    const int k = kind(i0 + lane);
    return make_uint2(__ballot_sync(0xffffffffu, k == 2), __ballot_sync(0xffffffffu, k == 1));
  };
  {
    int stay = 0, tie = 0;
    for (int i0 = i_lo; i0 < i_hi; i0 += 32) {
      const uint2 b = ballots_at(i0);
      if (cached && lane == 0) ballots[i0 >> 5] = b;
      stay += __popc(b.x);
      tie += __popc(b.y);
    }
    if (lane == 0) {
      warp_kept[warp] = stay;
      warp_ties[warp] = tie;
    }
  }
  __syncthreads();
  const int stay0 = sum_of(warp_kept, warp, lane), ties0 = sum_of(warp_ties, warp, lane);
  const int vec = 1 << vec_shift;
  const uint4* ks = static_cast<const uint4*>(src.k) + ((plane * src.capacity) << vec_shift);
  const uint4* vs = static_cast<const uint4*>(src.v) + ((plane * src.capacity) << vec_shift);
  uint4* kd = static_cast<uint4*>(dst.k) + ((plane * dst.capacity) << vec_shift);
  uint4* vd = static_cast<uint4*>(dst.v) + ((plane * dst.capacity) << vec_shift);
#pragma unroll 1
  for (int q_lo = p_lo; q_lo < p_hi; q_lo += kList) {
    const int q_hi = min(p_hi, q_lo + kList);
    __syncthreads();  // the list before is copied
    int stay = stay0, tie = ties0;
    for (int i0 = i_lo; i0 < i_hi && stay + min(tie, ties) < q_hi; i0 += 32) {
      const uint2 x = cached ? ballots[i0 >> 5] : ballots_at(i0);
      const int stay1 = stay + __popc(x.x), tie1 = tie + __popc(x.y);
      if (stay1 + min(tie1, ties) > q_lo) {
        const uint32_t below = (1u << lane) - 1;
        const int my_ties = tie + __popc(x.y & below);
        const int at = stay + __popc(x.x & below) + min(my_ties, ties);
        if ((((x.x >> lane) & 1) || (((x.y >> lane) & 1) && my_ties < ties)) && at >= q_lo && at < q_hi) list[at - q_lo] = i0 + lane;
      }
      stay = stay1;
      tie = tie1;
    }
    __syncthreads();
    const int count = q_hi - q_lo;
    for (int j = t; j < count; j += kThreads) {
      const int i = list[j];
      if (weights_out) weights_out[plane * dst.capacity + q_lo + j] = __ldcg(weights + i);
      if (kept) kept[plane * keep + q_lo + j] = i;
    }
    constexpr int kU = 4;
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
          kd[to + x] = k[u];
          vd[to + x] = v[u];
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
  const int smem_keys = src->capacity < kKeysMax ? (src->capacity + 31) / 32 * 32 : kKeysMax;
  static bool allowed[64];
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) {
    (void)cudaGetLastError();
    return SD_ERR_CUDA;
  }
  if (!allowed[dev]) {  // more than 48 KB of shared memory, once per device
    if (cudaFuncSetAttribute(evict_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kKeysMax * 4 + kKeysMax / 32 * 8) != cudaSuccess) {
      (void)cudaGetLastError();
      return SD_ERR_CUDA;
    }
    allowed[dev] = true;
  }
  if (sd_launch_pdl(evict_kernel, dim3(static_cast<unsigned>(parts), Hkv, B), dim3(kThreads), smem_keys * 4 + smem_keys / 32 * 8,
                    reinterpret_cast<cudaStream_t>(stream), *src, weights, *dst, keep, sinks, recent, weights_out, kept,
                    smem_keys, D == 64 ? 3 : 4) != cudaSuccess) {
    (void)cudaGetLastError();
    return SD_ERR_CUDA;
  }
  return SD_OK;
}
