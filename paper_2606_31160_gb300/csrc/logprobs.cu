// Log probabilities of given tokens with the entropy and the top alternatives of their
// rows (sm_103a). With x = (z - m) / T, m the row's largest logit, S = sum e^x and
// W = sum x e^x over the vocabulary:
//     log p(t) = x_t - ln S,    entropy = ln S - W / S,
//     alternatives: the top_n largest logits, equal ones by the lowest index.
//
// One pass over the logits. A cluster of CTAs has a row, each a contiguous segment; a
// thread folds chunks of 32 bytes, four in flight, into (m, S, W) under its running maximum,
// which it moves only when a chunk's maximum passes it. S and W merge over lanes, warps
// and CTAs in a fixed order.
//
// Alternatives without a second pass: a thread remembers which of its chunks holds its
// largest logit, and the second chunk's largest. The top_n-th largest of each warp's 4 or 8
// largest maxima is a bound that at least top_n elements of the segment reach, and few more
// do. A remembered chunk that reaches it is read again, one round trip; all chunks of a
// thread only where its second one does too. What reaches the bound is listed and ranked by
// counting; the cluster's first CTA ranks the CTAs' lists. (Every chunk of the threads whose
// maximum reaches the bound read again: 34.9 us for 256 rows of 608 KB where this takes
// 32.0; with two chunks remembered 32.7.) A bound
// of -inf (a masked vocabulary) lists the finite logits only, the lowest masked indices fill
// the rest; a list that overflows (hundreds of equal logits) is replaced by top_n passes for
// the next largest.
//
// Small CTAs, four an SM: while one merges and ranks, others stream. 256 rows of 608 KB:
// 4.8 TB/s, 0.71 of the measured copy rate; a CTA reads its segment for four fifths of the
// time, the merge and the list are the rest. 8 rows of 304 KB: 7.0 us, 5 of which is latency
// (launch, two round trips to DRAM, two cluster barriers).
#include "common.cuh"

#include <float.h>
#include <math.h>

SD_DEFINE_ERROR_ACCESSOR(sd_take_error_logprobs)

namespace {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr int kTopMax = 32;
constexpr int kList = 1024;      // candidates a CTA lists
constexpr int kUnroll = 4;       // 32-byte chunks a thread has in flight
constexpr int kMaxCluster = 8;
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

// An integer that orders as the logit does (-0 as +0).
__device__ __forceinline__ uint32_t order_of(float z) {
  const uint32_t u = __float_as_uint(z + 0.f);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t o) { return __uint_as_float(o & 0x80000000u ? o & 0x7fffffffu : ~o); }
constexpr uint32_t kOrderNegInf = 0x007fffffu;  // order_of(-inf)
// (value, lowest index first) as one integer
__device__ __forceinline__ uint64_t key_of(float z, int i) {
  return (static_cast<uint64_t>(order_of(z)) << 32) | static_cast<uint32_t>(~i);
}
__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float max_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ float max3_nan(float a, float b, float c) {
  float r;
  asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}
template <int kN>
__device__ __forceinline__ float largest(const float (&z)[kN]) {  // NaN if one is
  static_assert(kN % 2 == 0, "pairs");
  float m = max_nan(z[0], z[1]);
#pragma unroll
  for (int j = 2; j < kN; j += 2) m = max3_nan(m, z[j], z[j + 1]);
  return m;
}
__device__ __forceinline__ float redux_max(float x) {
  float r;
  asm("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(x));
  return r;
}
struct Chunk {
  uint32_t w[8];
};
__device__ __forceinline__ Chunk load32(const void* p) {
  Chunk c;
  asm volatile("ld.global.L1::no_allocate.v8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
               : "=r"(c.w[0]), "=r"(c.w[1]), "=r"(c.w[2]), "=r"(c.w[3]), "=r"(c.w[4]), "=r"(c.w[5]), "=r"(c.w[6]), "=r"(c.w[7])
               : "l"(p));
  return c;
}
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
__device__ __forceinline__ uint32_t smem_addr(const void* p) { return static_cast<uint32_t>(__cvta_generic_to_shared(p)); }
// Address of the same shared variable in the cluster's CTA 0.
__device__ __forceinline__ uint32_t in_first_cta(const void* p) {
  uint32_t r;
  asm volatile("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(r) : "r"(smem_addr(p)));
  return r;
}

template <bool kBf16>
struct Type {
  static constexpr int kElem = kBf16 ? 2 : 4;
  static constexpr int kPer = 32 / kElem;  // logits a chunk
  static __device__ __forceinline__ void unpack(const Chunk& c, float (&z)[kPer]) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      if constexpr (kBf16) {
        z[2 * j] = sd_bf16_lo(c.w[j]);
        z[2 * j + 1] = sd_bf16_hi(c.w[j]);
      } else {
        z[j] = __uint_as_float(c.w[j]);
      }
    }
  }
  static __device__ __forceinline__ float load(const void* z, long long i) {
    return kBf16 ? sd_ldcg_bf16(static_cast<const __nv_bfloat16*>(z) + i) : __ldcg(static_cast<const float*>(z) + i);
  }
};

__device__ __forceinline__ uint64_t pack2(float lo, float hi) {
  uint64_t d;
  asm("mov.b64 %0, {%1, %2};" : "=l"(d) : "f"(lo), "f"(hi));
  return d;
}
__device__ __forceinline__ void unpack2(uint64_t d, float& lo, float& hi) {
  asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(d));
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t d;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
  return d;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
  uint64_t d;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
  uint64_t d;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}

// Sums relative to the largest logit m, x = (z - m) log2(e) / T: S = sum 2^x, W = sum x 2^x.
struct Stat {
  float m, S, W;
};
// s moved to the maximum M >= s.m. Nothing seen: m = -inf, and S is 0 or NaN.
__device__ __forceinline__ void move_to(Stat& s, float M, float c) {
  if (s.m == M) return;
  if (s.m == -INFINITY) {
    s.S *= 0.f;
    s.W = s.S;
  } else {
    const float d = fmaxf((s.m - M) * c, -1000.f), f = ex2(d);  // (a mask's lowest value: 0 times -inf in W)
    s.W = f * fmaf(d, s.S, s.W);
    s.S *= f;
  }
  s.m = M;
}

// A thread's sums in two halves, for even and odd elements.
struct Fold {
  float m;
  uint64_t S, W;
  float m2;  // the second largest of the chunks' maxima
  int i1;    // the chunk of the largest, -1: none
};
__device__ __forceinline__ void move_fold(Fold& f, float M, float c) {
  Stat a{f.m, 0.f, 0.f}, b{f.m, 0.f, 0.f};
  unpack2(f.S, a.S, b.S);
  unpack2(f.W, a.W, b.W);
  move_to(a, M, c);
  move_to(b, M, c);
  f.m = M;
  f.S = pack2(a.S, b.S);
  f.W = pack2(a.W, b.W);
}
template <int kN>
__device__ __forceinline__ void fold(Fold& f, const float (&z)[kN], int chunk, float c) {
  const float bm = largest(z);
  if (bm == -INFINITY) return;  // nothing but tokens of probability 0
  if (bm > f.m2) {
    f.m2 = fminf(bm, f.m);
    if (bm > f.m) {
      f.i1 = chunk;
      move_fold(f, bm, c);
    }
  }
  const uint64_t c2 = pack2(c, c), m2 = pack2(-f.m, -f.m);
#pragma unroll
  for (int j = 0; j < kN; j += 2) {
    float x0, x1;
    unpack2(mul2(add2(pack2(z[j], z[j + 1]), m2), c2), x0, x1);
    x0 = max_nan(x0, -1000.f);  // -inf: 0 * -1000, not 0 * -inf
    x1 = max_nan(x1, -1000.f);
    const uint64_t e = pack2(ex2(x0), ex2(x1));
    f.S = add2(f.S, e);
    f.W = fma2(e, pack2(x0, x1), f.W);
  }
}

// Grid (cluster size, rows).
template <bool kBf16>
__global__ void __launch_bounds__(kThreads, 4)
    logprobs_kernel(const void* logits, long long stride, int V, const int32_t* tokens, float inv_t, int top_n,
                    float* logprob, float* entropy, int32_t* top_ids, float* top_logprobs) {
  using T = Type<kBf16>;
  constexpr int kPer = T::kPer;
  __shared__ __align__(16) uint64_t list[kList];
  __shared__ __align__(16) uint64_t best[kMaxCluster * kTopMax];  // of the first CTA: every rank's, top_n each
  __shared__ Stat stat[kWarps];
  __shared__ Stat cta_stat[kMaxCluster];
  __shared__ uint32_t warp_top[kWarps * 8];
  __shared__ int n_list;
  const int csize = gridDim.x, rank = blockIdx.x;
  const int t = threadIdx.x, warp = t >> 5, lane = t & 31;
  if (t == 0) n_list = 0;
  for (int i = t; i < kMaxCluster * kTopMax; i += kThreads) best[i] = 0;
  if (csize > 1) {  // waited for before the first store into another CTA
    __syncthreads();
    cluster_arrive();
  }
  sd_pdl_enter();
  const long long row = blockIdx.y;
  const char* z0 = static_cast<const char*>(logits) + row * stride * T::kElem;
  const float c = fminf(inv_t * kLog2e, FLT_MAX);  // (0 * c is 0 at the smallest temperatures too)
  // the token's logit travels with the rest
  int tok = -1;
  float z_tok = 0.f;
  if (rank == 0 && t == 0) {
    tok = __ldcg(tokens + row);
    if (tok >= 0 && tok < V) z_tok = T::load(z0, tok);
  }
  // whole chunks of the row: [lead, lead + n_vec * kPer); the ends are single elements
  const int lead = min(V, static_cast<int>(((32 - (reinterpret_cast<uintptr_t>(z0) & 31)) & 31) / T::kElem));
  const int n_vec = (V - lead) / kPer;
  const int tail = lead + n_vec * kPer;
  const Chunk* vec = reinterpret_cast<const Chunk*>(z0 + static_cast<long long>(lead) * T::kElem);
  const int v_lo = static_cast<int>(static_cast<long long>(rank) * n_vec / csize);
  const int v_hi = static_cast<int>(static_cast<long long>(rank + 1) * n_vec / csize);
  // single elements: thread t < lead of the first CTA, the next ones the tail's
  int edge = -1;
  if (rank == 0) edge = t < lead ? t : (t - lead < V - tail ? tail + t - lead : -1);

  Fold f{-INFINITY, 0ull, 0ull, -INFINITY, -1};
  for (int v = v_lo + t; v < v_hi; v += kUnroll * kThreads) {
    Chunk r[kUnroll];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u)
      if (v + u * kThreads < v_hi) r[u] = load32(vec + v + u * kThreads);
#pragma unroll
    for (int u = 0; u < kUnroll; ++u)
      if (v + u * kThreads < v_hi) {
        float z[kPer];
        T::unpack(r[u], z);
        fold(f, z, v + u * kThreads, c);
      }
  }
  float z_edge = -INFINITY;
  if (edge >= 0) {
    z_edge = T::load(z0, edge);
    float z[2] = {z_edge, -INFINITY};
    fold(f, z, -1, c);
  }
  const uint32_t mine = order_of(f.m);  // this thread's largest
  Stat s{f.m, 0.f, 0.f};
  {
    float a, b;
    unpack2(f.S, a, b);
    s.S = a + b;
    unpack2(f.W, a, b);
    s.W = a + b;
  }

  // ---- (m, S, W) over the warp, the CTA and the cluster
  move_to(s, redux_max(s.m), c);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    s.S += __shfl_xor_sync(0xffffffffu, s.S, o);
    s.W += __shfl_xor_sync(0xffffffffu, s.W, o);
  }
  if (lane == 0) stat[warp] = s;
  const int per_warp = top_n <= 16 ? 4 : 8;  // of a warp's maxima, the largest
  if (top_n > 0) {
    uint32_t o = mine, keep = 0;
    for (int j = 0; j < per_warp; ++j) {
      const uint32_t top = __reduce_max_sync(0xffffffffu, o);
      if (lane == j) keep = top;
      if (lane == __ffs(__ballot_sync(0xffffffffu, o == top)) - 1) o = 0;
    }
    if (lane < per_warp) warp_top[warp * per_warp + lane] = keep;
  }
  __syncthreads();
  if (csize > 1) cluster_wait();  // every CTA of the cluster has started
  if (warp == 0) {
    Stat a = lane < kWarps ? stat[lane] : Stat{-INFINITY, 0.f, 0.f};
    move_to(a, redux_max(a.m), c);
#pragma unroll
    for (int o = kWarps / 2; o > 0; o >>= 1) {
      a.S += __shfl_xor_sync(0xffffffffu, a.S, o);
      a.W += __shfl_xor_sync(0xffffffffu, a.W, o);
    }
    if (lane == 0) {
      if (csize == 1) {
        cta_stat[0] = a;
      } else {
        const uint32_t to = in_first_cta(&cta_stat[rank]);
        asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(to), "f"(a.m) : "memory");
        asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(to + 4), "f"(a.S) : "memory");
        asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(to + 8), "f"(a.W) : "memory");
      }
    }
  }
  if (top_n > 0) {
    // the top_n-th largest of the warps' largest, by every warp: the largest that top_n reach
    const uint32_t x0 = warp_top[lane], x1 = per_warp == 8 ? warp_top[32 + lane] : 0u;
    int c0 = 0, c1 = 0;
#pragma unroll
    for (int j = 0; j < 32; ++j) {
      const uint32_t y0 = __shfl_sync(0xffffffffu, x0, j);
      c0 += y0 >= x0;
      c1 += y0 >= x1;
    }
    if (per_warp == 8) {
#pragma unroll
      for (int j = 0; j < 32; ++j) {
        const uint32_t y1 = __shfl_sync(0xffffffffu, x1, j);
        c0 += y1 >= x0;
        c1 += y1 >= x1;
      }
    }
    uint32_t bound = __reduce_max_sync(0xffffffffu, max(c0 >= top_n ? x0 : 0u, c1 >= top_n ? x1 : 0u));
    bound = max(bound, kOrderNegInf + 1);  // finite logits only
    auto offer = [&](float z, int i) {
      if (order_of(z) >= bound) {
        const int at = atomicAdd(&n_list, 1);
        if (at < kList) list[at] = key_of(z, i);
      }
    };
    if (edge >= 0) offer(z_edge, edge);
    auto again = [&](int v, const Chunk& r) {
      float z[kPer];
      T::unpack(r, z);
      const float m = largest(z);
      if (order_of(m) >= bound || m != m) {
        const int i = lead + v * kPer;
#pragma unroll
        for (int j = 0; j < kPer; ++j) offer(z[j], i + j);
      }
    };
    // the chunk that a thread remembers
    const bool many = order_of(f.m2) >= bound;
    if (mine >= bound && f.i1 >= 0 && !many) again(f.i1, load32(vec + f.i1));
    // every chunk of the threads with a second one, two threads' at once
    uint32_t who = __ballot_sync(0xffffffffu, many);
    while (who) {
      const int v0 = v_lo + warp * 32 + __ffs(who) - 1 + lane * kThreads;
      who &= who - 1;
      const int v1 = who ? v_lo + warp * 32 + __ffs(who) - 1 + lane * kThreads : v_hi;
      who &= who - 1;
      for (int o = 0; v0 + o < v_hi || v1 + o < v_hi; o += 32 * kThreads) {
        Chunk r1, r2;
        if (v0 + o < v_hi) r1 = load32(vec + v0 + o);
        if (v1 + o < v_hi) r2 = load32(vec + v1 + o);
        if (v0 + o < v_hi) again(v0 + o, r1);
        if (v1 + o < v_hi) again(v1 + o, r2);
      }
    }
    __syncthreads();
    const int n = n_list;
    // the segment's j-th largest to place j of its part of the first CTA's array
    auto put = [&](int j, uint64_t k) {
      if (csize == 1) best[j] = k;
      else asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(in_first_cta(&best[rank * top_n + j])), "l"(k) : "memory");
    };
    if (n <= kList) {
      if (t == 0 && (n & 1) && n < kList) list[n] = 0;  // read in pairs
      __syncthreads();
      for (int i = t; i < n; i += kThreads) {
        const uint64_t k = list[i];
        int above = 0;
#pragma unroll 8
        for (int j = 0; j < n; j += 2) {
          const ulonglong2 y = *reinterpret_cast<const ulonglong2*>(list + j);
          above += (y.x > k) + (y.y > k);
        }
        if (above < top_n) put(above, k);
      }
    } else {
      // too many equals: the next largest, one by one
      __shared__ uint64_t part[kWarps];
      uint64_t limit = ~0ull;
      for (int j = 0; j < top_n; ++j) {
        uint64_t k = 0;
        auto look = [&](float z, int i) {
          const uint64_t x = key_of(z, i);
          if (x < limit && x > k) k = x;
        };
        if (edge >= 0) look(z_edge, edge);
        for (int v = v_lo + t; v < v_hi; v += kThreads) {
          float z[kPer];
          T::unpack(load32(vec + v), z);
#pragma unroll
          for (int e = 0; e < kPer; ++e) look(z[e], lead + v * kPer + e);
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) k = max(k, __shfl_xor_sync(0xffffffffu, k, o));
        __syncthreads();
        if (lane == 0) part[warp] = k;
        __syncthreads();
        for (int w = 0; w < kWarps; ++w) k = max(k, part[w]);
        limit = k;
        if (t == 0) put(j, k);
      }
    }
  }
  if (csize > 1) {
    cluster_arrive();
    cluster_wait();
    if (rank != 0) return;
  } else {
    __syncthreads();
  }
  // ---- the first CTA: the row's statistics
  float m, ln, W_over_S;
  {
    Stat a = lane < csize ? cta_stat[lane] : Stat{-INFINITY, 0.f, 0.f};
    m = redux_max(a.m);
    move_to(a, m, c);
#pragma unroll
    for (int o = kMaxCluster / 2; o > 0; o >>= 1) {
      a.S += __shfl_xor_sync(0xffffffffu, a.S, o);
      a.W += __shfl_xor_sync(0xffffffffu, a.W, o);
    }
    a.S = __shfl_sync(0xffffffffu, a.S, 0);
    a.W = __shfl_sync(0xffffffffu, a.W, 0);
    ln = m == -INFINITY ? __uint_as_float(0x7fc00000u) : logf(a.S);
    W_over_S = a.W * kLn2 / a.S;
  }
  if (t == 0) {
    if (entropy) entropy[row] = ln - W_over_S;
    float lp = 0.f;
    if (tok >= 0 && tok < V) {
      lp = (z_tok - m) * inv_t - ln;
    } else if (tok != -1) {
      sd_set_error(SD_DEVERR_TOKEN_RANGE);
      lp = __uint_as_float(0x7fc00000u);
    }
    logprob[row] = lp;
  }
  if (top_n == 0) return;
  // ---- its alternatives: rank by counting over the CTAs' lists
  __shared__ int n_found;
  if (t == 0) n_found = 0;
  __syncthreads();
  auto write = [&](int at, float z, int i) {
    top_ids[row * top_n + at] = i;
    top_logprobs[row * top_n + at] = (z - m) * inv_t - ln;
  };
  const int n_all = csize * top_n;
  for (int i = t; i < n_all; i += kThreads) {
    const uint64_t k = best[i];
    if (!k) continue;
    int above = 0;
#pragma unroll 8
    for (int j = 0; j < n_all; j += 2) {  // (zeros past the end)
      const ulonglong2 y = *reinterpret_cast<const ulonglong2*>(best + j);
      above += (y.x > k) + (y.y > k);
    }
    if (above < top_n) {
      write(above, value_of(static_cast<uint32_t>(k >> 32)), static_cast<int>(~static_cast<uint32_t>(k)));
      atomicAdd(&n_found, 1);
    }
  }
  __syncthreads();
  if (warp == 0 && n_found < top_n) {
    // tokens of probability 0, the lowest indices first (a row with NaN in it may have too
    // few of both: any index then)
    int at = n_found;
    for (int i0 = 0; i0 < V && at < top_n; i0 += 32) {
      const int i = i0 + lane;
      const bool is = i < V && T::load(z0, i) == -INFINITY;
      const uint32_t all = __ballot_sync(0xffffffffu, is);
      const int place = at + __popc(all & ((1u << lane) - 1));
      if (is && place < top_n) write(place, -INFINITY, i);
      at += __popc(all);
    }
    if (lane >= at && lane < top_n) write(lane, __uint_as_float(0x7fc00000u), lane);
  }
}

// CTAs a row: as many as fit at once over all rows (four an SM), as long as each keeps 32 KB
// of the row, four chunks a thread. 256 rows of 608 KB at 1 / 2 / 4 / 8: 36.5 / 32.0 / 37.8 /
// 50.1 us; 8 rows of 304 KB: 17.5 / 11.4 / 8.4 / 7.0, and no less at 16. (Two or three chunks
// in flight and five or six CTAs an SM: 37 to 40 for the first.)
int cluster_size(int rows, long long row_bytes) {
  int s = 1;
  while (s < kMaxCluster && 2LL * rows * s <= 4LL * sd_num_sms() && row_bytes / (2 * s) >= 32768) s *= 2;
  return s;
}

template <bool kBf16>
cudaError_t launch(cudaStream_t st, int S, const void* logits, int rows, long long stride, int V, const int32_t* tokens,
                   float inv_t, int top_n, float* logprob, float* entropy, int32_t* top_ids, float* top_logprobs) {
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = S;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.gridDim = dim3(S, rows);
  cfg.blockDim = dim3(kThreads);
  cfg.stream = st;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, logprobs_kernel<kBf16>, logits, stride, V, tokens, inv_t, top_n, logprob, entropy,
                            top_ids, top_logprobs);
}

}  // namespace

extern "C" sd_status sd_token_logprobs(const void* logits, sd_dtype dtype, int rows, int V, long long row_stride,
                                       const int32_t* tokens, float temperature, int top_n, float* logprob,
                                       float* entropy, int32_t* top_ids, float* top_logprobs, sd_stream_t stream) {
  if (rows < 0 || V <= 0 || row_stride < V) return SD_ERR_INVALID_ARG;
  if (dtype != SD_BF16 && dtype != SD_F32) return SD_ERR_INVALID_ARG;
  if (!(temperature > 0.f) || !isfinite(temperature) || !isfinite(1.f / temperature)) return SD_ERR_INVALID_ARG;
  if (top_n < 0 || top_n > V) return SD_ERR_INVALID_ARG;
  if (top_n > kTopMax) return SD_ERR_UNSUPPORTED;
  if (V > (1 << 30)) return SD_ERR_UNSUPPORTED;
  if (rows == 0) return SD_OK;
  if (!logits || !tokens || !logprob || (top_n > 0 && (!top_ids || !top_logprobs))) return SD_ERR_INVALID_ARG;
  const int elem = dtype == SD_BF16 ? 2 : 4;
  if (reinterpret_cast<uintptr_t>(logits) % elem) return SD_ERR_INVALID_ARG;  // (the kernel finds each row's alignment)
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  for (int r0 = 0; r0 < rows; r0 += 65535) {  // a grid's second dimension ends at 65535
    const int n = rows - r0 < 65535 ? rows - r0 : 65535;
    const int S = cluster_size(n, static_cast<long long>(V) * elem);
    const char* z = static_cast<const char*>(logits) + static_cast<long long>(r0) * row_stride * elem;
    const long long o = static_cast<long long>(r0) * top_n;
    const cudaError_t e = (dtype == SD_BF16 ? launch<true> : launch<false>)(
        st, S, z, n, row_stride, V, tokens + r0, 1.f / temperature, top_n, logprob + r0, entropy ? entropy + r0 : nullptr,
        top_ids ? top_ids + o : nullptr, top_logprobs ? top_logprobs + o : nullptr);
    if (e != cudaSuccess) {
      (void)cudaGetLastError();
      return SD_ERR_CUDA;
    }
  }
  return SD_OK;
}
