// Verify attention over the 8-bit KV cache on the 5th-generation tensor cores (sm_103a):
// the rows, masks and results of the bf16 verify attention, with key n = k_code[n] *
// k_scale[n / block] and value n = v_code[n] * v_scale[n / block].
//
// The codes go from HBM to the tensor cores as they are (kind::f8f6f4, e4m3 by e4m3, fp32
// sums): nothing widens a key or a value. What meets them has 8 significant bits and an
// e4m3 number 4, so queries and weights go in as two terms each, the second what rounding
// the first left over:
//   * the query rows, scaled by the power of two that brings their largest element into
//     [128, 256), are exact in two terms (bf16 has 8 bits; elements below 2^-10 of the
//     largest to 2^-18 of it), both products into the same sum;
//   * a weight is hi + lo / 16, hi = e4m3(P), lo = e4m3(16 (P - hi) + dither): 8 bits, as a
//     bf16 one would keep, down to P = 2^-5; below, the terms are subnormal and end at steps
//     of 2^-13. A long tail of weights that small may hold much of a row beside a few large
//     keys, and rounded to nearest, all alike, it would be lost or grow (a row with 0.8 of it
//     in one key of 16384 at P = 2^2: a tenth of the output). So a reference lets what stands
//     out stand high (below), and the dither, half a step at most and made of the key's
//     index, spreads the rounding: of equal weights a share of the keys rounds up that makes
//     their sum right. The terms are columns of one product, 2 kR wide (four of N = 2 kR
//     take 200 cycles at kR = 32, eight of N = kR 330).
// The packed query rows of a KV head (G * R) are few, so both products run transposed,
//     S^T[128 keys][kR rows] = K_tile . Q^T,   O^T[128 d][2 kR] += V_tile^T . P^T
// with kR = 32 or 48 and, above 48 rows, two or three m-blocks. Scales enter between the two: a
// thread has one key, t = S * k_scale * c, and
//     P = 2^(t * qscale + log2 v_scale - ref[row]),   l[row] += P / v_scale,
// so O / l is the attention whatever the scales are.
//
// Reference. P has to stay within e4m3's 448, and a row's largest weights far above 2^-13.
// ref[row] is the least number that gives the largest weight of the first tile no more than
// 2^8 and the lowest of the four largest of each 32 of its keys no more than 2^1: what
// stands out has up to 2^8, and rows of many alike, among which a later one may be larger,
// have room for it. It moves by the same rule when a later weight would pass 2^8.75. A row's
// weights then sum to 2^8 or more, or at the least to 2^3 (four keys alike), and a small one
// is off by less than 2^-13 in these units, at random. (By the largest weight alone: at 2^2
// the tail's error is 16 to 60 times this, at 2^6 the moves take 32 scenes from 103 to 116
// us, at 2^4 they take 104 with ten times the error.) Every thread compares its largest
// exponent and the group votes once a tile (an OR in its barrier). Moving takes the tile's
// exact row maxima over 32 keys (redux over the lanes), and rescales l and O in tensor memory.
//
// Warps (608 threads): 0 the TMA producer; 1 issues S and owns tensor memory; 2 issues
// PV; 3..18 two softmax groups of eight, which take alternate tiles. The groups are two
// independent softmaxes (own references, own O in tensor memory, own P buffer), joined
// at the end: neither waits for the other's references. One cluster per (scene, KV head,
// m-block); its CTAs take contiguous ranges of the keys and merge their partials through
// distributed shared memory. Where clusters fill the SMs badly (256 heads on 152 SMs: 1.7
// CTAs an SM take the time of two) and the caller gives a workspace, every SM takes an even
// share of the tiles of all units instead, and a second kernel joins what the shares' borders
// cut.
//
// What bounds it. 32 scenes of 6200 to 8192 keys, 8 heads, 36 rows: 103 us, 489 MB at
// 0.70 of the measured copy rate. The softmax: a tile takes an SM 1.6 thousand cycles, 16
// warps and 96 registers a thread (8 to 56 B of stores spilled); without its arithmetic
// 82 us (of the 112 of whole clusters), without the vote 101, without the conversions to two
// terms besides 92, and with every key from L2 still 111. One scene of 4096 keys (8 heads, 32
// rows: 8.1 us; 4 heads of one row each: 6.6) the chain of latencies: lengths, rows and keys,
// S, references, P, PV, merge.
#include "shares.cuh"
#include "tc_common.cuh"

#include <math.h>

#include <algorithm>
#include <atomic>

SD_DEFINE_ERROR_ACCESSOR(sd_take_error_attention_kv8)

namespace {

constexpr int kTile = 128;               // keys a tile
constexpr int kStages = 4;               // K slots, V slots and S buffers
constexpr int kFirstSoft = 3;            // the first softmax warp
constexpr int kSoft0 = 32 * kFirstSoft;
constexpr float kTop = 8.f;              // log2 of the largest weight that a reference gives the tile that sets it,
constexpr float kLow = 1.f;              // and of the lowest of the four largest of each 32 keys
constexpr float kHot = 8.75f;            // log2 of the largest weight a reference may leave (e4m3 ends at 448 = 2^8.81)

struct Args {
  const __nv_bfloat16* q;
  __nv_bfloat16* out;
  const float* ks;
  const float* vs;
  const int32_t* len;
  int R, Hq, Hkv, G, M, cap, nblk, block_shift, mblocks;
  int block_mask;
  float inv_g;       // 1 / G: p / G == int((p + 0.5) / G) exactly for the p < 128 used here
  float scale_log2;
  int B;             // even shares
  float* part;       // two partial tiles of rows a CTA
};

template <int kR, int kDim>
struct Cfg {
  static_assert(kR == 32 || kR == 48, "row tile");
  static_assert(kDim == 64 || kDim == 128, "head dim");
  // a softmax thread has one key and kUnits units of 8 rows: of its half every second one
  static constexpr int kUnits = kR / 16;
  static constexpr int kSoftWarps = 16;
  static constexpr int kSoftThreads = 32 * kSoftWarps;
  static constexpr int kGroupThreads = kSoftThreads / 2;
  static constexpr int kThreads = kSoft0 + kSoftThreads;
  static constexpr int kKV = kTile * kDim;        // one K (or V) tile
  static constexpr int kRingV = kStages * kKV;
  static constexpr int kRing = 2 * kStages * kKV;
  static constexpr int kQ = kR * kDim;            // one term of the query rows
  // P^T: 2 kR rows (hi, then lo), MN-major, 32-byte swizzle: 32 rows x 8 keys an atom; the
  // 32-row groups kPGroup apart
  static constexpr int kPGroup = kTile * 32;
  static constexpr int kP = 2 * kR / 32 * kPGroup;  // a group's weights
  static constexpr int kOffQ = kRing;             // hi, lo
  static constexpr int kOffP = kOffQ + 2 * kQ;    // [group]
  static constexpr int kOffBar = kOffP + 2 * kP;
  // full_k[4] full_v[4] s_ready[4] s_free[4] pv_done[4] p_full[2] recv tmem_done q_full
  static constexpr int kNumBars = 5 * kStages + 5;
  static constexpr int kOffMisc = round_up(kOffBar + kNumBars * 8, 16);
  static constexpr int kOffExp = kOffMisc + 16;             // [kR] exponents of the query rows
  static constexpr int kOffQs = kOffExp + kR * 4;           // [kR] scales of the query rows over the tile's
  static constexpr int kOffNref = kOffQs + kR * 4;          // [group][kR] negated references
  static constexpr int kOffRef = kOffNref + 2 * kR * 4;     // [group][kR] references
  static constexpr int kOffFac = kOffRef + 2 * kR * 4;      // [group][kR] rescale factors
  static constexpr int kOffMax = kOffFac + 2 * kR * 4;      // [group][4 lane quarters][kR] tile maxima
  static constexpr int kOffSum = kOffMax + 8 * kR * 4;      // [kR][8] row sums by group and lane quarter
  static constexpr int kOffJoin = kOffSum + kR * 32;        // [kR] {weight of O_0, of O_1, 1 / l or l, ref}
  static constexpr int kOffWalk = kOffJoin + kR * 16;       // even shares: the softmax warps' walk and run
  static constexpr int kSmemBytes = kOffWalk + 64 + 1024;
  static_assert(kSmemBytes <= 227 * 1024, "shared memory budget");
  static_assert(kOffQ % 1024 == 0 && kOffP % 1024 == 0, "swizzle atoms");
  static constexpr int kTmemO = 4 * kR;                     // S0..S3 | O_0 hi, lo | O_1 hi, lo
  static constexpr int kTmemCols = kR == 32 ? 256 : 512;
  static constexpr uint64_t kLayout = kDim == 128 ? 2 : 4;  // swizzle of K, V and Q rows: their whole width
  // a partial row sent to its owner: [O(kDim) | l | ref | 2 pad] fp32
  static constexpr int kRowF = kDim + 4;
  static constexpr int kRowBytes = kRowF * 4;
  // incoming rows in the K ring, this CTA's in the V ring; ceil(n / c) * c < n + 16
  static_assert((kR + 15) * kRowBytes <= kRingV && kR * kRowBytes <= kRingV, "merge buffers");
};

// kind::f8f6f4: fp32 sums, A and B e4m3
constexpr uint32_t idesc8(int M, int N, int a_mn_major, int b_mn_major) {
  return (1u << 4) | (static_cast<uint32_t>(a_mn_major) << 15) | (static_cast<uint32_t>(b_mn_major) << 16) |
         (static_cast<uint32_t>(N >> 3) << 17) | (static_cast<uint32_t>(M >> 4) << 24);
}
__device__ __forceinline__ void umma8(uint32_t d_tmem, uint64_t a, uint64_t b, uint32_t idesc, int accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}" ::"r"(d_tmem),
      "l"(a), "l"(b), "r"(idesc), "r"(accumulate)
      : "memory");
}
// fp32 columns of this warp's 32 TMEM lanes to and from registers; a load's registers
// hold them after tmem_wait_ld
__device__ __forceinline__ void tmem_ld4(uint32_t taddr, float* r) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x4.b32 {%0,%1,%2,%3}, [%4];"
               : "=f"(r[0]), "=f"(r[1]), "=f"(r[2]), "=f"(r[3])
               : "r"(taddr)
               : "memory");
}
__device__ __forceinline__ void tmem_ld8(uint32_t taddr, float* r) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
               : "=f"(r[0]), "=f"(r[1]), "=f"(r[2]), "=f"(r[3]), "=f"(r[4]), "=f"(r[5]), "=f"(r[6]), "=f"(r[7])
               : "r"(taddr)
               : "memory");
}
template <int kN>
__device__ __forceinline__ void tmem_wait_ld(float* r) {
  asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
  for (int j = 0; j < kN; j += 8)  // no use of the registers moves above the wait
    asm volatile("" : "+f"(r[j]), "+f"(r[j + 1]), "+f"(r[j + 2]), "+f"(r[j + 3]), "+f"(r[j + 4]), "+f"(r[j + 5]),
                 "+f"(r[j + 6]), "+f"(r[j + 7]));
}
__device__ __forceinline__ void tmem_st8(uint32_t taddr, const float* r) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%8], {%0,%1,%2,%3,%4,%5,%6,%7};" ::"f"(r[0]), "f"(r[1]), "f"(r[2]),
               "f"(r[3]), "f"(r[4]), "f"(r[5]), "f"(r[6]), "f"(r[7]), "r"(taddr)
               : "memory");
}
__device__ __forceinline__ uint64_t pack2f(float lo, float hi) {
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
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
  uint64_t d;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
  uint64_t d;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}
__device__ __forceinline__ float warp_max(float x) {
  float r;
  asm("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(x));
  return r;
}
__device__ __forceinline__ float lg2(float x) {
  float y;
  asm("lg2.approx.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// Two numbers of magnitude up to 448 as two e4m3 terms each, x = hi + lo / kLo (by way of
// fp16, whose 11 bits both terms together do not reach): codes in the low 16 bits. `dither`
// (two fp16 numbers) is added to lo before its rounding.
template <int kLo>
__device__ __forceinline__ void two_terms(float x0, float x1, uint32_t dither, uint32_t& hi, uint32_t& lo) {
  static_assert(kLo == 1 || kLo == 16, "as fp16 below");
  asm("{\n\t.reg .b32 f, b, d;\n\t.reg .b16 h, l;\n\t"
      "cvt.rn.f16x2.f32 f, %3, %2;\n\t"
      "cvt.rn.satfinite.e4m3x2.f16x2 h, f;\n\t"
      "cvt.rn.f16x2.e4m3x2 b, h;\n\t"
      "sub.f16x2 d, f, b;\n\t"
      "fma.rn.f16x2 d, d, %4, %5;\n\t"
      "cvt.rn.satfinite.e4m3x2.f16x2 l, d;\n\t"
      "cvt.u32.u16 %0, h;\n\tcvt.u32.u16 %1, l;\n\t}"
      : "=r"(hi), "=r"(lo)
      : "f"(x0), "f"(x1), "r"(kLo == 1 ? 0x3c003c00u : 0x4c004c00u), "r"(dither));
}
// Half an e4m3 step of subnormal numbers, 2^-10, times a number in [-1, 1) that is spread
// evenly over any run of keys, and over every second, third, ... of them (the multiples of
// the golden ratio); twice, as fp16.
__device__ __forceinline__ uint32_t dither_of(int key) {
  const float x = static_cast<float>(static_cast<int>(static_cast<uint32_t>(key) * 0x9e3779b9u)) * 0x1p-41f;
  uint32_t d;
  asm("cvt.rn.f16x2.f32 %0, %1, %1;" : "=r"(d) : "f"(x));
  return d;
}

__device__ __forceinline__ float rcp(float x) {
  float y;
  asm("rcp.approx.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// Sum over the 32 lanes of a warp of each of 8 per-lane values: lane L ends with the sum
// of value (L >> 2).
__device__ __forceinline__ float warp_sum8(float (&v)[8], int lane) {
#pragma unroll
  for (int n = 8, s = 16; n > 1; n >>= 1, s >>= 1) {
    const bool hi = (lane & s) != 0;
#pragma unroll
    for (int i = 0; i < n / 2; ++i) {
      const float keep = hi ? v[i + n / 2] : v[i];
      const float give = hi ? v[i] : v[i + n / 2];
      v[i] = keep + __shfl_xor_sync(0xffffffffu, give, s);
    }
  }
  float x = v[0];
  x += __shfl_xor_sync(0xffffffffu, x, 2);
  x += __shfl_xor_sync(0xffffffffu, x, 1);
  return x;
}

// A run of one unit's keys that a CTA takes.
struct Run {
  int b, kvh, mblock, n_keys, key_begin, key_end, n_tiles;
  bool whole;  // all the unit's tiles
};
// Even shares: units are (KV head, m-block).
__device__ __forceinline__ Scenes scenes_of(const Args& a) { return Scenes{a.len, nullptr, a.B, a.R, a.cap, a.Hkv * a.mblocks}; }
__device__ __forceinline__ Run take(Walk<false>& walk, const Args& a) {
  const Span s = walk.next(scenes_of(a));
  const int kvh = s.unit / a.mblocks;
  return Run{s.b, kvh, s.unit - kvh * a.mblocks, s.n_keys, s.key_begin, s.key_end, s.n_tiles, s.whole};
}

// ------------------------------------------------------------------ kernel
// kEven false: grid (cluster size, Hkv * m-blocks, B), the m-blocks of a head side by side.
// kEven true: grid (CTAs), no clusters; a CTA's runs one after the other, the producer ahead
// of the rest across their borders, and what is not a whole unit goes to a.part, for
// kv8_join_kernel. m-block mb takes packed rows mb * kR .. mb * kR + kR - 1 (packed row
// p = i * G + g: new row i, query head g of the group).
template <int kR, int kDim, bool kEven>
__global__ void __launch_bounds__(Cfg<kR, kDim>::kThreads, 1)
    kv8_attention_kernel(const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v, const Args a) {
  using C = Cfg<kR, kDim>;
  constexpr int kUnits = C::kUnits, kSoftWarps = C::kSoftWarps, kSoftThreads = C::kSoftThreads;
  constexpr int kGroupThreads = C::kGroupThreads, kKV = C::kKV, kRowF = C::kRowF, kRowBytes = C::kRowBytes;
  constexpr uint32_t kIdescS = idesc8(128, kR, 0, 0);
  constexpr uint32_t kIdescO = idesc8(128, 2 * kR, 1, 1);
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
  const uint32_t base = smem_addr(smem);
  auto bar = [&](int i) { return base + C::kOffBar + 8u * i; };
  // A wait names a phase by its parity: the phase before has completed by then, and the
  // next one cannot complete before the waiter has looked. Slot and buffer of tile T are
  // T % 4, so their next phase is tile T + 4, of the same group: K(T + 4) waits for S(T),
  // V(T + 4) for PV(T), S(T + 4) for the group's reading of S(T), P(T + 2) for PV(T). T
  // counts the CTA's tiles over its runs.
  auto FULLK = [&](int T) { return bar(T % kStages); };
  auto FULLV = [&](int T) { return bar(kStages + T % kStages); };
  auto SREADY = [&](int T) { return bar(2 * kStages + T % kStages); };
  auto SFREE = [&](int T) { return bar(3 * kStages + T % kStages); };
  auto PVDONE = [&](int T) { return bar(4 * kStages + T % kStages); };
  auto PFULL = [&](int T) { return bar(5 * kStages + (T & 1)); };
  const uint32_t RECV = bar(5 * kStages + 2);
  const uint32_t TMEMDONE = bar(5 * kStages + 3);
  const uint32_t QFULL = bar(5 * kStages + 4);
  auto par = [](int T) { return static_cast<uint32_t>((T / kStages) & 1); };
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(smem + C::kOffMisc);
  int* row_exp = reinterpret_cast<int*>(smem + C::kOffExp);
  float* row_nref = reinterpret_cast<float*>(smem + C::kOffNref);
  float* row_qs = reinterpret_cast<float*>(smem + C::kOffQs);
  float* row_ref = reinterpret_cast<float*>(smem + C::kOffRef);
  float* row_fac = reinterpret_cast<float*>(smem + C::kOffFac);
  float* row_max = reinterpret_cast<float*>(smem + C::kOffMax);
  float* row_sum = reinterpret_cast<float*>(smem + C::kOffSum);
  float4* row_join = reinterpret_cast<float4*>(smem + C::kOffJoin);

  auto gdiv = [&](int p) { return __float2int_rz((static_cast<float>(p) + 0.5f) * a.inv_g); };
  const int rank = kEven ? 0 : blockIdx.x, csize = kEven ? 1 : gridDim.x;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

  if (warp == 0 && lane == 0) {
    for (int s = 0; s < kStages; ++s) {
      mbar_init(FULLK(s), 1);
      mbar_init(FULLV(s), 1);
      mbar_init(SREADY(s), 1);
      mbar_init(SFREE(s), kSoftWarps / 2);
      mbar_init(PVDONE(s), 1);
    }
    mbar_init(PFULL(0), kSoftWarps / 2);
    mbar_init(PFULL(1), kSoftWarps / 2);
    mbar_init(RECV, 1);
    mbar_init(TMEMDONE, kSoftWarps);
    if (kEven) mbar_init(QFULL, kSoftWarps);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  __syncwarp();
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(tmem_slot)),
                 "r"(C::kTmemCols)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  // this CTA's runs: of its cluster's unit the rank's share of the keys, in blocks of 32, or
  // those of its share of all tiles
  Walk<false> walk = {};
  Run one = {};
  bool valid = true;
  if constexpr (!kEven) {
    one.b = blockIdx.z;
    one.kvh = blockIdx.y / a.mblocks;
    one.mblock = blockIdx.y - one.kvh * a.mblocks;
  }
  griddep_wait();  // nothing before this touches global memory
  if constexpr (kEven) {
    walk.begin(scenes_of(a), shares_of(scenes_of(a), lane, gridDim.x), lane);
  } else {
    one.n_keys = __ldcg(a.len + one.b);
    valid = one.n_keys >= a.R && one.n_keys <= a.cap;
    const int nblk32 = valid ? (one.n_keys + 31) / 32 : 0;
    const int blk_begin = static_cast<int>(static_cast<long long>(rank) * nblk32 / csize);
    const int blk_end = static_cast<int>(static_cast<long long>(rank + 1) * nblk32 / csize);
    one.key_begin = blk_begin * 32;
    one.key_end = min(blk_end * 32, valid ? one.n_keys : 0);
    one.n_tiles = (blk_end - blk_begin + 3) / 4;
  }
  auto more = [&](int n_run) {
    if constexpr (kEven) return walk.left > 0;
    else return n_run == 0;
  };
  auto next_run = [&] {
    if constexpr (kEven) return take(walk, a);
    else return one;
  };

  if (warp == 0) {
    // -------------------------------------------------------------- producer
    if constexpr (kEven) {
      if (blockIdx.x == 0)
        for (int b = lane; b < a.B; b += 32)
          if (keys_of(scenes_of(a), b) == 0) sd_set_error(SD_DEVERR_LENGTH);
      tc_fence_before();
      __syncthreads();
      tc_fence_after();
    } else if (!valid && rank == 0 && lane == 0 && blockIdx.y == 0) {
      sd_set_error(SD_DEVERR_LENGTH);
    }
    const uint64_t policy = l2_evict_first_policy();
    // a whole box even for a short last tile: keys past the range are masked, rows past
    // the capacity arrive zero-filled
    auto issue_k = [&](int T, int key, int z) {
      if (T >= kStages) mbar_wait(SREADY(T), par(T - kStages));
      if (elect_one()) {
        mbar_expect_tx(FULLK(T), static_cast<uint32_t>(kKV));
        tma_load_3d_hint(base + (T % kStages) * kKV, &tm_k, FULLK(T), 0, key, z, policy);
      }
      __syncwarp();
    };
    auto issue_v = [&](int T, int key, int z) {
      if (T >= kStages) mbar_wait(PVDONE(T), par(T - kStages));
      if (elect_one()) {
        mbar_expect_tx(FULLV(T), static_cast<uint32_t>(kKV));
        tma_load_3d_hint(base + C::kRingV + (T % kStages) * kKV, &tm_v, FULLV(T), 0, key, z, policy);
      }
      __syncwarp();
    };
    if constexpr (kEven) {
      int T = 0, key_v = 0, z_v = 0;
#pragma unroll 1
      while (walk.left > 0) {
        const Run r = take(walk, a);
        const int z = r.b * a.Hkv + r.kvh;
#pragma unroll 1
        for (int t = 0; t < r.n_tiles; ++t, ++T) {
          issue_k(T, r.key_begin + t * kTile, z);
          if (T > kStages) issue_v(T - 1, key_v, z_v);
          key_v = r.key_begin + t * kTile;
          z_v = z;
          if (T < kStages) issue_v(T, key_v, z_v);
        }
      }
      if (T > kStages) issue_v(T - 1, key_v, z_v);
    } else {
      const int z = one.b * a.Hkv + one.kvh, n0 = min(one.n_tiles, kStages);
#pragma unroll 1
      for (int T = 0; T < n0; ++T) {
        issue_k(T, one.key_begin + T * kTile, z);
        issue_v(T, one.key_begin + T * kTile, z);
      }
      tc_fence_before();
      __syncthreads();
      tc_fence_after();
      // past the ring the keys go one tile ahead of the values: their slot is free earlier
#pragma unroll 1
      for (int T = n0; T <= one.n_tiles; ++T) {
        if (T < one.n_tiles) issue_k(T, one.key_begin + T * kTile, z);
        if (T > n0) issue_v(T - 1, one.key_begin + (T - 1) * kTile, z);
      }
    }
    if (csize > 1) {
      cluster_arrive_relaxed();
      cluster_wait();
    }
  } else if (warp == 1) {
    // -------------------------------------------------------------- S issue
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *tmem_slot;
    const uint64_t dK0 = umma_desc(base, 16, kDim * 8, C::kLayout);
    const uint64_t dQ = umma_desc(base + C::kOffQ, 16, kDim * 8, C::kLayout);
    int T = 0;
#pragma unroll 1
    for (int n_run = 0; more(n_run); ++n_run) {
      const Run r = next_run();
      if (kEven) mbar_wait(QFULL, n_run & 1);
#pragma unroll 1
      for (int t = 0; t < r.n_tiles; ++t, ++T) {
        if (T >= kStages) mbar_wait(SFREE(T), par(T - kStages));
        mbar_wait(FULLK(T), par(T));
        tc_fence_after();
        const uint32_t ts = tmem + kR * (T % kStages);
        const uint64_t dk = dK0 + static_cast<uint64_t>(((T % kStages) * kKV) >> 4);
        if (elect_one()) {
#pragma unroll
          for (int term = 0; term < 2; ++term)
#pragma unroll
            for (int kk = 0; kk < kDim / 32; ++kk)
              umma8(ts, dk + (kk * 32 >> 4), dQ + ((term * C::kQ + kk * 32) >> 4), kIdescS, term + kk > 0 ? 1 : 0);
          umma_commit(SREADY(T));
        }
        __syncwarp();
      }
    }
    if (csize > 1) cluster_arrive_relaxed();
    mbar_wait(TMEMDONE, 0);  // every softmax warp has read its last column
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(C::kTmemCols) : "memory");
    if (csize > 1) cluster_wait();
  } else if (warp == 2) {
    // -------------------------------------------------------------- PV issue
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem_o = *tmem_slot + C::kTmemO;
    // V^T: MN-major. Head dim 64 keeps M = 128 with both 64-row halves of the operand on
    // the same rows (stride 0): O's lanes 64..127 repeat 0..63 and are not read
    const uint64_t dV0 = umma_desc(base + C::kRingV, 0, kDim * 8, C::kLayout);
    const uint64_t dP0 = umma_desc(base + C::kOffP, C::kPGroup, 256, 6);  // MN-major, 32-byte swizzle
    int T = 0;
#pragma unroll 1
    for (int n_run = 0; more(n_run); ++n_run) {
      const Run r = next_run();
#pragma unroll 1
      for (int t = 0; t < r.n_tiles; ++t, ++T) {
        mbar_wait(PFULL(T), (T >> 1) & 1);
        mbar_wait(FULLV(T), par(T));
        tc_fence_after();
        const uint64_t dv = dV0 + static_cast<uint64_t>(((T % kStages) * kKV) >> 4);
        const uint64_t dp = dP0 + static_cast<uint64_t>(((T & 1) * C::kP) >> 4);
        const uint32_t to = tmem_o + 2 * kR * (T & 1);
        const int n_steps = (min(kTile, r.key_end - r.key_begin - t * kTile) + 31) >> 5;
        if (elect_one()) {
#pragma unroll
          for (int kk = 0; kk < kTile / 32; ++kk)
            if (kk < n_steps)
              umma8(to, dv + (kk * 32 * kDim >> 4), dp + (kk * 1024 >> 4), kIdescO, t > 1 || kk > 0 ? 1 : 0);
          umma_commit(PVDONE(T));
        }
        __syncwarp();
      }
    }
    if (csize > 1) {
      cluster_arrive_relaxed();
      cluster_wait();
    }
  } else {
    // -------------------------------------------------------------- softmax
    const int st = static_cast<int>(threadIdx.x) - kSoft0;  // 0 .. 511
    const int sw = warp - kFirstSoft;
    const int group = sw >> 3;
    const int gt = st - group * kGroupThreads;
    const int half = gt >> 7;            // this warp has the 8-row units half, half + 2, ...
    const int quarter = warp & 3;        // TMEM lane quarter of this warp
    const int kl = quarter * 32 + lane;  // key lane of S^T / d lane of O^T
    const uint32_t lane_off = static_cast<uint32_t>(quarter * 32) << 16;
    if constexpr (kEven) {
      if (st == 0) *reinterpret_cast<Walk<false>*>(smem + C::kOffWalk) = walk;
      tc_fence_before();
      __syncthreads();
      tc_fence_after();
    }
    // (the walk and the run stand in shared memory: in registers they are spilled, and the
    // tile loop with them)
    Walk<false>* const my_walk = reinterpret_cast<Walk<false>*>(smem + C::kOffWalk);
    Run* const my_run = reinterpret_cast<Run*>(smem + C::kOffWalk + 32);
    static_assert(sizeof(*my_walk) <= 32 && sizeof(Run) <= 32, "shared memory layout");
    int T0 = 0;  // tiles before this run
#pragma unroll 1
    for (int n_run = 0; kEven ? my_walk->left > 0 : n_run == 0; ++n_run) {
      Run r = one;
      if constexpr (kEven) {
        walk = *my_walk;
        r = take(walk, a);
      }
      const int b = r.b, n_keys = r.n_keys, key_begin = r.key_begin, key_end = r.key_end, n_tiles = r.n_tiles;
      const int kvh = r.kvh, mblock = r.mblock;
      const int rows_in = max(1, min(kR, a.M - mblock * kR));
      // this warp's units that hold a row: it leaves the others out (their P stays stale and
      // reaches only O columns that are not read)
      const int n_units = ((rows_in + 7) / 8 - half + 1) / 2;
      auto q_off = [&](int b, int kvh, int p) {
        const int i = gdiv(p);
        return ((static_cast<long long>(b) * a.R + i) * a.Hq + kvh * a.G + (p - i * a.G)) * kDim;
      };
      // ---- the query rows as two terms (rows past M zero), a 16-byte chunk a thread
      constexpr int kChunks = kDim / 8;
      constexpr int kQc = (kR * kChunks + kSoftThreads - 1) / kSoftThreads;
      uint4 qv[kQc];
#pragma unroll
      for (int u = 0; u < kQc; ++u) {
        const int idx = st + u * kSoftThreads, p = mblock * kR + idx / kChunks;
        qv[u] = idx < kR * kChunks && p < a.M ? __ldcg(reinterpret_cast<const uint4*>(a.q + q_off(b, kvh, p) + (idx % kChunks) * 8))
                                              : make_uint4(0, 0, 0, 0);
      }
      if (n_run == 0 && st == 0) griddep_launch();  // every older kernel has finished: the next may launch
      // One scale for the tile's rows, 2^(e - 7) with 2^e its largest element's power: a score
      // then needs no factor of its own row (read from shared memory for every score, the
      // rows' factors and references took all its bandwidth). A row more than 2^6 below the
      // tile's largest would lose bits that way: it keeps its own scale, row_qs, and the
      // tile takes a slower form.
      int em[kQc];
#pragma unroll
      for (int u = 0; u < kQc; ++u) {
        const int idx = st + u * kSoftThreads;
        const uint32_t w[4] = {qv[u].x, qv[u].y, qv[u].z, qv[u].w};
        uint32_t m = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) m = max(m, max(w[j] & 0x7fffu, (w[j] >> 16) & 0x7fffu));
#pragma unroll
        for (int x = kChunks / 2; x > 0; x >>= 1) m = max(m, __shfl_xor_sync(0xffffffffu, m, x));
        // (2^-119 at least: its inverse is a number; 255: infinities or NaN in the row)
        em[u] = m >= 0x7f80u ? 255 : max(static_cast<int>(m >> 7), 8);
        if (idx < kR * kChunks && idx % kChunks == 0) row_exp[idx / kChunks] = em[u];
      }
      named_bar_sync(2, kSoftThreads);
      if (kEven && st == 0) {
        *my_walk = walk;
        *my_run = r;
      }
      int e_tile;
      bool small_rows;
      {
        int x0 = row_exp[lane], x1 = lane < kR - 32 ? row_exp[32 + lane] : 8;
        small_rows = __any_sync(0xffffffffu, max(x0, x1) == 255);
        x0 = x0 == 255 ? 8 : x0;
        x1 = x1 == 255 ? 8 : x1;
        e_tile = __reduce_max_sync(0xffffffffu, max(x0, x1));
        small_rows |= __any_sync(0xffffffffu, (x0 > 8 && x0 < e_tile - 6) || (x1 > 8 && x1 < e_tile - 6));
      }
#pragma unroll
      for (int u = 0; u < kQc; ++u) {
        const int idx = st + u * kSoftThreads, row = idx / kChunks, c = idx % kChunks;
        if (idx >= kR * kChunks) break;  // warp-uniform
        const uint32_t w[4] = {qv[u].x, qv[u].y, qv[u].z, qv[u].w};
        // (rows of zeros, those past M among them, take the tile's scale)
        const int e = em[u] > 8 && em[u] < e_tile - 6 ? em[u] : e_tile;
        const float inv = __uint_as_float(static_cast<uint32_t>(min(261 - e, 254)) << 23);
        uint32_t hi[4], lo[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) two_terms<1>(sd_bf16_lo(w[j]) * inv, sd_bf16_hi(w[j]) * inv, 0u, hi[j], lo[j]);
        // the swizzle moves 16-byte chunks: of 8 rows of 128 bytes, or of 4 pairs of rows of 64
        const uint32_t sw16 = kDim == 128 ? ((c >> 1) ^ (row & 7)) : ((c >> 1) ^ ((row >> 1) & 3));
        const uint32_t dst = base + C::kOffQ + row * kDim + (sw16 << 4) + (c & 1) * 8;
        asm volatile("st.shared.v2.u32 [%0], {%1, %2};" ::"r"(dst), "r"(hi[0] | (hi[1] << 16)), "r"(hi[2] | (hi[3] << 16)) : "memory");
        asm volatile("st.shared.v2.u32 [%0], {%1, %2};" ::"r"(dst + C::kQ), "r"(lo[0] | (lo[1] << 16)), "r"(lo[2] | (lo[3] << 16))
                     : "memory");
        if (c == 0) {
          // a row with infinities or NaN in it has no attention: NaN throughout
          row_qs[row] = em[u] == 255 ? __uint_as_float(0x7fc00000u)
                                     : __uint_as_float(static_cast<uint32_t>(max(127 + e - e_tile, 1)) << 23);
          row_nref[row] = row_nref[kR + row] = INFINITY;
          row_ref[row] = row_ref[kR + row] = -INFINITY;  // no reference yet: any key's weight passes every bound
        }
      }
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      if constexpr (kEven) {
        named_bar_sync(2, kSoftThreads);  // the rows' scales and references
        if (lane == 0) mbar_arrive(QFULL);
      } else {
        tc_fence_before();
        __syncthreads();
        tc_fence_after();
      }
      const uint32_t tmem = *tmem_slot;

      // ---- this group's tiles
      const float c_log2 = a.scale_log2 * __uint_as_float(static_cast<uint32_t>(max(e_tile - 7, 1)) << 23);
      uint64_t lp2[kUnits][4];  // this key lane's row sums, in pairs
      const float* nref = row_nref + group * kR + half * 8;  // unit u: + 16 u
#pragma unroll
      for (int u = 0; u < kUnits; ++u)
#pragma unroll
        for (int j = 0; j < 4; ++j) lp2[u][j] = 0ull;
      const uint32_t pkey = base + C::kOffP + group * C::kP + kl * 32;
      const uint32_t psw = (kl >> 2) & 1;  // 32-byte swizzle
      const long long plane = static_cast<long long>(b) * a.Hkv + kvh;
      const float* ks = a.ks + plane * a.nblk;
      const float* vs = a.vs + plane * a.nblk;
      // rows below which a key is masked (causal: new row i sees new keys 0..i; kR: all)
      auto first_row = [&](int key) {
        if (key >= key_end) return kR;
        const int i = key - (n_keys - a.R);
        return a.block_mask || i <= 0 ? 0 : min(kR, max(0, i * a.G - mblock * kR));
      };
      float ks_next = 0.f, vs_next = 1.f;
      auto load_scales = [&](int t) {
        const int key = key_begin + t * kTile + kl;
        if (t < n_tiles && key < key_end) {
          ks_next = __ldcg(ks + (key >> a.block_shift));
          vs_next = __ldcg(vs + (key >> a.block_shift));
        }
      };
      const int t_first = (group ^ T0) & 1;
      load_scales(t_first);
#pragma unroll 1
      for (int t = t_first; t < n_tiles; t += 2) {
        const int T = T0 + t, tile0 = key_begin + t * kTile;
        const float kc = ks_next * c_log2, lv = lg2(vs_next), iv = rcp(vs_next);
        load_scales(t + 2);
        // whether a key of the tile is masked for some row
        const bool masks = tile0 + kTile > min(key_end, a.block_mask ? key_end : n_keys - a.R + 1);
        const uint64_t kc2 = pack2f(kc, kc), lv2 = pack2f(lv, lv), iv2 = pack2f(iv, iv);
        const uint32_t ts = tmem + kR * (T % kStages) + half * 8 + lane_off;  // unit u: + 16 u
        mbar_wait(SREADY(T), par(T));
        tc_fence_after();
        float y[kUnits][8];
        // y = log2 of the weights of this thread's key under the present references (raw:
        // without them); the largest
        auto exponents = [&](bool raw) {
#pragma unroll
          for (int u = 0; u < kUnits; ++u)
            if (u < n_units) tmem_ld8(ts + 16 * u, y[u]);
          tmem_wait_ld<8 * kUnits>(&y[0][0]);
          if (__builtin_expect(small_rows, 0)) {
#pragma unroll
            for (int u = 0; u < kUnits; ++u)
#pragma unroll
              for (int j = 0; j < 8; ++j) y[u][j] *= row_qs[16 * u + half * 8 + j];
          }
          float m = -INFINITY;
#pragma unroll
          for (int u = 0; u < kUnits; ++u)
            if (u < n_units) {
#pragma unroll
              for (int j = 0; j < 8; j += 4) {
                const float4 nr = *reinterpret_cast<const float4*>(nref + 16 * u + j);
                const uint64_t a0 = raw ? lv2 : add2(lv2, pack2f(nr.x, nr.y)), a1 = raw ? lv2 : add2(lv2, pack2f(nr.z, nr.w));
                unpack2(fma2(pack2f(y[u][j], y[u][j + 1]), kc2, a0), y[u][j], y[u][j + 1]);
                unpack2(fma2(pack2f(y[u][j + 2], y[u][j + 3]), kc2, a1), y[u][j + 2], y[u][j + 3]);
              }
              if (masks) {  // whatever the score, NaN included
                const int below = first_row(tile0 + kl) - 16 * u - half * 8;
#pragma unroll
                for (int j = 0; j < 8; ++j)
                  if (j < below) y[u][j] = -INFINITY;
              }
              m = fmaxf(m, fmaxf(fmaxf(fmaxf(y[u][0], y[u][1]), fmaxf(y[u][2], y[u][3])),
                                 fmaxf(fmaxf(y[u][4], y[u][5]), fmaxf(y[u][6], y[u][7]))));
            }
          return m;
        };
        const bool hot = exponents(false) > kHot;
        if (__builtin_expect(named_bar_or(4 + group, kGroupThreads, hot), 0)) {
          // ---- move the references by the rows' exact maxima over this tile
          exponents(true);
#pragma unroll
          for (int u = 0; u < kUnits; ++u)
            if (u < n_units) {
              float mine = 0.f;
#pragma unroll
              for (int j = 0; j < 8; ++j) {
                const float x = warp_max(y[u][j]);
                if (lane == j) mine = x;
              }
              if (lane < 8) row_max[(group * 4 + quarter) * kR + 16 * u + half * 8 + lane] = mine;
            }
          named_bar_sync(4 + group, kGroupThreads);
          if (gt < ((rows_in + 7) & ~7)) {  // (rows that do not exist, in a unit with some that do, need one too)
            const float* rm = row_max + group * 4 * kR + gt;
            const float x = fmaxf(fmaxf(rm[0], rm[kR]), fmaxf(rm[2 * kR], rm[3 * kR]));
            const float low = fminf(fminf(rm[0], rm[kR]), fminf(rm[2 * kR], rm[3 * kR]));
            const float old = row_ref[group * kR + gt], now = fmaxf(old, fmaxf(x - kTop, low - kLow));
            row_ref[group * kR + gt] = now;
            row_nref[group * kR + gt] = -now;
            row_fac[group * kR + gt] = old == -INFINITY ? 0.f : ex2(old - now);
          }
          if (t >= 2) mbar_wait(PVDONE(T - 2), par(T - 2));
          named_bar_sync(4 + group, kGroupThreads);
          if (t >= 2) {
            tc_fence_after();
#pragma unroll
            for (int u = 0; u < kUnits; ++u)
              if (u < n_units) {
                const int row = 16 * u + half * 8;
                const float* fac = row_fac + group * kR + row;
#pragma unroll
                for (int e = 0; e < 4; ++e) lp2[u][e] = mul2(lp2[u][e], pack2f(fac[2 * e], fac[2 * e + 1]));
#pragma unroll 1
                for (int term = 0; term < 2; ++term) {
                  float o[8];
                  const uint32_t to = tmem + C::kTmemO + (2 * group + term) * kR + row + lane_off;
                  tmem_ld8(to, o);
                  tmem_wait_ld<8>(o);
#pragma unroll
                  for (int j = 0; j < 8; ++j) o[j] *= fac[j];
                  tmem_st8(to, o);
                }
              }
            asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
          }
          exponents(false);
        }
        // the tile's scores are all in registers: its buffer may take S(T + 4)
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(SFREE(T));
        if (T >= 2) mbar_wait(PVDONE(T - 2), par(T - 2));  // PV(T - 2) has read the P buffer
        const uint32_t dither = dither_of(tile0 + kl);
#pragma unroll
        for (int u = 0; u < kUnits; ++u)
          if (u < n_units) {
            uint32_t h[4], l[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const float e0 = ex2(y[u][2 * e]), e1 = ex2(y[u][2 * e + 1]);
              lp2[u][e] = fma2(pack2f(e0, e1), iv2, lp2[u][e]);
              two_terms<16>(e0, e1, dither, h[e], l[e]);
            }
            auto store = [&](int row, const uint32_t (&w)[4]) {  // rows row .. row + 7 of 2 kR
              const uint32_t dst = pkey + (row >> 5) * C::kPGroup + ((((row >> 4) & 1) ^ psw) << 4) + (row & 8);
              asm volatile("st.shared.v2.u32 [%0], {%1, %2};" ::"r"(dst), "r"(w[0] | (w[1] << 16)), "r"(w[2] | (w[3] << 16))
                           : "memory");
            };
            store(16 * u + half * 8, h);
            store(kR + 16 * u + half * 8, l);
          }
        const int n_here = min(kTile, key_end - tile0);
        if (n_here & 31) {
          // stale rows that the product reads may hold NaN, whose product with 0 is not 0:
          // zeros, once the tile has landed
          mbar_wait(FULLV(T), par(T));
          const int stale = 32 - (n_here & 31);
          if (gt < stale * (kDim / 16))
            st_shared_v4(base + C::kRingV + (T % kStages) * kKV + n_here * kDim + gt * 16, 0u, 0u, 0u, 0u);
        }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
        if (lane == 0) mbar_arrive(PFULL(T));
      }
      const int n_mine = (n_tiles - t_first + 1) / 2;
      // ---- row sums: lane L ends with that of row L >> 2 of the unit
#pragma unroll
      for (int u = 0; u < kUnits; ++u) {
        float v[8];
#pragma unroll
        for (int j = 0; j < 4; ++j) unpack2(lp2[u][j], v[2 * j], v[2 * j + 1]);
        const float x = warp_sum8(v, lane);
        if ((lane & 3) == 0) row_sum[(16 * u + half * 8 + (lane >> 2)) * 8 + group * 4 + quarter] = x;
      }
      const bool merge = csize > 1;
      if (merge) cluster_arrive_relaxed();  // the group has seen its last S, and the MMA warps arrive after theirs
      if (n_mine > 0) {
        const int T = T0 + t_first + 2 * (n_mine - 1);
        mbar_wait(PVDONE(T), par(T));
      }
      named_bar_sync(2, kSoftThreads);
      // ---- the groups' softmaxes joined: O = w_0 O_0 + w_1 O_1, l likewise
      const int rpc = (rows_in + csize - 1) / csize;  // rank c merges rows [c * rpc, ...)
      auto rows_of = [&](int c) { return max(0, min(rpc, rows_in - c * rpc)); };
      const int my_rows = rows_of(rank);
      if (st < kR) {
        const float4 s0 = reinterpret_cast<const float4*>(row_sum + st * 8)[0];
        const float4 s1 = reinterpret_cast<const float4*>(row_sum + st * 8)[1];
        const float l0 = (s0.x + s0.y) + (s0.z + s0.w), l1 = (s1.x + s1.y) + (s1.z + s1.w);
        const float r0 = row_ref[st], r1 = row_ref[kR + st], ref = fmaxf(r0, r1);
        // a group without a key for the row counts for nothing, one whose keys are no numbers (it
        // has no reference, or one far below) leaves NaN in l
        const float w0 = r0 == -INFINITY ? 0.f : ex2(r0 - ref), w1 = r1 == -INFINITY ? 0.f : ex2(r1 - ref);
        const float l = w0 * l0 + w1 * l1;
        bool part = merge;
        if constexpr (kEven) part = !my_run->whole;
        row_join[st] = make_float4(w0, w1, part ? l : 1.f / l, ref);
      }
      named_bar_sync(2, kSoftThreads);
      tc_fence_after();
      constexpr int kOr = kR / 4;  // this warp: its 32 d lanes of a quarter of the rows
      const int orow0 = (sw >> 2) * kOr;
      float o[kOr];
#pragma unroll
      for (int j = 0; j < kOr; ++j) o[j] = 0.f;
#pragma unroll
      for (int g = 0; g < 2; ++g)
        if (((g ^ T0) & 1) < n_tiles) {
#pragma unroll
          for (int j0 = 0; j0 < kOr; j0 += 4) {
            float r[8];  // hi and lo of 4 rows
            const uint32_t to = tmem + C::kTmemO + 2 * g * kR + orow0 + j0 + lane_off;
            tmem_ld4(to, r);
            tmem_ld4(to + kR, r + 4);
            tmem_wait_ld<8>(r);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const float4 jn = row_join[orow0 + j0 + j];
              const float w = g == 0 ? jn.x : jn.y;
              if (w != 0.f) o[j0 + j] = fmaf(w, fmaf(r[4 + j], 0.0625f, r[j]), o[j0 + j]);
            }
          }
        }
      if (kEven) {
        const Run r = *my_run;
        const int kvh = r.kvh, mblock = r.mblock, b = r.b;
        if (!r.whole) {
          // to kv8_join_kernel: a CTA's first run, or its last
          float* to = a.part + (2ll * blockIdx.x + (n_run > 0)) * (kR * kRowF);
#pragma unroll
          for (int j = 0; j < kOr; ++j)
            if (kl < kDim && orow0 + j < rows_in) __stcg(to + (orow0 + j) * kRowF + kl, o[j]);
          if (st < rows_in) __stcg(reinterpret_cast<float2*>(to + st * kRowF + kDim), make_float2(row_join[st].z, row_join[st].w));
        } else {
#pragma unroll
          for (int j = 0; j < kOr; ++j) {
            const int row = orow0 + j, p = mblock * kR + row;
            if (p < a.M && kl < kDim) a.out[q_off(b, kvh, p) + kl] = __float2bfloat16_rn(o[j] * row_join[row].z);
          }
        }
        T0 += r.n_tiles;
        continue;
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(TMEMDONE);
      if (!merge) {
#pragma unroll
        for (int j = 0; j < kOr; ++j) {
          const int row = orow0 + j, p = mblock * kR + row;
          if (valid && p < a.M && kl < kDim) a.out[q_off(b, kvh, p) + kl] = __float2bfloat16_rn(o[j] * row_join[row].z);
        }
      } else {
        float* send = reinterpret_cast<float*>(smem + C::kRingV);
        if (kl < kDim)
#pragma unroll
          for (int j = 0; j < kOr; ++j) send[(orow0 + j) * kRowF + kl] = o[j];
        if (st < kR) *reinterpret_cast<float2*>(send + st * kRowF + kDim) = make_float2(row_join[st].z, row_join[st].w);
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        named_bar_sync(2, kSoftThreads);
        if (st == 0) mbar_expect_tx(RECV, static_cast<uint32_t>(csize * my_rows * kRowBytes));
        cluster_wait();  // every peer's K ring is free to receive
        // softmax warp w sends rank w's rows to it, into its slots [rank * rpc, ...)
        if (elect_one()) {
          if (sw < csize && rows_of(sw) > 0)
            bulk_copy_s2s(cluster_map(base + rank * rpc * kRowBytes, sw), base + C::kRingV + sw * rpc * kRowBytes,
                          static_cast<uint32_t>(rows_of(sw) * kRowBytes), cluster_map(RECV, sw));
          asm volatile("cp.async.bulk.commit_group;" ::: "memory");
        }
        __syncwarp();
        // ---- merge of the rows this CTA owns, a warp a row; slot c * rpc + r came from rank c
        const float* recv = reinterpret_cast<const float*>(smem);
        const int cstep = rpc * kRowF;
        constexpr int kPer = kDim / 32;
        struct alignas(kPer * 4) Row {
          float v[kPer];
        };
#pragma unroll 1
        for (int r = sw; r < my_rows; r += kSoftWarps) {
          const float* part = recv + r * kRowF;
          const int p = mblock * kR + rank * rpc + r;
          if (r == sw) mbar_wait(RECV, 0);
          const float2 lr = lane < csize ? *reinterpret_cast<const float2*>(part + lane * cstep + kDim)
                                         : make_float2(0.f, -INFINITY);
          const float ref = warp_max(lr.y);
          const float w = lr.y == -INFINITY ? 0.f : ex2(lr.y - ref);
          float l = w * lr.x;  // (NaN stays whatever its weight)
#pragma unroll
          for (int x = 16; x > 0; x >>= 1) l += __shfl_xor_sync(0xffffffffu, l, x);
          Row ov = {};
#pragma unroll 4
          for (int c = 0; c < csize; ++c) {
            const float wc = __shfl_sync(0xffffffffu, w, c);
            const Row x = reinterpret_cast<const Row*>(part + c * cstep)[lane];
#pragma unroll
            for (int j = 0; j < kPer; ++j)
              if (wc != 0.f) ov.v[j] = fmaf(wc, x.v[j], ov.v[j]);
          }
          if (valid && p < a.M) {
            const float inv_l = 1.f / l;
            __nv_bfloat16* dst = a.out + q_off(b, kvh, p) + lane * kPer;
#pragma unroll
            for (int j = 0; j < kPer; j += 2)
              *reinterpret_cast<uint32_t*>(dst + j) = cvt_bf16x2(ov.v[j] * inv_l, ov.v[j + 1] * inv_l);
          }
        }
        if (elect_one()) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
        __syncwarp();
      }
    }
    if (kEven) {
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(TMEMDONE);
    }
  }
  // no CTA-wide barrier at the end: every warp leaves when its own work is done
}

// The units that a border between shares cuts: the first border in a unit joins its parts,
// in the order of the keys. Grid (CTAs of the attention - 1, row groups), kJoinRows rows a
// warp. CTAs small enough to stand beside the attention's: they have found their unit when
// its last part is written.
constexpr int kJoinWarps = 4, kJoinRows = 4;
template <int kR, int kDim>
__global__ void __launch_bounds__(32 * kJoinWarps) kv8_join_kernel(const Args a, int ctas) {
  constexpr int kRowF = kDim + 4, kPer = kDim / 32;
  const int lane = threadIdx.x & 31, c = blockIdx.x + 1;
  // (the lengths are older than the attention, which let this kernel start after its own wait)
  const Scenes scenes = scenes_of(a);
  const Shares s = shares_of(scenes, lane, ctas);
  const int pos = s.begin(c);
  bool mine = pos < s.total;
  Place at = {};
  if (mine) at = locate(scenes, s, pos, lane);
  const int unit_begin = at.first, unit_end = unit_begin + at.tiles;
  mine = mine && at.tile > 0 && s.begin(c - 1) <= unit_begin;
  const int kvh = at.unit / a.mblocks, mblock = at.unit - kvh * a.mblocks;
  const int row0 = (blockIdx.y * kJoinWarps + (threadIdx.x >> 5)) * kJoinRows;
  const int n_rows = min(min(kR, a.M - mblock * kR) - row0, kJoinRows);
  // part 0: the last run of CTA c - 1, its first where it begins with the unit; then the
  // first runs of those after it (their shares may be empty)
  int ends = c;  // the CTA whose share ends the unit
  while (mine && s.begin(ends + 1) < unit_end) ++ends;
  const int n_parts = ends - c + 2;
  auto part = [&](int i) {
    const int slot = 2 * (c - 1 + i) + (i == 0 && s.begin(c - 1) < unit_begin ? 1 : 0);
    return a.part + (static_cast<long long>(slot) * kR + row0) * kRowF;
  };
  griddep_wait();  // (the next kernel waits for this one's end: beside its large CTAs these ran late, 107 us)
  if (!mine || n_rows <= 0) return;
  float m[kJoinRows], l[kJoinRows], o[kJoinRows][kPer];
#pragma unroll
  for (int r = 0; r < kJoinRows; ++r) {
    m[r] = -INFINITY;
    l[r] = 0.f;
#pragma unroll
    for (int j = 0; j < kPer; ++j) o[r][j] = 0.f;
  }
#pragma unroll 2
  for (int i = 0; i < n_parts; ++i) {
    if (s.begin(c + i) == s.begin(c - 1 + i)) continue;
    const float* x = part(i);
#pragma unroll
    for (int r = 0; r < kJoinRows; ++r) {
      if (r >= n_rows) break;
      const float2 lr = __ldcg(reinterpret_cast<const float2*>(x + r * kRowF + kDim));
      float v[kPer];
#pragma unroll
      for (int j = 0; j < kPer; j += 2) {
        const float2 y = __ldcg(reinterpret_cast<const float2*>(x + r * kRowF + lane * kPer + j));
        v[j] = y.x;
        v[j + 1] = y.y;
      }
      // (no key of the part that the row sees: its reference is -inf, its weight 0)
      const float now = fmaxf(m[r], lr.y), f = m[r] == -INFINITY ? 0.f : ex2(m[r] - now);
      const float w = lr.y == -INFINITY ? 0.f : ex2(lr.y - now);
      l[r] = l[r] * f + w * lr.x;  // (NaN stays whatever its weight)
#pragma unroll
      for (int j = 0; j < kPer; ++j) o[r][j] = o[r][j] * f + (w != 0.f ? w * v[j] : 0.f);
      m[r] = now;
    }
  }
#pragma unroll
  for (int r = 0; r < kJoinRows; ++r) {
    if (r >= n_rows) break;
    const int p = mblock * kR + row0 + r, i = __float2int_rz((static_cast<float>(p) + 0.5f) * a.inv_g);
    __nv_bfloat16* out = a.out + ((static_cast<long long>(at.b) * a.R + i) * a.Hq + kvh * a.G + (p - i * a.G)) * kDim;
    const float inv_l = 1.f / l[r];
#pragma unroll
    for (int j = 0; j < kPer; j += 2)
      *reinterpret_cast<uint32_t*>(out + lane * kPer + j) = cvt_bf16x2(o[r][j] * inv_l, o[r][j + 1] * inv_l);
  }
}

// ------------------------------------------------------------------ host
constexpr int kClusterSizes[] = {1, 2, 4, 5, 6, 8, 10, 12, 16};
constexpr int kNumSizes = sizeof(kClusterSizes) / sizeof(int);

template <int kR, int kDim>
bool set_attributes(int* active) {
  const void* k = reinterpret_cast<const void*>(kv8_attention_kernel<kR, kDim, false>);
  const void* even = reinterpret_cast<const void*>(kv8_attention_kernel<kR, kDim, true>);
  constexpr int smem = Cfg<kR, kDim>::kSmemBytes;
  if (cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, smem) != cudaSuccess ||
      cudaFuncSetAttribute(even, cudaFuncAttributeMaxDynamicSharedMemorySize, smem) != cudaSuccess ||
      cudaFuncSetAttribute(k, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) != cudaSuccess) {
    (void)cudaGetLastError();
    return false;
  }
  for (int i = 0; i < kNumSizes; ++i) {
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = kClusterSizes[i];
    attr[0].val.clusterDim.y = 1;
    attr[0].val.clusterDim.z = 1;
    cfg.gridDim = dim3(kClusterSizes[i], 1, 1);
    cfg.blockDim = dim3(Cfg<kR, kDim>::kThreads, 1, 1);
    cfg.dynamicSmemBytes = smem;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    int m = 0;
    if (cudaOccupancyMaxActiveClusters(&m, k, &cfg) != cudaSuccess) {
      (void)cudaGetLastError();
      m = 0;
    }
    active[i] = m;
  }
  return true;
}

struct DevState {
  std::once_flag once;
  bool ok = false;
  int active[4][kNumSizes] = {};  // [head dim 64, 128][rows 32, 48]
};

DevState* state() {
  static DevState states[64];
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) {
    (void)cudaGetLastError();
    return nullptr;
  }
  DevState& s = states[dev];
  std::call_once(s.once, [&s] {
    s.ok = set_attributes<32, 64>(s.active[0]) && set_attributes<48, 64>(s.active[1]) &&
           set_attributes<32, 128>(s.active[2]) && set_attributes<48, 128>(s.active[3]);
  });
  return &s;
}

// CTAs a unit: the size that sd_set_cluster_size forces, else the one of least cost, in
// 128-key tiles: waves x (tiles a CTA + a fixed cost a wave). 0: even shares over all SMs,
// where they cost less (tiles a CTA + 4 a unit + the start and the join) and the call may
// have them. Clusters / even shares in us, 8 KV heads of 4096 keys (3/4 to all of them
// filled) and 32 rows: 10 scenes 24.0 / 26.6, 16: 25.4 / 31.9, 20: 44.9 / 38.2, 24: 46.6 /
// 42.6, 32: 49.2 / 50.3, 64: 102 / 86; 32 scenes of 8192 keys and 36 rows 113 / 103, 64 of
// 1024 41 / 44. Head dim 64, 4 KV heads of 4096: 20 scenes 34.7 / 32.6, 40: 57.0 / 49.6.
int pick_cluster(const int* active, long long units, int cap, int D, bool may) {
  const int forced = sd_internal_forced_cluster();
  for (int i = 0; i < kNumSizes && forced > 0; ++i)
    if (kClusterSizes[i] == forced && active[i] > 0) return forced;
  const double nblk = (cap + 31) / 32;
  double best_cost = -1;
  int best = -1;
  for (int i = 0; i < kNumSizes; ++i) {
    const int cs = kClusterSizes[i];
    if (active[i] <= 0 || (cs > 1 && nblk < 2.0 * cs)) continue;
    const long long waves = (units + active[i] - 1) / active[i];
    const double fixed = (waves > 1 ? 5.0 : 1.0) + (cs > 8 ? 0.8 : 0.0);
    const double cost = static_cast<double>(waves) * (nblk / (4.0 * cs) + fixed);
    if (best < 0 || cost < best_cost) {
      best_cost = cost;
      best = cs;
    }
  }
  const double start = D == 128 ? 14.5 : 17.0, tiles = static_cast<double>(units) * ((cap + kTile - 1) / kTile);
  if (may && active[0] > 1 && tiles < 2e9 && (tiles + 4.0 * units) / active[0] + start < best_cost) return 0;
  return best;
}

// [planes][cap][D] codes in boxes of one whole row x 128 rows, swizzled by the row's width
bool make_map8(CUtensorMap* map, void* base, int cap, int planes, int D) {
  EncodeTiledFn fn = encode_fn();
  if (!fn) return false;
  cuuint64_t dims[3] = {static_cast<cuuint64_t>(D), static_cast<cuuint64_t>(cap), static_cast<cuuint64_t>(planes)};
  cuuint64_t strides[2] = {static_cast<cuuint64_t>(D), static_cast<cuuint64_t>(cap) * static_cast<cuuint64_t>(D)};
  cuuint32_t box[3] = {static_cast<cuuint32_t>(D), kTile, 1};
  cuuint32_t estr[3] = {1, 1, 1};
  return fn(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 3, base, dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
            D == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// cs: CTAs a cluster, 0: even shares over `ctas`
template <int kR, int kDim>
sd_status launch(const sd_kv8_cache* c, const Args& a, int cs, int ctas, cudaStream_t stream) {
  CUtensorMap k, v;
  if (!make_map8(&k, c->k, c->capacity, c->batch * c->n_kv_heads, kDim) ||
      !make_map8(&v, c->v, c->capacity, c->batch * c->n_kv_heads, kDim))
    return SD_ERR_CUDA;
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = cs;
  attr[1].val.clusterDim.y = 1;
  attr[1].val.clusterDim.z = 1;
  cfg.blockDim = dim3(Cfg<kR, kDim>::kThreads, 1, 1);
  cfg.dynamicSmemBytes = Cfg<kR, kDim>::kSmemBytes;
  cfg.stream = stream;
  cfg.attrs = attr;
  cudaError_t e;
  if (cs > 0) {
    cfg.gridDim = dim3(cs, c->n_kv_heads * a.mblocks, c->batch);
    cfg.numAttrs = 2;
    e = cudaLaunchKernelEx(&cfg, kv8_attention_kernel<kR, kDim, false>, k, v, a);
  } else {
    cfg.gridDim = dim3(ctas, 1, 1);
    cfg.numAttrs = 1;
    e = cudaLaunchKernelEx(&cfg, kv8_attention_kernel<kR, kDim, true>, k, v, a);
    if (e == cudaSuccess) {
      cfg.gridDim = dim3(ctas - 1, (std::min(a.M, kR) + kJoinWarps * kJoinRows - 1) / (kJoinWarps * kJoinRows), 1);
      cfg.blockDim = dim3(32 * kJoinWarps, 1, 1);
      cfg.dynamicSmemBytes = 0;
      e = cudaLaunchKernelEx(&cfg, kv8_join_kernel<kR, kDim>, a, ctas);
    }
  }
  if (e != cudaSuccess) {
    (void)cudaGetLastError();
    return SD_ERR_CUDA;
  }
  return SD_OK;
}

// How a shape is taken on the current device.
struct Plan {
  int mblocks, rows, cs, ctas;  // cs 0: even shares over `ctas` CTAs
  size_t ws_bytes;
};
sd_status make_plan(int B, int R, int Hq, int Hkv, int D, int cap, bool may, Plan* p) {
  const int M = Hq / Hkv * R;
  // the fewest m-blocks of up to 48 rows, and the smaller tile that holds one. (64 rows in
  // two m-blocks of 32, which read every key twice, mostly from L2: 154.7 us for 32 scenes
  // of 8192 keys, 9.9 for one of 4096; one tile of 64, 32 rows a thread in registers, took
  // 150 to 165 and 12.5.)
  p->mblocks = (M + 47) / 48;
  p->rows = (M + p->mblocks - 1) / p->mblocks <= 32 ? 32 : 48;
  DevState* dev = state();
  if (!dev || !dev->ok) return SD_ERR_CUDA;
  const int* active = dev->active[(D == 128 ? 2 : 0) + (p->rows == 48)];
  p->cs = pick_cluster(active, static_cast<long long>(B) * Hkv * p->mblocks, cap, D, may);
  p->ctas = active[0];
  p->ws_bytes = p->cs == 0 ? 2 * static_cast<size_t>(p->ctas) * p->rows * (D + 4) * sizeof(float) : 0;
  return p->cs < 0 ? SD_ERR_CUDA : SD_OK;
}

}  // namespace

extern "C" size_t sd_kv8_attention_workspace(int B, int R, int Hq, int Hkv, int D, int capacity) {
  if (B <= 0 || R <= 0 || Hkv <= 0 || Hq <= 0 || Hq % Hkv || (D != 64 && D != 128) || capacity <= 0 ||
      static_cast<long long>(Hq / Hkv) * R > 128)
    return 0;
  Plan p = {};
  return make_plan(B, R, Hq, Hkv, D, capacity, true, &p) == SD_OK ? p.ws_bytes : 0;
}

extern "C" sd_status sd_kv8_attention_ex(const void* q, const sd_kv8_cache* cache, void* out, int R, int Hq, float scale,
                                         int flags, void* workspace, size_t ws_bytes, sd_stream_t stream) {
  const sd_status s = sd_internal_kv8_check(cache);
  if (s != SD_OK) return s;
  const int B = cache->batch, Hkv = cache->n_kv_heads, D = cache->head_dim;
  if (R <= 0 || Hq <= 0 || Hq % Hkv || (flags & ~SD_ATTN_BLOCK_MASK)) return SD_ERR_INVALID_ARG;
  if (!(scale >= 0.f) || !isfinite(scale)) return SD_ERR_INVALID_ARG;
  if (static_cast<long long>(Hq / Hkv) * R > 128) return SD_ERR_UNSUPPORTED;
  if (B == 0) return SD_OK;
  if (!q || !out || !sd_aligned16(q) || !sd_aligned16(out)) return SD_ERR_INVALID_ARG;
  if (workspace && !sd_aligned16(workspace)) return SD_ERR_INVALID_ARG;
  Plan p = {};
  const sd_status planned = make_plan(B, R, Hq, Hkv, D, cache->capacity, workspace != nullptr, &p);
  if (planned != SD_OK) return planned;
  if (p.ws_bytes > ws_bytes) return SD_ERR_WORKSPACE;
  const double sc = scale > 0.f ? scale : 1.0 / sqrt(static_cast<double>(D));
  Args a = {};
  a.q = static_cast<const __nv_bfloat16*>(q);
  a.out = static_cast<__nv_bfloat16*>(out);
  a.ks = cache->k_scale;
  a.vs = cache->v_scale;
  a.len = cache->len;
  a.part = static_cast<float*>(workspace);
  a.B = B;
  a.R = R;
  a.Hq = Hq;
  a.Hkv = Hkv;
  a.G = Hq / Hkv;
  a.M = a.G * R;
  a.cap = cache->capacity;
  a.nblk = (cache->capacity + cache->block - 1) / cache->block;
  a.block_shift = cache->block == 32 ? 5 : (cache->block == 64 ? 6 : 7);
  a.mblocks = p.mblocks;
  a.block_mask = (flags & SD_ATTN_BLOCK_MASK) != 0;
  a.inv_g = 1.0f / static_cast<float>(a.G);
  a.scale_log2 = static_cast<float>(sc * 1.4426950408889634);
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  const auto run = D == 128 ? (p.rows == 32 ? launch<32, 128> : launch<48, 128>)
                            : (p.rows == 32 ? launch<32, 64> : launch<48, 64>);
  return run(cache, a, p.cs, p.ctas, st);
}

extern "C" sd_status sd_kv8_attention(const void* q, const sd_kv8_cache* cache, void* out, int R, int Hq, float scale,
                                      int flags, sd_stream_t stream) {
  return sd_kv8_attention_ex(q, cache, out, R, Hq, scale, flags, nullptr, 0, stream);
}
