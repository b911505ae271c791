// The 8-bit KV cache: rows quantised as they are appended, or a whole bf16 cache
// stored at once (sm_103a).
//
// A cached value is code * scale, the code an e4m3 number (4 significant bits, at most
// 448), the scale one fp32 number for a block of `block` consecutive tokens of one KV
// head of one scene, keys and values apart. A block that begins with new rows takes the
// smallest power of two that keeps its largest finite value within 448:
//     s = 2^e,  e = min { e >= -100 : amax <= 448 * 2^e },   code = e4m3(x / s)
// (a power of two costs a floating-point code no precision, and moves it exactly). A
// block that already holds rows keeps its scale s, times the least power of two 2^g,
// g >= 0, that fits the new rows; its older codes then move by 2^-g, which rounds only
// those that become subnormal. Codes round to nearest even; infinities saturate, NaN
// stays NaN, and neither counts for amax.
//
// One CTA quantises one block of one head's keys or values: its rows stay in registers
// between the maximum and the rounding, so every value is read once and every code
// written once. A store is bound by memory: 368 MB in 58.5 us, 0.92 of the measured copy
// rate. What it needs is bytes in flight over its barrier: four units of 32 bytes a thread
// take 33 us for 201 MB whatever the head dim and block, two 36, one 45 (a thread for each
// two, of up to 256, took 65.8 for the first), eight, at fewer warps, 43. An append (3.5 us)
// is two round trips and its ticket.
#include "common.cuh"

SD_DEFINE_ERROR_ACCESSOR(sd_take_error_kv8)

namespace {

constexpr int kMinExp = -100;

struct Kv8Args {
  const uint4* k_new;     // bf16 rows: scene stride sb, row stride sr, head stride sh, in 16-byte units
  const uint4* v_new;
  long long sb, sr, sh;
  uint8_t* k;
  uint8_t* v;
  float* k_scale;
  float* v_scale;
  int32_t* len;
  uint32_t* ticket;
  const int32_t* src_len; // store: rows of the bf16 cache; append: nullptr
  int R, Hkv, cap, src_cap, nblk;
};

// Exponent of the smallest power of two s with x <= 448 s (448 = 1.75 * 2^8), x > 0 a
// normal number with exponent field and mantissa in `bits`.
__device__ __forceinline__ int scale_exp(uint32_t bits) {
  return static_cast<int>(bits >> 23) - 127 - ((bits & 0x7fffffu) <= 0x600000u ? 8 : 7);
}
__device__ __forceinline__ float pow2f(int e) { return __uint_as_float(static_cast<uint32_t>(e + 127) << 23); }

// Two fp32 -> two e4m3 codes (round to nearest even, saturating), lo in the low byte.
__device__ __forceinline__ uint32_t e4m3x2(float lo, float hi) {
  uint16_t r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
  return r;
}
// Two e4m3 codes -> two fp16 numbers (exact).
__device__ __forceinline__ float2 e4m3x2_to_float(uint32_t w) {
  uint32_t h;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"(static_cast<uint16_t>(w)));
  float lo, hi;
  asm("{\n\t.reg .f16 a, b;\n\tmov.b32 {a, b}, %2;\n\tcvt.f32.f16 %0, a;\n\tcvt.f32.f16 %1, b;\n\t}"
      : "=f"(lo), "=f"(hi)
      : "r"(h));
  return make_float2(lo, hi);
}

// 16 bf16 numbers (two 16-byte chunks) -> 16 codes. kMul: x * m, exact for the inverse
// of a power of two; otherwise x / m.
template <bool kMul>
__device__ __forceinline__ uint4 encode16(const uint4 (&x)[2], float m) {
  uint32_t o[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint4& c = x[i >> 1];
    const uint32_t w0 = (i & 1) ? c.z : c.x, w1 = (i & 1) ? c.w : c.y;
    float f[4] = {sd_bf16_lo(w0), sd_bf16_hi(w0), sd_bf16_lo(w1), sd_bf16_hi(w1)};
#pragma unroll
    for (int j = 0; j < 4; ++j) f[j] = kMul ? f[j] * m : __fdiv_rn(f[j], m);
    o[i] = e4m3x2(f[0], f[1]) | (e4m3x2(f[2], f[3]) << 16);
  }
  return make_uint4(o[0], o[1], o[2], o[3]);
}

// The largest finite |x| of a chunk, as the 15 bits of a bf16.
__device__ __forceinline__ uint32_t amax8(const uint4& c) {
  uint32_t m = 0;
  const uint32_t w[4] = {c.x, c.y, c.z, c.w};
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const uint32_t lo = w[j] & 0x7fffu, hi = (w[j] >> 16) & 0x7fffu;
    m = max(m, max(lo < 0x7f80u ? lo : 0u, hi < 0x7f80u ? hi : 0u));
  }
  return m;
}

// Grid (token blocks, 2 * Hkv, B): y < Hkv the keys of head y, else the values of head
// y - Hkv; x counts from the first block that the new rows touch.
template <int D, int kBlock>
struct Kv8Cfg {
  static constexpr int kRowUnits = D / 16;             // 16 values: 32 bytes in, 16 out
  static constexpr int kUnits = kBlock * kRowUnits;
  static constexpr int kPer = 4;                       // a thread's units, all on their way at once
  static constexpr int kThreads = kUnits / kPer;
};

template <int D, int kBlock>
__global__ void __launch_bounds__(Kv8Cfg<D, kBlock>::kThreads) kv8_append_kernel(const Kv8Args a) {
  using C = Kv8Cfg<D, kBlock>;
  sd_pdl_enter();
  const int b = blockIdx.z, h = blockIdx.y % a.Hkv;
  const bool values = blockIdx.y >= static_cast<unsigned>(a.Hkv);
  const int n0 = a.src_len ? 0 : __ldcg(a.len + b);
  const int n = a.src_len ? __ldcg(a.src_len + b) : a.R;
  const bool ok = n0 >= 0 && n >= 0 && static_cast<long long>(n0) + n <= a.cap && (!a.src_len || n <= a.src_cap);
  // behind a barrier that follows the CTA's reads of the length: an append's last CTA of
  // the scene to come here advances it (a store reads the other cache's length only)
  auto advance = [&] {
    if (threadIdx.x != 0) return;
    if (a.src_len) {
      if (blockIdx.x || blockIdx.y) return;
    } else {
      __threadfence();
      if (atomicAdd(&a.ticket[b], 1u) != gridDim.x * gridDim.y - 1) return;
      a.ticket[b] = 0;
    }
    if (ok) a.len[b] = n0 + n;
    else sd_set_error(a.src_len && (n < 0 || n > a.src_cap) ? SD_DEVERR_LENGTH : SD_DEVERR_KV_OVERFLOW);
  };
  const int blk = n0 / kBlock + static_cast<int>(blockIdx.x);
  const int row0 = blk * kBlock;
  if (!ok || row0 >= n0 + n) {
    __syncthreads();
    advance();
    return;
  }
  const uint4* src = (values ? a.v_new : a.k_new) + b * a.sb + h * a.sh;
  const long long plane = static_cast<long long>(b) * a.Hkv + h;
  uint4* dst = reinterpret_cast<uint4*>((values ? a.v : a.k) + (plane * a.cap + row0) * D);
  float* scale = (values ? a.v_scale : a.k_scale) + plane * a.nblk + blk;

  uint4 x[C::kPer][2];
  uint32_t m = 0;
#pragma unroll
  for (int u = 0; u < C::kPer; ++u) {
    const int unit = threadIdx.x + u * C::kThreads, r = row0 + unit / C::kRowUnits - n0;
    if (r >= 0 && r < n) {
      const uint4* p = src + r * a.sr + (unit % C::kRowUnits) * 2;
      x[u][0] = __ldcg(p);
      x[u][1] = __ldcg(p + 1);
    } else {
      x[u][0] = x[u][1] = make_uint4(0, 0, 0, 0);
    }
  }
#pragma unroll
  for (int u = 0; u < C::kPer; ++u) m = max(m, max(amax8(x[u][0]), amax8(x[u][1])));
  __shared__ uint32_t warp_max[8];
  m = __reduce_max_sync(0xffffffffu, m);
  if ((threadIdx.x & 31) == 0) warp_max[threadIdx.x >> 5] = m;
  __syncthreads();
  advance();
#pragma unroll
  for (int w = 0; w < C::kThreads / 32; ++w) m = max(m, warp_max[w]);
  const uint32_t amax = m << 16;  // the bits of an fp32 number
  float s;
  if (row0 >= n0) {
    s = pow2f(amax ? max(kMinExp, scale_exp(amax)) : kMinExp);
    if (threadIdx.x == 0) *scale = s;
  } else {
    const float old = __ldcg(scale);
    int g = 0;
    if (amax) {
      // the ratio in 64 bits: a block of zeros has the smallest scale
      const double ratio = static_cast<double>(__uint_as_float(amax)) / static_cast<double>(old);
      const uint64_t bits = static_cast<uint64_t>(__double_as_longlong(ratio));
      g = max(0, static_cast<int>(bits >> 52) - 1023 - ((bits & 0xfffffffffffffull) <= 0xc000000000000ull ? 8 : 7));
    }
    s = old;
    if (g) {  // the same for the whole CTA
      s = static_cast<float>(ldexp(static_cast<double>(old), g));
      const float f = pow2f(-min(g, 60));
#pragma unroll
      for (int u = 0; u < C::kPer; ++u) {
        const int unit = threadIdx.x + u * C::kThreads;
        if (row0 + unit / C::kRowUnits >= n0) continue;
        const uint4 c = dst[unit];
        uint32_t w[4] = {c.x, c.y, c.z, c.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float2 p = e4m3x2_to_float(w[j]), q = e4m3x2_to_float(w[j] >> 16);
          w[j] = e4m3x2(p.x * f, p.y * f) | (e4m3x2(q.x * f, q.y * f) << 16);
        }
        dst[unit] = make_uint4(w[0], w[1], w[2], w[3]);
      }
      __syncthreads();  // every thread has read the old scale
      if (threadIdx.x == 0) *scale = s;
    }
  }
  // (2^127 has no normal inverse)
  const bool pow2 = (__float_as_uint(s) & 0x7fffffu) == 0 && __float_as_uint(s) < 0x7f000000u;
  const float inv = pow2f(127 - static_cast<int>(__float_as_uint(s) >> 23));
#pragma unroll
  for (int u = 0; u < C::kPer; ++u) {
    const int unit = threadIdx.x + u * C::kThreads, r = row0 + unit / C::kRowUnits - n0;
    if (r >= 0 && r < n) dst[unit] = pow2 ? encode16<true>(x[u], inv) : encode16<false>(x[u], s);
  }
}

template <int D>
cudaError_t launch_block(int block, const Kv8Args& a, int blocks, int B, cudaStream_t st) {
  const dim3 grid(blocks, 2 * a.Hkv, B);
  if (block == 32) return sd_launch_pdl(kv8_append_kernel<D, 32>, grid, dim3(Kv8Cfg<D, 32>::kThreads), 0, st, a);
  if (block == 64) return sd_launch_pdl(kv8_append_kernel<D, 64>, grid, dim3(Kv8Cfg<D, 64>::kThreads), 0, st, a);
  return sd_launch_pdl(kv8_append_kernel<D, 128>, grid, dim3(Kv8Cfg<D, 128>::kThreads), 0, st, a);
}

sd_status launch(const sd_kv8_cache* c, const Kv8Args& a, int blocks, cudaStream_t st) {
  const cudaError_t e = c->head_dim == 64 ? launch_block<64>(c->block, a, blocks, c->batch, st)
                                          : launch_block<128>(c->block, a, blocks, c->batch, st);
  if (e != cudaSuccess) {
    (void)cudaGetLastError();
    return SD_ERR_CUDA;
  }
  return SD_OK;
}

Kv8Args args_of(const sd_kv8_cache* c) {
  Kv8Args a = {};
  a.k = static_cast<uint8_t*>(c->k);
  a.v = static_cast<uint8_t*>(c->v);
  a.k_scale = c->k_scale;
  a.v_scale = c->v_scale;
  a.len = c->len;
  a.ticket = c->ticket;
  a.Hkv = c->n_kv_heads;
  a.cap = c->capacity;
  a.nblk = (c->capacity + c->block - 1) / c->block;
  return a;
}

}  // namespace

sd_status sd_internal_kv8_check(const sd_kv8_cache* c) {
  if (!c || c->batch < 0 || c->n_kv_heads <= 0 || c->capacity <= 0) return SD_ERR_INVALID_ARG;
  if (c->head_dim != 64 && c->head_dim != 128) return SD_ERR_UNSUPPORTED;
  if (c->block != 32 && c->block != 64 && c->block != 128) return SD_ERR_UNSUPPORTED;
  if (c->batch > 65535 || c->n_kv_heads > 32767) return SD_ERR_UNSUPPORTED;
  if (c->batch == 0) return SD_OK;
  if (!c->k || !c->v || !c->k_scale || !c->v_scale || !c->len || !c->ticket) return SD_ERR_INVALID_ARG;
  if (!sd_aligned16(c->k) || !sd_aligned16(c->v)) return SD_ERR_INVALID_ARG;
  return SD_OK;
}

extern "C" sd_status sd_kv8_append(const sd_kv8_cache* cache, const void* k_new, const void* v_new, int R,
                                   sd_stream_t stream) {
  const sd_status s = sd_internal_kv8_check(cache);
  if (s != SD_OK) return s;
  if (R < 0) return SD_ERR_INVALID_ARG;
  if (cache->batch == 0 || R == 0) return SD_OK;
  if (!k_new || !v_new || !sd_aligned16(k_new) || !sd_aligned16(v_new)) return SD_ERR_INVALID_ARG;
  if (R > cache->capacity) return SD_ERR_INVALID_ARG;
  Kv8Args a = args_of(cache);
  const long long row = cache->head_dim / 8;
  a.k_new = static_cast<const uint4*>(k_new);
  a.v_new = static_cast<const uint4*>(v_new);
  a.sh = row;
  a.sr = row * a.Hkv;
  a.sb = a.sr * R;
  a.R = R;
  // a scene's rows touch at most this many blocks, wherever its length lies in one
  return launch(cache, a, min((R - 1) / cache->block + 2, a.nblk), reinterpret_cast<cudaStream_t>(stream));
}

extern "C" sd_status sd_kv8_store(const sd_kv8_cache* cache, const sd_kv_cache* src, sd_stream_t stream) {
  const sd_status s = sd_internal_kv8_check(cache);
  if (s != SD_OK) return s;
  if (!src || src->batch != cache->batch || src->n_kv_heads != cache->n_kv_heads ||
      src->head_dim != cache->head_dim || src->capacity <= 0)
    return SD_ERR_INVALID_ARG;
  if (cache->batch == 0) return SD_OK;
  if (!src->k || !src->v || !src->len || !sd_aligned16(src->k) || !sd_aligned16(src->v)) return SD_ERR_INVALID_ARG;
  Kv8Args a = args_of(cache);
  const long long row = cache->head_dim / 8;
  a.k_new = static_cast<const uint4*>(src->k);
  a.v_new = static_cast<const uint4*>(src->v);
  a.sr = row;
  a.sh = row * src->capacity;
  a.sb = a.sh * a.Hkv;
  a.src_len = src->len;
  a.src_cap = src->capacity;
  const int rows = min(src->capacity, cache->capacity);
  return launch(cache, a, (rows + cache->block - 1) / cache->block, reinterpret_cast<cudaStream_t>(stream));
}
