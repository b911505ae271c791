// The attention weight that every cached key gathers from the rows of a pass (sm_103a):
// with p the softmax of q . k * scale over the keys a row sees (as in the verify
// attention),
//     out[b][g][n] = decay * in[b][g][n] + sum over rows i < committed[b] and the query
//                    heads h of KV head g of p[b][i][h][n]
// where a key appended with these rows (n >= len[b] - R) brings no weight with it.
//
// A weight needs its row's sum over all keys, so every score is needed twice. Up to 64
// packed rows (G * R) it is formed once: S^T[128 keys][kR rows] = K_tile . Q^T on the
// tensor cores (tcgen05), every tile to its own columns of tensor memory, where it waits
// for the sums (512 columns: 16 tiles of 32 rows, 8 of 64). A CTA with more tiles than
// that, and any with 128 rows, reads its keys and forms its scores a second time. One
// cluster per (KV head, scene); its CTAs take contiguous ranges of the keys and send each
// other their rows' (maximum, sum), (m, l).
//
// Pass A, the rows' sums: a thread has one key lane and a quarter of the rows, and keeps
// its own reference for each, the first score it meets, moved only when one lies 2^100
// above it: no exchange between threads before the end. There the lanes' references are
// brought to their maximum and the sums added, in a fixed order. With 128 rows, whose
// references and sums do not fit a thread, the product is not transposed here, S[128
// rows][128 keys] = Q . K_tile^T: a thread has one row of every fourth tile.
// Pass B, the keys' weights: with its row's log sum every weight is final, 2^(S c - lse).
// A thread has one key and all rows, so a key's sum needs no exchange at all; the four
// warps of a lane quarter take every fourth tile.
// More than 128 rows go through both passes in turn.
// Even shares. Where clusters fill the SMs badly and the caller gives a workspace, every SM
// takes an even share of all scenes' tiles, in two kernels: pass A leaves its runs' sums in
// the workspace, pass B joins a unit's and goes through its share backwards.
//
// What bounds it. One scene (8 heads, L = 4096, 32 rows: 6.9 us) the chain of latencies:
// lengths, keys and rows, products, sums, their exchange, weights. Eight scenes of 8192
// keys and 128 rows (51.4 us, 121 MB of keys read twice) the SMs' reading of 242 MB, 35 us
// by itself on 128 CTAs (36 bytes a cycle and SM); the second reading finds about two
// thirds of the keys in L2 (152 MB from DRAM), and a CTA's last four tiles in their slots.
// With the products 38, with the exponentials of both passes 48 from L2. Two CTAs an SM,
// each with half the warps and tensor memory, were slower (one scene 9.7, eight 52 at their
// best size).
#include "shares.cuh"
#include "tc_common.cuh"

#include <math.h>

SD_DEFINE_ERROR_ACCESSOR(sd_take_error_weights)

namespace {

constexpr int kTile = 128;
constexpr int kHalf = kTile * 128;       // one 64-column half of a tile's keys
constexpr int kSlices = 4;
constexpr int kSoftWarps = 4 * kSlices;
constexpr int kSoftThreads = 32 * kSoftWarps;
constexpr int kFirstSoft = 2;
constexpr int kSoft0 = 32 * kFirstSoft;
constexpr int kThreads = kSoft0 + kSoftThreads;
constexpr int kMaxCluster = 16;
constexpr int kMaxBufs = 16;
constexpr int kStages = 4;
constexpr float kFar = 100.f;            // log2 of what a weight may lie above its reference
constexpr float kHuge = 1e30f;           // a tile's sum that moves the reference
constexpr float kNone = -3e38f;          // no reference yet: finite, so that a score of -inf has weight 0

struct Args {
  const __nv_bfloat16* q;
  const int32_t* len;
  const int32_t* committed;
  const float* in;
  float* out;
  float2* sums;      // even shares: a run's (m, l) of the row tile
  int B, R, Hq, Hkv, G, M, cap;
  float inv_g;       // 1 / G: p / G == int((p + 0.5) / G) exactly for p < 2^20 and G < 2^12
  float scale_log2, decay;
};

template <int kR, int kDim>
struct Cfg {
  static_assert(kR == 32 || kR == 64 || kR == 128, "row tile");
  static constexpr int kHalves = kDim / 64;
  static constexpr int kK = kHalves * kHalf;       // one tile of keys
  static constexpr int kQHalf = kR * 128;
  static constexpr int kBufs = 512 / kR;           // tiles of scores in tensor memory
  static constexpr bool kTurned = kR == 128;       // pass A on S, not S^T
  static constexpr int kRpt = kTurned ? 8 : kR / kSlices;  // rows of a thread in pass A on S^T
  static constexpr int kOffQ = kStages * kK;
  static constexpr int kOffBar = kOffQ + kHalves * kQHalf;
  // full[stages] free[stages] s_ready[bufs] s_free[bufs] q_full gathered[2]
  static constexpr int kNumBars = 2 * kStages + 2 * kMaxBufs + 3;
  static constexpr int kOffMisc = round_up(kOffBar + kNumBars * 8, 16);
  static constexpr int kOffPart = kOffMisc + 16;                  // [kR][4 lane quarters, or slices] (m, l)
  static constexpr int kOffGather = kOffPart + 4 * kR * 8;        // [2][cluster rank][kR] (m, l)
  static constexpr int kOffLse = kOffGather + 2 * kMaxCluster * kR * 8;  // [kR] negated log sums
  static constexpr int kSmemBytes = kOffLse + kR * 4 + 1024;
  static_assert(kSmemBytes <= 227 * 1024, "shared memory budget");
};

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

// kBoth: grid (cluster size, Hkv, B), both passes. Else even shares, grid (CTAs), up to kR
// rows: kSums forms the runs' row sums, kWeights joins a unit's and forms its keys' weights,
// run by run from the share's last tile back to its first.
enum Pass { kBoth, kSums, kWeights };
template <int kR, int kDim, int kPass>
__global__ void __launch_bounds__(kThreads, 1)
    key_weights_kernel(const __grid_constant__ CUtensorMap tm_k, const Args a) {
  using C = Cfg<kR, kDim>;
  constexpr int kHalves = C::kHalves, kK = C::kK, kBufs = C::kBufs, kRpt = C::kRpt;
  constexpr uint32_t kIdesc = umma_idesc(128, kR, 0, 0);
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
  const uint32_t base = smem_addr(smem);
  auto bar = [&](int i) { return base + C::kOffBar + 8u * i; };
  // T counts the tiles of scores formed, over passes and row groups; a barrier's next phase
  // waits for the one before to have been seen: S(T + bufs) for the last reading of S(T), and
  // the next keys of a slot for its last S
  auto FULL = [&](int slot) { return bar(slot); };
  auto FREE = [&](int slot) { return bar(kStages + slot); };
  auto SREADY = [&](int T) { return bar(2 * kStages + T % kBufs); };
  auto SFREE = [&](int T) { return bar(2 * kStages + kMaxBufs + T % kBufs); };
  const uint32_t QFULL = bar(2 * kStages + 2 * kMaxBufs);
  auto GATHERED = [&](int grp) { return bar(2 * kStages + 2 * kMaxBufs + 1 + (grp & 1)); };
  auto parS = [](int T) { return static_cast<uint32_t>((T / kBufs) & 1); };
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(smem + C::kOffMisc);
  float2* part = reinterpret_cast<float2*>(smem + C::kOffPart);
  float2* gather = reinterpret_cast<float2*>(smem + C::kOffGather);
  float* nlse = reinterpret_cast<float*>(smem + C::kOffLse);

  constexpr bool kEven = kPass != kBoth;
  const int rank = kEven ? 0 : blockIdx.x, csize = kEven ? 1 : gridDim.x;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (warp == 0 && lane == 0) {
    for (int s = 0; s < kStages; ++s) {
      mbar_init(FULL(s), 1);
      mbar_init(FREE(s), 1);
    }
    for (int i = 0; i < kBufs; ++i) {
      mbar_init(SREADY(i), 1);
      mbar_init(SFREE(i), C::kTurned ? 4 : kSoftWarps);  // the warps that read the buffer
    }
    mbar_init(QFULL, kSoftWarps);
    mbar_init(GATHERED(0), 1);
    mbar_init(GATHERED(1), 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  __syncwarp();
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(tmem_slot)), "r"(512)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  if (!kEven) cluster_arrive_relaxed();  // waited for before the first store into another CTA
  griddep_wait();  // nothing before this touches global memory
  const Scenes scenes{a.len, a.committed, a.B, a.R, a.cap, a.Hkv};
  Shares shares = {};
  Walk<kPass == kWeights> walk = {};
  Span one = {};
  bool valid = true;
  int counted = a.R;  // rows that count
  if constexpr (kEven) {
    shares = shares_of(scenes, lane, gridDim.x);
    walk.begin(scenes, shares, lane);
  } else {
    one.b = blockIdx.z;
    one.unit = blockIdx.y;
    one.n_keys = __ldcg(a.len + one.b);
    if (a.committed) counted = __ldcg(a.committed + one.b);
    valid = one.n_keys >= a.R && one.n_keys <= a.cap && counted >= 0 && counted <= a.R;
    const int nblk32 = valid ? (one.n_keys + 31) / 32 : 0;
    const int blk_begin = static_cast<int>(static_cast<long long>(rank) * nblk32 / csize);
    const int blk_end = static_cast<int>(static_cast<long long>(rank + 1) * nblk32 / csize);
    one.key_begin = blk_begin * 32;
    one.key_end = min(blk_end * 32, valid ? one.n_keys : 0);
    one.n_tiles = (blk_end - blk_begin + 3) / 4;
  }
  // What a run of keys takes: its row groups, and the tiles of scores that each forms. A
  // second reading goes backwards, and the next group's first forwards again: what was read
  // last is the likeliest to be in L2 still, and the last tiles are in their slots.
  struct Work {
    int m_rows, n_groups, n_tiles, formed;
    bool resident;
  };
  struct Use {  // of a tile's keys, for the j-th tile of scores of a group
    int tile, slot;
    bool second, load, last;  // in pass B; not in its slot yet; the slot's last before another load
  };
  auto use_of = [](const Work& w, int grp, int j, int T) {
    Use u;
    const int n = w.n_tiles, keep = min(n, kStages);
    u.second = kPass == kWeights || j >= n;
    u.tile = kPass == kWeights ? n - 1 - j : (u.second ? 2 * n - 1 - j : j);
    u.slot = (kEven ? T : u.tile) % kStages;
    u.load = kEven || (w.resident ? grp == 0 || n > kStages : (u.second ? u.tile < n - keep : grp == 0 || u.tile >= keep));
    u.last = kEven || (w.resident ? n > kStages : (u.second ? u.tile >= keep : u.tile < n - keep));
    return u;
  };
  auto work_of = [&](const Span& r) {
    Work w;
    if (kEven && a.committed) counted = __ldcg(a.committed + r.b);
    w.m_rows = valid ? counted * a.G : 0;  // the packed rows that count
    w.n_groups = kEven ? 1 : max(1, (w.m_rows + kR - 1) / kR);  // (no rows: the weights from before still move on)
    w.n_tiles = r.n_tiles;
    w.resident = !kEven && !C::kTurned && r.n_tiles <= kBufs;
    w.formed = r.n_tiles * (kEven || w.resident ? 1 : 2);
    return w;
  };
  // f(run) for every run of this CTA
  auto for_runs = [&](auto f) {
    if constexpr (kEven) {
#pragma unroll 1
      while (walk.left > 0) f(walk.next(scenes));
    } else {
      f(one);
    }
  };
  tc_fence_before();
  __syncthreads();
  tc_fence_after();

  if (warp == 0) {
    // -------------------------------------------------------------- producer
    if constexpr (kPass == kSums) {
      if (blockIdx.x == 0)
        for (int b = lane; b < a.B; b += 32)
          if (keys_of(scenes, b) == 0) {
            const int n = __ldcg(a.len + b);
            sd_set_error(n >= a.R && n <= a.cap ? SD_DEVERR_ROLLBACK : SD_DEVERR_LENGTH);
          }
    }
    if (!valid && rank == 0 && lane == 0 && one.unit == 0)
      sd_set_error(one.n_keys >= a.R && one.n_keys <= a.cap ? SD_DEVERR_ROLLBACK : SD_DEVERR_LENGTH);
    int T = 0;
    uint32_t held = 0, phase = 0;  // slots that have been loaded; the phases of FREE
    for_runs([&](const Span& r) {
      const Work w = work_of(r);
      const int z = r.b * a.Hkv + r.unit;
#pragma unroll 1
      for (int grp = 0; grp < w.n_groups; ++grp)
#pragma unroll 1
        for (int j = 0; j < w.formed; ++j, ++T) {
          const Use u = use_of(w, grp, j, T);
          if (!u.load) continue;
          if ((held >> u.slot) & 1) {
            mbar_wait(FREE(u.slot), (phase >> u.slot) & 1);
            phase ^= 1u << u.slot;
          }
          held |= 1u << u.slot;
          const int key0 = r.key_begin + u.tile * kTile;
          const int boxes = (min(kTile, r.key_end - key0) + 31) / 32;  // of 32 keys, as many as there are
          if (lane == 0) mbar_expect_tx(FULL(u.slot), static_cast<uint32_t>(boxes * 32 * 128 * kHalves));
          __syncwarp();
          if (lane < boxes * kHalves) {
            const int h = lane / boxes, x = lane - h * boxes;
            asm volatile(
                "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];" ::"r"(
                    base + u.slot * kK + h * kHalf + x * 32 * 128),
                "l"(reinterpret_cast<uint64_t>(&tm_k)), "r"(FULL(u.slot)), "r"(h * 64), "r"(key0 + x * 32), "r"(z)
                : "memory");
          }
          __syncwarp();
        }
    });
  } else if (warp == 1) {
    // -------------------------------------------------------------- S issue
    const uint32_t tmem = *tmem_slot;
    const uint64_t dK0 = umma_desc(base, 16, 1024);
    const uint64_t dQ = umma_desc(base + C::kOffQ, 16, 1024);
    int T = 0, n_q = 0;
    uint32_t phase = 0;  // of FULL
    for_runs([&](const Span& r) {
      const Work w = work_of(r);
#pragma unroll 1
      for (int grp = 0; grp < w.n_groups; ++grp)
#pragma unroll 1
        for (int j = 0; j < w.formed; ++j, ++T) {
          const Use u = use_of(w, grp, j, T);
          if (j == 0) mbar_wait(QFULL, n_q++ & 1);
          if (T >= kBufs) mbar_wait(SFREE(T), parS(T - kBufs));
          if (u.load) {
            mbar_wait(FULL(u.slot), (phase >> u.slot) & 1);
            phase ^= 1u << u.slot;
          }
          tc_fence_after();
          const uint64_t dk = dK0 + static_cast<uint64_t>((u.slot * kK) >> 4);
          const bool turned = C::kTurned && !u.second;  // (both operands 128 rows of one layout)
          const uint64_t da = turned ? dQ : dk, db = turned ? dk : dQ;
          const int half_a = turned ? C::kQHalf : kHalf, half_b = turned ? kHalf : C::kQHalf;
          if (elect_one()) {
#pragma unroll
            for (int kk = 0; kk < kDim / 16; ++kk)
              umma(tmem + kR * (T % kBufs), da + (((kk >> 2) * half_a + (kk & 3) * 32) >> 4),
                   db + (((kk >> 2) * half_b + (kk & 3) * 32) >> 4), kIdesc, kk > 0 ? 1 : 0);
            umma_commit(SREADY(T));
            if (u.last) umma_commit(FREE(u.slot));
          }
          __syncwarp();
        }
    });
  } else {
    // -------------------------------------------------------------- softmax
    const uint32_t tmem = *tmem_slot;
    const int st = static_cast<int>(threadIdx.x) - kSoft0;
    const int slice = st >> 7;           // pass A: rows slice * kRpt ..; pass B: tiles t % 4 == slice
    const int quarter = warp & 3;
    const int kl = quarter * 32 + lane;
    const uint32_t lane_off = static_cast<uint32_t>(quarter * 32) << 16;
    auto gdiv = [&](int p) { return __float2int_rz((static_cast<float>(p) + 0.5f) * a.inv_g); };
    const uint64_t c2 = [&] {
      uint64_t d;
      asm("mov.b64 %0, {%1, %1};" : "=l"(d) : "f"(a.scale_log2));
      return d;
    }();
    auto pack2 = [](float x0, float x1) {
      uint64_t d;
      asm("mov.b64 %0, {%1, %2};" : "=l"(d) : "f"(x0), "f"(x1));
      return d;
    };
    auto sum2 = [](uint64_t d) {
      float x0, x1;
      asm("mov.b64 {%0, %1}, %2;" : "=f"(x0), "=f"(x1) : "l"(d));
      return x0 + x1;
    };
    auto scaled = [&](float x0, float x1, float n0, float n1, float& y0, float& y1) {  // x * c + n, in pairs
      uint64_t y;
      asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(y) : "l"(pack2(x0, x1)), "l"(c2), "l"(pack2(n0, n1)));
      asm("mov.b64 {%0, %1}, %2;" : "=f"(y0), "=f"(y1) : "l"(y));
    };
    auto add2 = [&](uint64_t s, float x0, float x1) {
      uint64_t d;
      asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(s), "l"(pack2(x0, x1)));
      return d;
    };
    int T_run = 0;  // tiles formed before this run
    for_runs([&](const Span& r) {
      const Work w = work_of(r);
      const int b = r.b, kvh = r.unit, n_keys = r.n_keys, key_begin = r.key_begin, key_end = r.key_end;
      const int n_tiles = w.n_tiles, m_rows = w.m_rows;
      const bool resident = w.resident;
      const long long plane = static_cast<long long>(b) * a.Hkv + kvh;
#pragma unroll 1
      for (int grp = 0; grp < w.n_groups; ++grp) {
        const int p0 = grp * kR, T0 = T_run + grp * w.formed;
        const int rows_in = max(0, min(kR, m_rows - p0));
        // ---- the group's query rows (zero past the last that counts)
        constexpr int kChunks = kDim / 8, kQc = (kR * kChunks + kSoftThreads - 1) / kSoftThreads;
        uint4 qv[kQc];
#pragma unroll
        for (int u = 0; u < kQc; ++u) {
          const int idx = st + u * kSoftThreads, row = idx / kChunks, p = p0 + row;
          qv[u] = make_uint4(0, 0, 0, 0);
          if (row < rows_in) {
            const int i = gdiv(p);
            qv[u] = __ldcg(reinterpret_cast<const uint4*>(
                a.q + ((static_cast<long long>(b) * a.R + i) * a.Hq + kvh * a.G + (p - i * a.G)) * kDim + (idx % kChunks) * 8));
          }
        }
#pragma unroll
        for (int u = 0; u < kQc; ++u) {
          const int idx = st + u * kSoftThreads, row = idx / kChunks, c = idx % kChunks;
          if (row < kR)
            st_shared_v4(base + C::kOffQ + (c >> 3) * C::kQHalf + row * 128 + (((c & 7) ^ (row & 7)) << 4), qv[u].x, qv[u].y,
                         qv[u].z, qv[u].w);
        }
        if (T0 == 0 && st == 0) griddep_launch();  // every older kernel has finished: the next may launch
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
        if (lane == 0) mbar_arrive(QFULL);
        // rows of the group below which a key is masked (kR: all)
        auto first_row = [&](int key) {
          if (key >= key_end) return kR;
          const int i = key - (n_keys - a.R);
          return i <= 0 ? 0 : static_cast<int>(min(static_cast<long long>(kR), max(0ll, static_cast<long long>(i) * a.G - p0)));
        };
        auto masked_tile = [&](int t) { return key_begin + (t + 1) * kTile > min(key_end, n_keys - a.R + 1); };

        // ---- pass A
        if constexpr (kPass == kWeights) {
          // (the sums of all shares are there)
        } else if constexpr (C::kTurned) {
          // this thread's row: its reference and sum over every fourth tile's keys (with a quarter
          // of every tile the 16 warps met at each tile, and its chain of latencies set the pace:
          // 53.8 us for eight scenes of 8192 keys)
          float ref = -INFINITY, l = 0.f;
          const bool idle = quarter * 32 >= rows_in;
          // keys below this one are seen
          const int seen = kl < rows_in ? min(key_end, n_keys - a.R + gdiv(p0 + kl) + 1) : key_end;
          auto fold = [&](float* x, int lim, bool masks) {
            if (masks) {  // whatever the score, NaN included
#pragma unroll
              for (int j = 0; j < 16; ++j)
                if (j >= lim) x[j] = -INFINITY;
            }
            auto sum = [&] {
              uint64_t s0 = 0ull, s1 = 0ull;
#pragma unroll
              for (int j = 0; j < 16; j += 4) {
                float y[4];
                scaled(x[j], x[j + 1], -ref, -ref, y[0], y[1]);
                scaled(x[j + 2], x[j + 3], -ref, -ref, y[2], y[3]);
                s0 = add2(s0, ex2(y[0]), ex2(y[1]));
                s1 = add2(s1, ex2(y[2]), ex2(y[3]));
              }
              return sum2(s0) + sum2(s1);
            };
            // relative to the present reference, unless there is none (the sum is then
            // infinite, or not a number) or scores lie too far above it
            float s = sum();
            if (!(s < kHuge)) {
              float m = x[0];
#pragma unroll
              for (int j = 1; j < 16; ++j) m = fmaxf(m, x[j]);
              m *= a.scale_log2;
              if (m > ref) {
                l *= ref == -INFINITY ? 0.f : ex2(ref - m);
                ref = m;
              }
              if (ref > -INFINITY) {
                s = sum();
              } else {
                s = 0.f;  // no key seen, or no number among them: NaN stays
#pragma unroll
                for (int j = 0; j < 16; ++j) s += x[j] == -INFINITY ? 0.f : x[j] * 0.f;
              }
            }
            l += s;
          };
#pragma unroll 1
          for (int t = slice; t < n_tiles; t += kSlices) {
            const int T = T0 + t;
            mbar_wait(SREADY(T), parS(T));
            tc_fence_after();
            if (!idle) {
              const int lim = seen - (key_begin + t * kTile);
              const bool masks = masked_tile(t);
              const uint32_t ts = tmem + kR * (T % kBufs) + lane_off;
              float x[2][16];
              auto load = [&](int c, float* to) {
                tmem_ld8(ts + 16 * c, to);
                tmem_ld8(ts + 16 * c + 8, to + 8);
              };
              load(0, x[0]);
#pragma unroll 1
              for (int c = 0; c < kTile / 16; c += 2) {  // a chunk's scores on their way while the one before is summed
                tmem_wait_ld<16>(x[0]);
                load(c + 1, x[1]);
                fold(x[0], lim - 16 * c, masks);
                tmem_wait_ld<16>(x[1]);
                if (c + 2 < kTile / 16) load(c + 2, x[0]);
                fold(x[1], lim - 16 * c - 16, masks);
              }
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(SFREE(T));
          }
          part[kl * 4 + slice] = make_float2(ref, l);
        } else {
          // references and sums of this key lane
          float ref[kRpt], l[kRpt];
#pragma unroll
          for (int j = 0; j < kRpt; ++j) {
            ref[j] = kNone;
            l[j] = 0.f;
          }
          const bool idle = slice * kRpt >= rows_in;
#pragma unroll 1
          for (int t = 0; t < n_tiles; ++t) {
            const int T = T0 + t;
            mbar_wait(SREADY(T), parS(T));
            tc_fence_after();
            if (!idle) {
              const int below = masked_tile(t) ? first_row(key_begin + t * kTile + kl) - slice * kRpt : 0;
              float x[kRpt];
#pragma unroll
              for (int u = 0; u < kRpt; u += 8) tmem_ld8(tmem + kR * (T % kBufs) + slice * kRpt + u + lane_off, x + u);
              tmem_wait_ld<kRpt>(x);
#pragma unroll
              for (int u = 0; u < kRpt; u += 8) {
                float y[8];
#pragma unroll
                for (int j = 0; j < 8; j += 2) scaled(x[u + j], x[u + j + 1], -ref[u + j], -ref[u + j + 1], y[j], y[j + 1]);
                if (below > u) {  // whatever the score, NaN included
#pragma unroll
                  for (int j = 0; j < 8; ++j)
                    if (u + j < below) y[j] = -INFINITY;
                }
                const float m = fmaxf(fmaxf(fmaxf(y[0], y[1]), fmaxf(y[2], y[3])), fmaxf(fmaxf(y[4], y[5]), fmaxf(y[6], y[7])));
                if (m > kFar) {  // the first score, or one far above it: the new reference
#pragma unroll
                  for (int j = 0; j < 8; ++j)
                    if (y[j] > kFar) {
                      const float now = x[u + j] * a.scale_log2;
                      l[u + j] *= ex2(ref[u + j] - now);
                      ref[u + j] = now;
                      y[j] = now - now;  // (a score of +inf: NaN)
                    }
                }
#pragma unroll
                for (int j = 0; j < 8; ++j) l[u + j] += ex2(y[j]);
              }
            }
            if (!resident) {
              tc_fence_before();
              __syncwarp();
              if (lane == 0) mbar_arrive(SFREE(T));
            }
          }
          // the rows' (m, l) over the warp's lanes
#pragma unroll
          for (int u = 0; u < kRpt; u += 8) {
            float v[8], mine = -INFINITY;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
              const float m = warp_max(ref[u + j]);  // (a lane whose every score is NaN has no reference, and a sum that is NaN)
              v[j] = l[u + j] * ex2(ref[u + j] - m);
              if ((lane >> 2) == j) mine = m;
            }
            const float s = warp_sum8(v, lane);
            if ((lane & 3) == 0) part[(slice * kRpt + u + (lane >> 2)) * 4 + quarter] = make_float2(mine, s);
          }
        }
        if (kPass != kWeights) named_bar_sync(2, kSoftThreads);
        if (!kEven && grp == 0) cluster_wait();  // every CTA of the cluster has started
        // ---- (m, l) over 4 or 16 lanes; NaN stays, in l
        auto joined = [&](float2 x, int lanes) {
          float m = x.x;
          for (int o = 1; o < lanes; o <<= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
          float l = x.y * (x.x == -INFINITY ? 0.f : ex2(x.x - m));
          for (int o = 1; o < lanes; o <<= 1) l += __shfl_xor_sync(0xffffffffu, l, o);
          return make_float2(m, l);
        };
        if constexpr (kPass == kBoth) {
          float2* box = gather + (grp & 1) * kMaxCluster * kR;
          // to every CTA of the cluster, this one too: the stores complete on its barrier. (A CTA
          // sends a group's sums when it has read the boxes of the one before, so those of two
          // groups before are free)
          if (st == 0) mbar_expect_tx(GATHERED(grp), static_cast<uint32_t>(csize * kR * 8));
          if (st < 4 * kR) {  // (whole warps)
            const int row = st >> 2;
            const float2 ml = joined(part[st], 4);
            for (int to = st & 3; to < csize; to += 4)
              asm volatile("st.async.weak.shared::cluster.mbarrier::complete_tx::bytes.v2.f32 [%0], {%1, %2}, [%3];" ::"r"(
                               cluster_map(smem_addr(box + rank * kR + row), to)),
                           "f"(ml.x), "f"(ml.y), "r"(cluster_map(GATHERED(grp), to))
                           : "memory");
          }
          mbar_wait(GATHERED(grp), (grp >> 1) & 1);
#pragma unroll
          for (int r0 = 0; r0 < kR; r0 += kSoftThreads / kMaxCluster) {
            const int row = r0 + (st >> 4), from = st & 15;
            const float2 ml = joined(from < csize ? box[from * kR + row] : make_float2(-INFINITY, 0.f), kMaxCluster);
            // rows that do not count give no weight
            if (from == 0) nlse[row] = row < rows_in ? -(ml.x + lg2(ml.y)) : -INFINITY;
          }
          named_bar_sync(2, kSoftThreads);
        } else if (st < 4 * kR) {  // (whole warps)
          // a run's sums lie at its unit's number + its CTA's: no two runs share one
          const int row = st >> 2;
          float2* sums = a.sums + static_cast<long long>(b * a.Hkv + kvh) * kR + row;
          if constexpr (kPass == kSums) {
            const float2 ml = joined(part[st], 4);
            if ((st & 3) == 0) __stcg(sums + static_cast<long long>(blockIdx.x) * kR, ml);
          } else {
            // of the unit's shares, every fourth to a lane
            float2 ml = make_float2(-INFINITY, 0.f);
            const int c_last = shares.cta_of(r.first + tiles_of(n_keys) - 1);
            for (int c = shares.cta_of(r.first) + (st & 3); c <= c_last; c += 4) {
              const float2 x = __ldcg(sums + static_cast<long long>(c) * kR);
              const float m = fmaxf(ml.x, x.x);
              ml.y = ml.y * (ml.x == -INFINITY ? 0.f : ex2(ml.x - m)) + x.y * (x.x == -INFINITY ? 0.f : ex2(x.x - m));
              ml.x = m;
            }
            ml = joined(ml, 4);
            if ((st & 3) == 0) nlse[row] = row < rows_in ? -(ml.x + lg2(ml.y)) : -INFINITY;
          }
        }
        if (kPass == kWeights) named_bar_sync(2, kSoftThreads);


        // ---- pass B: the keys' weights
#pragma unroll 1
        for (int i = 0; kPass != kSums && i < n_tiles; ++i) {
          const int t = resident ? i : n_tiles - 1 - i;
          const int T = T0 + i + (resident || kEven ? 0 : n_tiles);
          if (C::kTurned && (t & 3) != slice) continue;
          if (!resident) {
            mbar_wait(SREADY(T), parS(T));
            tc_fence_after();
          }
          if ((t & 3) == slice) {
            const int key = key_begin + t * kTile + kl;
            const int below = masked_tile(t) ? first_row(key) : 0;
            const long long at = plane * a.cap + key;
            float before = 0.f;
            if (key < key_end) {
              if (grp > 0) before = a.out[at];
              else if (a.in && key < n_keys - a.R) before = __ldcg(a.in + at) * a.decay;
            }
            uint64_t w0 = 0ull, w1 = 0ull;
            const int units = (rows_in + 7) / 8;
            float x[2][8];
            auto load = [&](int u, float* to) { tmem_ld8(tmem + kR * (T % kBufs) + 8 * u + lane_off, to); };
            auto add = [&](int u, const float* x, bool masks) {
              const float4 n0 = *reinterpret_cast<const float4*>(nlse + 8 * u), n1 = *reinterpret_cast<const float4*>(nlse + 8 * u + 4);
              float y[8];
              scaled(x[0], x[1], n0.x, n0.y, y[0], y[1]);
              scaled(x[2], x[3], n0.z, n0.w, y[2], y[3]);
              scaled(x[4], x[5], n1.x, n1.y, y[4], y[5]);
              scaled(x[6], x[7], n1.z, n1.w, y[6], y[7]);
#pragma unroll
              for (int j = 0; j < 8; ++j) y[j] = ex2(y[j]);
              if (masks) {  // (a score that is masked or no row's may be NaN)
#pragma unroll
                for (int j = 0; j < 8; ++j)
                  if (8 * u + j < below || 8 * u + j >= rows_in) y[j] = 0.f;
              }
              w0 = add2(add2(w0, y[0], y[1]), y[2], y[3]);
              w1 = add2(add2(w1, y[4], y[5]), y[6], y[7]);
            };
            auto all = [&](bool masks) {  // a unit's scores on their way while the one before is summed
              if (units > 0) load(0, x[0]);
#pragma unroll 1
              for (int u = 0; u < units; u += 2) {
                tmem_wait_ld<8>(x[0]);
                if (u + 1 < units) load(u + 1, x[1]);
                add(u, x[0], masks);
                if (u + 1 < units) {
                  tmem_wait_ld<8>(x[1]);
                  if (u + 2 < units) load(u + 2, x[0]);
                  add(u + 1, x[1], masks);
                }
              }
            };
            if (masked_tile(t) || (rows_in & 7)) all(true);
            else all(false);
            if (key < key_end) a.out[at] = before + (sum2(w0) + sum2(w1));
          }
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(SFREE(T));
        }
        named_bar_sync(2, kSoftThreads);  // nlse, part and the query rows are free again
      }
      T_run += w.n_groups * w.formed;
    });
  }
  if (!kEven && warp < kFirstSoft) cluster_wait();
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(*tmem_slot), "r"(512) : "memory");
  }
}

// ------------------------------------------------------------------ host
constexpr int kEvenAbove = 32;  // rows up to which a batch never takes even shares (pick_cluster)

template <int kR, int kDim>
bool allow() {
  constexpr int smem = Cfg<kR, kDim>::kSmemBytes;
  const void* k = reinterpret_cast<const void*>(key_weights_kernel<kR, kDim, kBoth>);
  bool ok = cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, smem) == cudaSuccess &&
            cudaFuncSetAttribute(k, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) == cudaSuccess;
  if constexpr (kR > kEvenAbove) {
    const void* k1 = reinterpret_cast<const void*>(key_weights_kernel<kR, kDim, kSums>);
    const void* k2 = reinterpret_cast<const void*>(key_weights_kernel<kR, kDim, kWeights>);
    ok = ok && cudaFuncSetAttribute(k1, cudaFuncAttributeMaxDynamicSharedMemorySize, smem) == cudaSuccess &&
         cudaFuncSetAttribute(k2, cudaFuncAttributeMaxDynamicSharedMemorySize, smem) == cudaSuccess;
  }
  if (!ok) (void)cudaGetLastError();
  return ok;
}

constexpr int kClusterSizes[] = {1, 2, 3, 4, 5, 6, 8, 10, 12, 16};
constexpr int kNumSizes = sizeof(kClusterSizes) / sizeof(int);

template <int kR, int kDim>
bool active_clusters(int* active) {
  if (!allow<kR, kDim>()) return false;
  for (int i = 0; i < kNumSizes; ++i) {
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = kClusterSizes[i];
    attr[0].val.clusterDim.y = 1;
    attr[0].val.clusterDim.z = 1;
    cfg.gridDim = dim3(kClusterSizes[i], 1, 1);
    cfg.blockDim = dim3(kThreads, 1, 1);
    cfg.dynamicSmemBytes = Cfg<kR, kDim>::kSmemBytes;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    if (cudaOccupancyMaxActiveClusters(&active[i], reinterpret_cast<const void*>(key_weights_kernel<kR, kDim, kBoth>), &cfg) != cudaSuccess) {
      (void)cudaGetLastError();
      active[i] = 0;
    }
  }
  return true;
}

// What the launches need, once per device: the attributes, and how many clusters of each
// size fit at once (one CTA an SM whatever the rows).
struct DevState {
  std::once_flag once;
  bool ok = false;
  int active[kNumSizes] = {};
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
    s.ok = allow<32, 64>() && allow<64, 64>() && allow<128, 64>() && allow<32, 128>() && allow<64, 128>() &&
           active_clusters<128, 128>(s.active);
  });
  return s.ok ? &s : nullptr;
}

// Cluster size: the one forced by sd_set_cluster_size, else the least waves x (a fixed
// cost + a cost a tile, in us), the tile's as measured: on 32, 64 and 128 rows, more where
// the scores are formed twice and where more waves than one share the memory. (One scene of
// 8 heads, L = 4096, at 4 / 6 / 8 / 16: 10.7 / 9.2 / 7.4 / 12.3 us; eight scenes, L = 8192,
// at 2 / 4 / 8: 43 / 38 / 57 on 32 rows, 51 / 53 / 75 on 64, 52 / 56 / 89 on 128.) 0: even
// shares, where those cost less and the call may have them. Clusters / even shares in us, 8
// heads of 8192 keys (3/4 to all of them filled, in a cache with room for a few more): 128
// rows, 8 scenes 52 / 54, 12: 90 / 74, 16: 93 / 91, 24: 145 / 135, 24 of 2048 keys 55 / 53,
// 16: 30 / 37; 64 rows, 8: 43 / 47, 12: 78 / 65, 24: 124 / 119. Not for 32 rows, whose scores
// clusters of 4 form once: 12: 56 / 62, 24: 113 / 115 (but where the room makes a CTA's
// tiles 17 the choice above is 1, for 72 and 120).
int pick_cluster(const int* active, long long units, int cap, int rows, bool may) {
  const int forced = sd_internal_forced_cluster();
  for (int i = 0; i < kNumSizes && forced > 0; ++i)
    if (kClusterSizes[i] == forced && active[i] > 0) return forced;
  const int n_tiles = (cap + kTile - 1) / kTile;
  double best_cost = -1;
  int best = 1;
  for (int i = 0; i < kNumSizes; ++i) {
    const int cs = kClusterSizes[i];
    if (active[i] <= 0 || (cs > 1 && n_tiles < cs)) continue;
    const double waves = static_cast<double>((units + active[i] - 1) / active[i]);
    const double tiles = static_cast<double>(n_tiles) / cs;
    const bool once = rows < 128 && tiles <= 512.0 / rows;
    const double a_tile = (rows == 32 ? (once ? 0.85 : 1.22) : (rows == 64 ? (once ? 1.1 : 1.47) : 1.5)) +
                          (waves > 1 ? (rows == 32 ? 0.45 : 0.7) : 0.0);
    const double cost = waves * (4.0 + a_tile * tiles);
    if (best_cost < 0 || cost < best_cost) {
      best_cost = cost;
      best = cs;
    }
  }
  const double tiles = static_cast<double>(units) * n_tiles;
  if (may && active[0] > 1 && tiles < 2e9 && rows > kEvenAbove && 14.0 + 1.45 * tiles / active[0] < best_cost) return 0;
  return best;
}

// [planes][cap][D] bf16 keys in boxes of 64 columns x 32 rows, 128-byte swizzle
bool make_key_map(CUtensorMap* map, void* k, int D, int cap, int planes) { return make_map(map, k, cap, planes, 32, D); }

// cs: CTAs a cluster, 0: even shares over `ctas`
template <int kR, int kDim>
sd_status launch(const sd_kv_cache* c, const Args& a, int cs, int ctas, cudaStream_t stream) {
  CUtensorMap k;
  if (!make_key_map(&k, c->k, kDim, c->capacity, c->batch * c->n_kv_heads)) return SD_ERR_CUDA;
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = cs;
  attr[1].val.clusterDim.y = 1;
  attr[1].val.clusterDim.z = 1;
  cfg.gridDim = cs > 0 ? dim3(cs, c->n_kv_heads, c->batch) : dim3(ctas);
  cfg.blockDim = dim3(kThreads, 1, 1);
  cfg.dynamicSmemBytes = Cfg<kR, kDim>::kSmemBytes;
  cfg.stream = stream;
  cfg.attrs = attr;
  cfg.numAttrs = cs > 0 ? 2 : 1;
  cudaError_t e = cudaErrorInvalidValue;
  if (cs > 0) {
    e = cudaLaunchKernelEx(&cfg, key_weights_kernel<kR, kDim, kBoth>, k, a);
  } else if constexpr (kR > kEvenAbove) {
    e = cudaLaunchKernelEx(&cfg, key_weights_kernel<kR, kDim, kSums>, k, a);
    if (e == cudaSuccess) e = cudaLaunchKernelEx(&cfg, key_weights_kernel<kR, kDim, kWeights>, k, a);
  }
  if (e != cudaSuccess) {
    (void)cudaGetLastError();
    return SD_ERR_CUDA;
  }
  return SD_OK;
}

template <int kDim>
sd_status launch_rows(const sd_kv_cache* c, const Args& a, int cs, int ctas, cudaStream_t stream) {
  if (a.M <= 32) return launch<32, kDim>(c, a, cs, ctas, stream);
  if (a.M <= 64) return launch<64, kDim>(c, a, cs, ctas, stream);
  return launch<128, kDim>(c, a, cs, ctas, stream);
}
int tile_rows(int M) { return M <= 32 ? 32 : (M <= 64 ? 64 : 128); }

// How a shape is taken on the current device.
struct Plan {
  int cs, ctas;  // cs 0: even shares over `ctas` CTAs
  size_t ws_bytes;
};
sd_status make_plan(int B, int Hkv, int M, int cap, bool may, Plan* p) {
  DevState* dev = state();
  if (!dev) return SD_ERR_CUDA;
  const long long units = static_cast<long long>(B) * Hkv;
  p->cs = pick_cluster(dev->active, units, cap, tile_rows(M), may && M <= 128);
  p->ctas = dev->active[0];
  p->ws_bytes = p->cs == 0 ? static_cast<size_t>(units + p->ctas) * tile_rows(M) * sizeof(float2) : 0;
  return SD_OK;
}

}  // namespace

extern "C" size_t sd_attention_weights_workspace(int B, int R, int Hq, int Hkv, int D, int capacity) {
  if (B <= 0 || R <= 0 || Hkv <= 0 || Hq <= 0 || Hq % Hkv || (D != 64 && D != 128) || capacity <= 0 || B > 65535 || Hkv > 65535 ||
      static_cast<long long>(Hq / Hkv) * R > 128)
    return 0;
  Plan p = {};
  return make_plan(B, Hkv, Hq / Hkv * R, capacity, true, &p) == SD_OK ? p.ws_bytes : 0;
}

extern "C" sd_status sd_attention_weights_ex(const void* q, const sd_kv_cache* cache, int R, int Hq, float scale,
                                             const int32_t* committed, const float* weights_in, float decay,
                                             float* weights, void* workspace, size_t ws_bytes, sd_stream_t stream) {
  if (!cache) return SD_ERR_INVALID_ARG;
  const int B = cache->batch, Hkv = cache->n_kv_heads, D = cache->head_dim, cap = cache->capacity;
  if (B < 0 || R <= 0 || Hq <= 0 || Hkv <= 0 || cap <= 0 || Hq % Hkv) return SD_ERR_INVALID_ARG;
  if (D != 64 && D != 128) return SD_ERR_UNSUPPORTED;
  if (B > 65535 || Hkv > 65535 || Hq / Hkv > 4095 || static_cast<long long>(Hq / Hkv) * R > (1 << 20)) return SD_ERR_UNSUPPORTED;
  if (!(scale >= 0.f) || !isfinite(scale) || !isfinite(decay)) return SD_ERR_INVALID_ARG;
  if (B == 0) return SD_OK;
  if (!q || !cache->k || !cache->len || !weights) return SD_ERR_INVALID_ARG;
  if (!sd_aligned16(q) || !sd_aligned16(cache->k) || !sd_aligned16(weights) || !sd_aligned16(weights_in))
    return SD_ERR_INVALID_ARG;
  if (!sd_aligned16(workspace)) return SD_ERR_INVALID_ARG;
  Plan p = {};
  const sd_status planned = make_plan(B, Hkv, Hq / Hkv * R, cap, workspace != nullptr, &p);
  if (planned != SD_OK) return planned;
  if (p.ws_bytes > ws_bytes) return SD_ERR_WORKSPACE;
  const double sc = scale > 0.f ? scale : 1.0 / sqrt(static_cast<double>(D));
  Args a = {};
  a.q = static_cast<const __nv_bfloat16*>(q);
  a.len = cache->len;
  a.committed = committed;
  a.in = weights_in;
  a.out = weights;
  a.sums = static_cast<float2*>(workspace);
  a.B = B;
  a.R = R;
  a.Hq = Hq;
  a.Hkv = Hkv;
  a.G = Hq / Hkv;
  a.M = a.G * R;
  a.cap = cap;
  a.inv_g = 1.0f / static_cast<float>(a.G);
  a.scale_log2 = static_cast<float>(sc * 1.4426950408889634);
  a.decay = decay;
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  return D == 64 ? launch_rows<64>(cache, a, p.cs, p.ctas, st) : launch_rows<128>(cache, a, p.cs, p.ctas, st);
}

extern "C" sd_status sd_attention_weights(const void* q, const sd_kv_cache* cache, int R, int Hq, float scale,
                                          const int32_t* committed, const float* weights_in, float decay,
                                          float* weights, sd_stream_t stream) {
  return sd_attention_weights_ex(q, cache, R, Hq, scale, committed, weights_in, decay, weights, nullptr, 0, stream);
}
