// Attention of a drafted tree's rows over a paged cache (sm_103a, tcgen05).
//
// For row i of a scene (its position behind the prefix) and query head h of KV head g
//     o_i = sum_n softmax_n(q_i k_n scale) v_n,   n < prefix, and the ancestors of i and i.
// The G n_new rows that share a KV head are packed, so that every key is read once for up to
// 256 of them (an m-block):
//     S[128 rows][128 keys] = Q K^T        (both from shared memory, K-major)
//     O[128 rows][D]       += P V          (P from tensor memory, V MN-major)
// with one running reference and sum a row. The reference is the maximum of the first tile in
// which the row sees a key, and moves only where a later tile's weights sum to more than 2^16
// relative to it (O is then scaled in place): sums stay far inside fp32, and no tile but the
// first looks for its maximum. P is bf16, and the sum is taken over the rounded
// weights, so that they add up to 1 whatever their rounding.
//
// Two softmax groups of four warps, each with an S | P buffer and an O accumulator of its
// own. Up to 128 packed rows the groups take alternate key tiles of the same rows; with more,
// the same tile for 128 rows each. A group's next S goes where P was, so it is issued when PV
// is done; while one group's products run, the other's softmax does. With two row tiles each
// group has a warp that issues its products (a wait on a barrier, even one that is over, takes
// such a warp ~135 cycles, a commit ~150: one for both groups took 1900 cycles a product pair
// of 1024). Few rows leave most of the 128 lanes idle, so up to
// 64 (32) of them are put into the tile two (four) times, each copy with its own half
// (quarter) of the keys: its weights for the other keys are 0, and copies, groups and shares
// join at the end by one rule
//     m = max m_c,  l = sum l_c 2^(m_c - m),  o = sum O_c 2^(m_c - m) / l.
//
// Work. Few units (scene, KV head, m-block): a cluster of CTAs a unit, which split its 128-key
// tiles and join their parts through distributed shared memory. Many: one CTA an SM, the tiles
// of all units, one unit after the other, in one even share each; a unit that a share's border
// cuts leaves its parts in the workspace, and a second kernel joins them.
//
// What it takes on a GB300 (cold inputs, the device alone), and what bounds it. 32 ragged scenes
// of up to 8192 keys, 61 rows, 32 / 8 heads x 128 (1.0 GB): 205 us, 4.9 TB/s or 0.73 of a copy's
// rate. About 160 of them are the tile loop (98.6 tiles a CTA): a pair of row tiles takes 1.61 to
// 1.65 us, ~2960 cycles, a key tile, of which the exponentials (16 a cycle and SM) need 2048 and the products
// 2048: a group's weights (1280) wait for its S, and its PV and next S (1650) for the weights,
// and only the other group's stand between. The launch, a CTA's first queries and its last
// output take 15, every further run's end and start 9.8 (two row tiles; 6.5 at head dim 64), 1.7
// times a CTA here, and the parts of cut units and their joining 12 to 15. One scene of
// 131072 keys and 8 rows: 94 us, 0.86 of the copy's rate on 96 SMs. One scene of 4096 keys is
// one launch of dependent phases, 1 row 9.8 us, 26 rows 13.2 (the cluster's join of 104 rows a
// head, 55 KB into every CTA at ~16 bytes a cycle, a quarter of it).
//
// What a row does not see does not reach it: hidden scores are replaced before the maximum,
// and in the tiles that hold new rows, values that are no numbers are taken out of V (0 times
// them would be NaN) and added at the end to the rows that see them.
#include "tmem.cuh"

#include <math.h>
#include <algorithm>
#include <type_traits>

SD_DEFINE_ERROR_ACCESSOR(sd_take_error_attention_tree)

namespace {

constexpr int kMaxRows = 256;    // rows of a tree
constexpr int kTile = 128;       // keys a tile
constexpr int kSoft = 256;       // softmax threads
// warps: 8 brings keys, 9 issues products, 10 brings values (one row tile) or issues the second
// group's products (and warp 8 brings both), 11 cleans
constexpr int kProducer = 8, kProduct = 9, kSecond = 10, kCleaner = 11;
constexpr int kThreads = kSoft + 128;
constexpr int kJoin = 256;       // threads of the joining kernel
constexpr int kMaxCtas = 192;    // shares

struct TreeArgs {
  const __nv_bfloat16* q;
  __nv_bfloat16* out;
  const __nv_bfloat16* v;   // (only for values that are no numbers)
  const int32_t *table, *len, *parents, *n_new;
  long long q_stride;
  float* part;              // even shares: per CTA two parts, O [D / 4][rows][4], then (m, l) [rows][2]
  int B, R, Hq, Hkv, G, n_pages, shift, max_pages, cap, rows, row_shift, mblocks;  // rows (1 << row_shift): of an m-block
  float scale_log2, inv_g;
};

// The largest of three (NaN loses); products and sums of pairs.
__device__ __forceinline__ float max3(float a, float b, float c) {
  float d;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
  float2 d;
  asm("{\n\t.reg .b64 a, b, c, d;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\tmov.b64 c, {%6, %7};\n\t"
      "fma.rn.f32x2 d, a, b, c;\n\tmov.b64 {%0, %1}, d;\n\t}"
      : "=f"(d.x), "=f"(d.y)
      : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
  return d;
}
// Adds the two bf16 numbers of w, each to a sum of its own.
__device__ __forceinline__ void add_pair(uint32_t w, float& lo, float& hi) {
  asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %2;\n\t"
      "add.rn.f32.bf16 %0, a, %0;\n\tadd.rn.f32.bf16 %1, b, %1;\n\t}"
      : "+f"(lo), "+f"(hi)
      : "r"(w));
}
__device__ __forceinline__ void named_bar_arrive(int id, int threads) {
  asm volatile("bar.arrive %0, %1;" ::"r"(id), "r"(threads) : "memory");
}

// ------------------------------------------------------------------ shares
struct Scene {
  int n_keys, m, tiles, mblocks;  // tiles 0: not valid, or no rows that count
};
__device__ __forceinline__ Scene scene_of(const TreeArgs& a, int b) {
  Scene s;
  s.n_keys = __ldcg(a.len + b);
  s.m = a.n_new ? __ldcg(a.n_new + b) : a.R;
  const bool ok = s.m > 0 && s.m <= a.R && s.n_keys >= s.m && s.n_keys <= a.cap;
  s.tiles = ok ? (s.n_keys + kTile - 1) / kTile : 0;
  s.mblocks = (s.m * a.G + a.rows - 1) >> a.row_shift;
  if (!ok) s.n_keys = s.m = s.mblocks = 0;
  return s;
}
__device__ __forceinline__ bool length_error(const TreeArgs& a, int b) {
  const int n = __ldcg(a.len + b), m = a.n_new ? __ldcg(a.n_new + b) : a.R;
  return m < 0 || m > a.R || n < m || n > a.cap;
}

struct Plan {
  int total, each, rest;  // tiles, tiles a share, shares with one more
  __device__ __forceinline__ int begin(int cta) const { return cta * each + min(cta, rest); }
  __device__ __forceinline__ int cta_of(int pos) const {
    const int more = rest * (each + 1);
    return pos < more ? pos / (each + 1) : rest + (pos - more) / each;
  }
};

// A run of one unit's tiles in a share.
struct Run {
  int b, kvh, mb, n_keys, m, tiles;  // of the unit
  int tile0, n_tiles;                // the run
  int first;                         // the unit's first tile among all
};
struct Walk {
  int b, kvh, mb, tile, first, left;
  Scene s;
  // Cuts all tiles into even shares of `ctas` CTAs and stands at the first tile of share
  // `cta`, with its tiles to go (kOn: with all that follow). A warp; up to 32 scenes are
  // looked at once.
  template <bool kOn>
  __device__ __forceinline__ Plan begin(const TreeArgs& a, int cta, int ctas, int lane) {
    Scene mine = {};
    if (lane < a.B) mine = scene_of(a, lane);
    int n = mine.tiles * mine.mblocks * a.Hkv;
    for (int b0 = lane + 32; b0 < a.B; b0 += 32) {
      const Scene x = scene_of(a, b0);
      n += x.tiles * x.mblocks * a.Hkv;
    }
    Plan p;
    p.total = static_cast<int>(__reduce_add_sync(0xffffffffu, static_cast<uint32_t>(n)));
    p.each = p.total / ctas;
    p.rest = p.total - p.each * ctas;
    const int pos = p.begin(cta);
    left = (kOn ? p.total : p.begin(cta + 1)) - pos;
    if (left <= 0) return p;
    int before = 0;
    for (int b0 = 0; b0 < a.B; b0 += 32) {
      if (b0 > 0) {
        mine = Scene{};
        if (b0 + lane < a.B) mine = scene_of(a, b0 + lane);
      }
      const int own = mine.tiles * mine.mblocks * a.Hkv;
      int upto = own;
#pragma unroll
      for (int x = 1; x < 32; x <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, upto, x);
        if (lane >= x) upto += y;
      }
      const uint32_t past = __ballot_sync(0xffffffffu, before + upto > pos);
      if (past) {
        const int at = __ffs(past) - 1;
        b = b0 + at;
        s.n_keys = __shfl_sync(0xffffffffu, mine.n_keys, at);
        s.m = __shfl_sync(0xffffffffu, mine.m, at);
        s.tiles = __shfl_sync(0xffffffffu, mine.tiles, at);
        s.mblocks = __shfl_sync(0xffffffffu, mine.mblocks, at);
        const int in = pos - before - __shfl_sync(0xffffffffu, upto - own, at);
        const int unit = in / s.tiles;
        kvh = unit / s.mblocks;
        mb = unit - kvh * s.mblocks;
        tile = in - unit * s.tiles;
        first = pos - tile;
        return p;
      }
      before += __shfl_sync(0xffffffffu, upto, 31);
    }
    left = 0;  // (only if a length changed under the kernel)
    return p;
  }
  // Stands at the tiles that CTA `rank` of a cluster of `cs` takes of a unit.
  __device__ __forceinline__ void begin_part(const TreeArgs& a, int scene, int head, int block, int rank, int cs) {
    b = scene, kvh = head, mb = block;
    s = scene_of(a, b);
    if (mb >= s.mblocks) s.tiles = 0;
    const int each = s.tiles / cs, rest = s.tiles - each * cs;
    tile = rank * each + min(rank, rest);
    first = 0;
    left = each + (rank < rest ? 1 : 0);
  }
  __device__ __forceinline__ bool next(const TreeArgs& a, Run& r) {
    if (left <= 0) return false;
    if (tile == s.tiles) {
      first += s.tiles;
      tile = 0;
      if (++mb == s.mblocks) {
        mb = 0;
        if (++kvh == a.Hkv) {
          kvh = 0;
          do {
            if (++b >= a.B) return false;  // (only if a length changed under the kernel)
            s = scene_of(a, b);
          } while (s.tiles == 0);
        }
      }
    }
    r.b = b;
    r.kvh = kvh;
    r.mb = mb;
    r.n_keys = s.n_keys;
    r.m = s.m;
    r.tiles = s.tiles;
    r.first = first;
    r.tile0 = tile;
    r.n_tiles = min(s.tiles - tile, left);
    left -= r.n_tiles;
    tile += r.n_tiles;
    return true;
  }
};

// ------------------------------------------------------------------ configuration
// kCopies: times that the packed rows stand in the 128-row tile; kQ: row tiles.
template <int kDim, int kCopies, int kQ>
struct Cfg {
  static_assert(kCopies == 1 || kQ == 1, "copies of one tile");
  static constexpr int kRows = kTile / kCopies;            // packed rows a tile
  static constexpr int kCols = kTile / kCopies;            // keys of a tile that a lane looks at
  static constexpr int kHalf = kTile * 128;                // 64 columns of 128 rows
  static constexpr int kTileBytes = kHalf * (kDim / 64);
  static constexpr int kKSlots = kDim == 64 ? 4 : 3, kVSlots = kDim == 64 ? 4 : (kQ == 1 ? 3 : 2);
  static constexpr int kOffV = kKSlots * kTileBytes;
  static constexpr int kOffQ = kOffV + kVSlots * kTileBytes;
  static constexpr int kOffParent = kOffQ + kQ * kTileBytes;     // [256] int16
  static constexpr int kOffMl = kOffParent + kMaxRows * 2;       // [2][128] float2
  static constexpr int kOffBar = kOffMl + 2 * kTile * 8;
  static constexpr int kBars = 2 * (kKSlots + kVSlots) + 11;
  static constexpr int kOffMisc = kOffBar + kBars * 8;           // tensor memory, bad pages, [8] rows with bad values
  static constexpr int kSmem = kOffMisc + 48;
  static_assert(kSmem <= 227 * 1024, "shared memory");
  static_assert(kOffBar % 8 == 0 && kOffMisc % 8 == 0 && kOffQ % 1024 == 0, "alignment");
};
__host__ __device__ constexpr size_t part_floats(int rows, int D) { return static_cast<size_t>(rows) * (D + 2); }

// A part in a cluster's shared memory: chunk c4 of four columns of a row, the chunks of a row
// in an order of its own (rows along the lanes to write, chunks to read), and its (m, l).
template <int kDim>
__device__ __forceinline__ uint32_t cluster_o(int row, int c4) {
  return static_cast<uint32_t>(row * (kDim / 4) + (c4 ^ (row & (kDim / 4 - 1)))) * 16;
}
template <int kDim>
__device__ __forceinline__ uint32_t cluster_ml(int rows, int row) {
  return static_cast<uint32_t>(rows * kDim * 4 + row * 8);
}

// Nonzero where one of the two bf16 numbers of w is no number: its exponent, all ones, carries.
__device__ __forceinline__ uint32_t bad_pair(uint32_t w) { return ((w & 0x7f807f80u) + 0x00800080u) & 0x80008000u; }

// Sum of the values that are no numbers at column d of the bad rows that row i of scene b sees.
__device__ __noinline__ float bad_values(const TreeArgs& a, const int16_t* parent, const uint32_t* bad, int b, int kvh, int prefix,
                                         int i, int d, int dim) {
  float sum = 0.f;
  for (int j = i; j >= 0; j = a.parents ? parent[j] : j - 1) {
    if (!(bad[j >> 5] >> (j & 31) & 1)) continue;
    const int n = prefix + j, id = __ldcg(a.table + static_cast<long long>(b) * a.max_pages + (n >> a.shift));
    if (id < 0 || id >= a.n_pages) continue;
    const long long row = ((static_cast<long long>(id) * a.Hkv + kvh) << a.shift) + (n & ((1 << a.shift) - 1));
    const float v = sd_ldcg_bf16(a.v + row * dim + d);
    if (!(fabsf(v) < INFINITY)) sum += v;
  }
  return sum;
}

// Four columns of a row, joined from its parts.
struct Joined {
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
  float top = -INFINITY, total = 0.f;
  bool skip = false;  // its tree is not valid
  template <int kN>
  __device__ __forceinline__ void add(const float2 (&ml)[kN], const float4 (&v)[kN]) {
    float now = top;
#pragma unroll
    for (int u = 0; u < kN; ++u) {
      skip |= ml[u].x != ml[u].x;
      now = fmaxf(now, ml[u].x);
    }
    const float ref = now == -INFINITY ? 0.f : now, f0 = ex2(top - ref);
    o.x *= f0, o.y *= f0, o.z *= f0, o.w *= f0, total *= f0;
    top = now;
#pragma unroll
    for (int u = 0; u < kN; ++u) {
      const float f = ex2(ml[u].x - ref);
      total = fmaf(f, ml[u].y, total);
      o.x = fmaf(f, v[u].x, o.x), o.y = fmaf(f, v[u].y, o.y), o.z = fmaf(f, v[u].z, o.z), o.w = fmaf(f, v[u].w, o.w);
    }
  }
  __device__ __forceinline__ void store(__nv_bfloat16* out) const {
    const float inv = 1.f / total;
    if (!skip) *reinterpret_cast<uint2*>(out) = make_uint2(cvt_bf16x2(o.x * inv, o.y * inv), cvt_bf16x2(o.z * inv, o.w * inv));
  }
};

// ------------------------------------------------------------------ kernel
// kCluster: grid (cluster size, KV heads x m-blocks, scenes), else (shares).
template <int kDim, int kCopies, int kQ, bool kCluster>
__global__ void __launch_bounds__(kThreads, 1)
    tree_attention_kernel(const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v,
                          const __grid_constant__ TreeArgs a) {
  using C = Cfg<kDim, kCopies, kQ>;
  constexpr int kKS = C::kKSlots, kVS = C::kVSlots;
  extern __shared__ __align__(1024) uint8_t smem[];  // (the kernel has no other shared memory)
  const uint32_t base = smem_addr(smem);
  auto bar = [&](int i) { return base + C::kOffBar + 8u * i; };
  // K and V slots are filled by the producer and freed by the products that read them (one
  // arrival a row tile); SREADY, PFULL, PVDONE: one of each a group, once a tile of it. A
  // barrier tells phases by their parity only: whoever waits for a slot's phase knows that the
  // one before is over (the products take the slots in order, and a group's S comes after them)
  auto FULLK = [&](int s) { return bar(s); };
  auto FREEK = [&](int s) { return bar(kKS + s); };
  auto FULLV = [&](int s) { return bar(2 * kKS + s); };
  auto FREEV = [&](int s) { return bar(2 * kKS + kVS + s); };
  auto SREADY = [&](int g) { return bar(2 * (kKS + kVS) + g); };
  auto PFULL = [&](int g) { return bar(2 * (kKS + kVS) + 2 + g); };
  auto PVDONE = [&](int g) { return bar(2 * (kKS + kVS) + 4 + g); };
  const uint32_t QFULL = bar(2 * (kKS + kVS) + 6);  // a run's query tile, and O may be written
  // tiles with new rows, one after the other: the scores of the j-th are under way (so that its
  // values may be waited for), and its values are all numbers
  auto VTOLD = [&](int j) { return bar(2 * (kKS + kVS) + 7 + (j & 1)); };
  auto VCLEAN = [&](int j) { return bar(2 * (kKS + kVS) + 9 + (j & 1)); };
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(smem + C::kOffMisc);
  volatile uint32_t* bad_page = reinterpret_cast<uint32_t*>(smem + C::kOffMisc + 4);  // bit: a run's number mod 32
  uint32_t* bad_rows = reinterpret_cast<uint32_t*>(smem + C::kOffMisc + 8);           // [8]
  int16_t* s_parent = reinterpret_cast<int16_t*>(smem + C::kOffParent);
  float2* s_ml = reinterpret_cast<float2*>(smem + C::kOffMl);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

  if (threadIdx.x == 0) {
    for (int s = 0; s < kKS; ++s) {
      mbar_init(FULLK(s), 1);
      mbar_init(FREEK(s), kQ);
    }
    for (int s = 0; s < kVS; ++s) {
      mbar_init(FULLV(s), 1);
      mbar_init(FREEV(s), kQ);
    }
    for (int g = 0; g < 2; ++g) {
      mbar_init(SREADY(g), 1);
      mbar_init(PFULL(g), 4);
      mbar_init(PVDONE(g), 1);
    }
    mbar_init(QFULL, 1);
    for (int j = 0; j < 2; ++j) {
      mbar_init(VTOLD(j), kQ);
      mbar_init(VCLEAN(j), 1);
    }
    *const_cast<uint32_t*>(bad_page) = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  int early[4] = {};
  // tensor memory is taken after the wait for the kernel before (which may hold some) and
  // before the next kernel may come
  griddep_wait();
  if (kCluster && (warp == kProducer || warp == kSecond) && a.max_pages <= 128) {
    const int32_t* table = a.table + static_cast<long long>(blockIdx.z) * a.max_pages;
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (lane + 32 * k < a.max_pages) early[k] = __ldcg(table + lane + 32 * k);
  }
  if (warp == kProduct) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(tmem_slot)), "r"(512)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  Walk walk;
  const int unit_head = a.mblocks == 1 ? blockIdx.y : blockIdx.y / a.mblocks, unit_block = blockIdx.y - unit_head * a.mblocks;
  if (kCluster) walk.begin_part(a, blockIdx.z, unit_head, unit_block, blockIdx.x, gridDim.x);
  else walk.begin<false>(a, blockIdx.x, gridDim.x, lane);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  griddep_launch();
  const uint32_t tmem = *tmem_slot;
  const uint32_t tmem_o = tmem + 256;  // S | P of group g at column 128 g, O at 256 + kDim g

  // whether tile t of a run holds new rows (or rows behind the last key)
  auto new_rows = [](const Run& x, int t) { return (x.tile0 + t + 1) * kTile > x.n_keys - x.m; };
  Run r;
  if (warp == kProducer || (kQ == 1 && warp == kSecond)) {
    // -------------------------------------------------------------- producers
    // of keys and values: with one row tile and many copies a tile (~60 cycles each to issue;
    // pages of 16 rows take 16) each its own (one scene of 4096 keys in such pages, 1 row: 10.5 ->
    // 10.2 us; with pages of 64 and 128 rows no difference)
    const bool keys = warp == kProducer;
    const bool apart = kQ == 1 && (kTile >> a.shift) * (kDim / 64) >= 8, values = keys != apart;
    if (!keys && !values) walk.left = 0;
    if (keys && (kCluster ? blockIdx.x == 0 && blockIdx.y == 0 : blockIdx.x == 0))
      for (int b = kCluster ? blockIdx.z + 32 * lane : lane; b < (kCluster ? blockIdx.z + 1 : a.B); b += 32)
        if (length_error(a, b)) sd_set_error(SD_DEVERR_LENGTH);
    const uint64_t evict_first = l2_evict_first_policy();
    const int page = 1 << a.shift, pages = kTile >> a.shift;  // pages a tile
    int T = 0, run = 0;
    while (walk.next(a, r)) {
      const int32_t* table = a.table + static_cast<long long>(r.b) * a.max_pages;
      auto page_id = [&](int t) {  // the lane's page of tile t
        const int at = t * pages + lane;
        return lane < pages && (at << a.shift) < r.n_keys ? __ldcg(table + at) : INT32_MIN;
      };
      int id;
      if (kCluster && a.max_pages <= 128) {
        // the scene's pages were on their way before its length was known
        const int at = r.tile0 * pages + lane;
        id = INT32_MIN;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const int x = __shfl_sync(0xffffffffu, early[k], at & 31);
          if ((at >> 5) == k) id = x;
        }
      } else {
        id = page_id(r.tile0);
      }
      for (int t = 0; t < r.n_tiles; ++t, ++T) {
        const int tile = r.tile0 + t;
        const bool need = lane < pages && ((tile * pages + lane) << a.shift) < r.n_keys, ok = need && id >= 0 && id < a.n_pages;
        if (keys && __any_sync(0xffffffffu, need && !ok) && lane == 0) {
          atomicOr(const_cast<uint32_t*>(bad_page), 1u << (run & 31));
          sd_set_error(SD_DEVERR_PAGE);
        }
        const uint32_t bytes = __popc(__ballot_sync(0xffffffffu, ok)) * page * kDim * 2;
        const int z = id * a.Hkv + r.kvh;
        if (t + 1 < r.n_tiles) id = page_id(tile + 1);
        auto load = [&](const CUtensorMap* map, uint32_t full, uint32_t dst) {
          if (lane == 0) mbar_expect_tx(full, bytes);
          __syncwarp();
          if (ok) {
#pragma unroll
            for (int h = 0; h < kDim / 64; ++h)
              tma_load_3d_hint(dst + h * C::kHalf + lane * page * 128, map, full, h * 64, 0, z, evict_first);
          }
          __syncwarp();
        };
        if (keys) {
          if (T >= kKS) mbar_wait(FREEK(T % kKS), (T / kKS - 1) & 1);
          load(&tm_k, FULLK(T % kKS), base + (T % kKS) * C::kTileBytes);
        }
        if (values) {
          if (T >= kVS) mbar_wait(FREEV(T % kVS), (T / kVS - 1) & 1);
          load(&tm_v, FULLV(T % kVS), base + C::kOffV + (T % kVS) * C::kTileBytes);
        }
        // the first queries do not queue behind all the slots' keys
        if (!kCluster && T == 0 && r.n_tiles > 1) mbar_wait(QFULL, 0);
      }
      ++run;
    }
  } else if (warp == kProduct || (kQ == 2 && warp == kSecond)) {
    // -------------------------------------------------------------- products
    // of group warp - kProduct with two row tiles, else of both
    const int x0 = warp - kProduct;
    constexpr int kStep = kQ;
    constexpr uint32_t kIdescS = umma_idesc(128, kTile, 0, 0), kIdescO = umma_idesc(128, kDim, 0, 1);
    const uint64_t dK = umma_desc(base, 16, 1024), dV = umma_desc(base + C::kOffV, C::kHalf, 1024);
    const uint64_t dQ = umma_desc(base + C::kOffQ, 16, 1024);
    int n0 = 0, n1 = 0, T0 = 0, run = 0, told = 0, cleaned = 0;  // n0, n1: products of the groups so far
    while (walk.next(a, r)) {
      // item x: group x mod 2, of tile x / 2 (two row tiles) or x
      const int items = kQ * r.n_tiles;
      auto tile_of = [&](int x) { return T0 + (kQ == 2 ? x >> 1 : x); };
      auto wait_k = [&](int x) {
        const int T = tile_of(x);
        mbar_wait(FULLK(T % kKS), (T / kKS) & 1);
      };
      auto scores = [&](int x) {
        const int g = x & 1, ks = tile_of(x) % kKS;
        tc_fence_after();
        if (elect_one()) {
#pragma unroll
          for (int kk = 0; kk < kDim / 16; ++kk) {
            const uint64_t step = ((kk >> 2) * C::kHalf + (kk & 3) * 32) >> 4;
            umma(tmem + 128 * g, dQ + (kQ == 2 ? (g * C::kTileBytes) >> 4 : 0) + step, dK + ((ks * C::kTileBytes) >> 4) + step, kIdescS,
                 kk > 0 ? 1 : 0);
          }
          umma_commit(SREADY(g));
          umma_commit(FREEK(ks));
        }
        __syncwarp();
        if (new_rows(r, tile_of(x) - T0)) {
          if (lane == 0) mbar_arrive(VTOLD(told));
          ++told;
        }
      };
      mbar_wait(QFULL, run & 1);
      for (int x = x0; x < min(2, items); x += kStep) {
        wait_k(x);
        scores(x);
      }
      for (int x = x0; x < items; x += kStep) {
        const int g = x & 1, T = tile_of(x), vs = T % kVS, n = g ? n1 : n0;
        const int steps = (min(r.n_keys - (r.tile0 + T - T0) * kTile, kTile) + 15) / 16;  // 16 keys each
        mbar_wait(FULLV(vs), (T / kVS) & 1);
        if (new_rows(r, T - T0)) {
          mbar_wait(VCLEAN(cleaned), (cleaned >> 1) & 1);
          ++cleaned;
        }
        mbar_wait(PFULL(g), n & 1);
        tc_fence_after();
        if (elect_one()) {
          auto product = [&](int kk) {
            umma_ta(tmem_o + kDim * g, tmem + 128 * g + kk * 8, dV + ((vs * C::kTileBytes + kk * 2048) >> 4), kIdescO,
                    x >= 2 || kk > 0 ? 1 : 0);
          };
          if (steps == kTile / 16) {
#pragma unroll
            for (int kk = 0; kk < kTile / 16; ++kk) product(kk);
          } else {
#pragma unroll 1
            for (int kk = 0; kk < steps; ++kk) product(kk);
          }
          umma_commit(PVDONE(g));
          umma_commit(FREEV(vs));
        }
        __syncwarp();
        if (x + 2 < items) {
          wait_k(x + 2);               // (while the product runs)
          mbar_wait(PVDONE(g), n & 1); // P lies where S goes
          scores(x + 2);
        }
        if (g) ++n1;
        else ++n0;
      }
      T0 += r.n_tiles;
      ++run;
    }
  } else if (warp == kCleaner) {
    // -------------------------------------------------------------- values of the last tiles
    // V rows behind the last key (of its 16) become 0, whatever they hold, and so do values of
    // new rows that are no numbers: 0 times them would be NaN
    int T0 = 0, cleaned = 0;
    while (walk.next(a, r)) {
      const int prefix = r.n_keys - r.m;
      for (int t = 0; t < r.n_tiles; ++t) {
        if (!new_rows(r, t)) continue;
        const int T = T0 + t, key0 = (r.tile0 + t) * kTile;
        mbar_wait(VTOLD(cleaned), (cleaned >> 1) & 1);
        mbar_wait(FULLV(T % kVS), (T / kVS) & 1);
        const uint32_t tile = base + C::kOffV + (T % kVS) * C::kTileBytes;
        const int rows = min((r.n_keys - key0 + 15) / 16 * 16, kTile);  // that the product reads
        // rows lane / 8, + 4, + 8, + 12 at once, a chunk of each half a lane
        constexpr int kAt = 4, kHalves = kDim / 64;
#pragma unroll 1
        for (int row0 = max(0, prefix - key0) + lane / 8; row0 < rows; row0 += 4 * kAt) {
          uint32_t w[kAt][kHalves][4];
          auto chunk = [&](int i, int h) { return tile + h * C::kHalf + (row0 + 4 * i) * 128 + ((lane & 7) << 4); };
#pragma unroll
          for (int i = 0; i < kAt; ++i)
#pragma unroll
            for (int h = 0; h < kHalves; ++h)
              if (key0 + row0 + 4 * i < r.n_keys)
                asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];"
                             : "=r"(w[i][h][0]), "=r"(w[i][h][1]), "=r"(w[i][h][2]), "=r"(w[i][h][3])
                             : "r"(chunk(i, h)));
#pragma unroll
          for (int i = 0; i < kAt; ++i) {
            const int row = row0 + 4 * i, node = key0 + row - prefix;
            if (row >= rows) break;
#pragma unroll
            for (int h = 0; h < kHalves; ++h) {
              uint32_t(&x)[4] = w[i][h];
              if (key0 + row >= r.n_keys) {
                st_shared_v4(chunk(i, h), 0u, 0u, 0u, 0u);
              } else if (bad_pair(x[0]) | bad_pair(x[1]) | bad_pair(x[2]) | bad_pair(x[3])) {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                  if ((x[j] & 0x7f80u) == 0x7f80u) x[j] &= 0xffff0000u;
                  if ((x[j] & 0x7f800000u) == 0x7f800000u) x[j] &= 0x0000ffffu;
                }
                st_shared_v4(chunk(i, h), x[0], x[1], x[2], x[3]);
                atomicOr(&bad_rows[node >> 5], 1u << (node & 31));
              }
            }
          }
        }
        __syncwarp();
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
        if (lane == 0) mbar_arrive(VCLEAN(cleaned));
        ++cleaned;
      }
      T0 += r.n_tiles;
    }
  } else {
    // -------------------------------------------------------------- softmax
    const int g = warp >> 2, rl = threadIdx.x & 127;      // lane of the 128-row tile
    const int copy = rl / C::kRows, row = (kQ == 2 ? g * kTile : 0) + rl % C::kRows;
    const uint32_t lane_off = static_cast<uint32_t>((warp & 3) * 32) << 16;
    const uint32_t ts = tmem + 128 * g + lane_off, to = tmem_o + lane_off;
    const float sl = a.scale_log2;
    constexpr int kWords = C::kCols / 32;
    int n = 0, run = 0;
    while (walk.next(a, r)) {
      const int prefix = r.n_keys - r.m, M = r.m * a.G, p = r.mb * a.rows + row;
      const bool live = p < M;
      auto gdiv = [&](int x) { return __float2int_rz((static_cast<float>(x) + 0.5f) * a.inv_g); };  // exact below 2^21
      const int node = live ? gdiv(p) : 0;
      const bool masked_run = new_rows(r, r.n_tiles - 1);
      // ---- the packed queries; the tree where the run reaches the new rows
      static_assert(kMaxRows <= kSoft, "a row a thread");
      int up = -1;
      if (masked_run && a.parents && static_cast<int>(threadIdx.x) < r.m)
        up = __ldcg(a.parents + static_cast<long long>(r.b) * a.R + threadIdx.x);
      constexpr int kBatch = kQ * C::kRows * (kDim / 8) / kSoft;  // 16-byte chunks a thread
      {
        uint4 v[kBatch];
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
          const int x = threadIdx.x + u * kSoft, qr = x / (kDim / 8), c = x % (kDim / 8), pq = r.mb * a.rows + qr;
          v[u] = make_uint4(0, 0, 0, 0);
          if (pq < M) {
            const int i = gdiv(pq);
            v[u] = __ldcg(reinterpret_cast<const uint4*>(a.q + (static_cast<long long>(r.b) * a.R + i) * a.q_stride +
                                                         (r.kvh * a.G + pq - i * a.G) * kDim) + c);
          }
        }
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
          const int x = threadIdx.x + u * kSoft, qr = x / (kDim / 8), c = x % (kDim / 8);
#pragma unroll
          for (int cp = 0; cp < kCopies; ++cp) {
            const int at = cp * C::kRows + (qr & 127);
            st_shared_v4(base + C::kOffQ + (kQ == 2 ? (qr >> 7) * C::kTileBytes : 0) + (c >> 3) * C::kHalf + at * 128 +
                             (((c & 7) ^ (at & 7)) << 4),
                         v[u].x, v[u].y, v[u].z, v[u].w);
          }
        }
      }
      const bool wrong = up < -1 || up >= static_cast<int>(threadIdx.x);
      if (masked_run && a.parents) s_parent[threadIdx.x] = static_cast<int16_t>(wrong ? -1 : up);
      if (threadIdx.x < 8) bad_rows[threadIdx.x] = 0;
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      tc_fence_before();  // (the run before: its O has been read)
      __syncwarp();
      const bool tree_ok = !named_bar_or(1, kSoft, wrong);
      if (threadIdx.x == 0) mbar_arrive(QFULL);
      // ---- tiles. Two row tiles: the groups' weights in turn, so that one group's products run
      // meanwhile
      if (kQ == 2 && g == 1) named_bar_arrive(2, kSoft);
      float m_ref = -INFINITY, l = 0.f;
      for (int t = kQ == 1 ? g : 0; t < r.n_tiles; t += 3 - kQ, ++n) {
        const int key0 = (r.tile0 + t) * kTile;
        const bool masked = new_rows(r, t);
        uint32_t see[kWords];
        if (masked) {
          const int c0 = key0 + copy * C::kCols;  // the lane's first key
#pragma unroll
          for (int w = 0; w < kWords; ++w) {
            // keys of the prefix; of a chain, up to the row itself
            const int cnt = min(max((a.parents ? prefix : prefix + node + 1) - c0 - 32 * w, 0), 32);
            see[w] = !live ? 0u : (cnt == 32 ? 0xffffffffu : (1u << cnt) - 1);
          }
          if (a.parents && live && tree_ok)
            for (int j = node; j >= 0; j = s_parent[j]) {
              const int c = prefix + j - c0;
#pragma unroll
              for (int w = 0; w < kWords; ++w)
                if ((c >> 5) == w) see[w] |= 1u << (c & 31);
            }
        }
        mbar_wait(SREADY(g), n & 1);
        __syncwarp();
        if (kQ == 2) named_bar_sync(2 + g, kSoft);  // the other group's weights are done
        tc_fence_after();
        // of 32 scores of the lane, hidden ones become -inf
        auto hide = [&](int c, uint32_t (&s)[32]) {
          if (masked) {
            uint32_t w = see[0];
#pragma unroll
            for (int x = 1; x < kWords; ++x)
              if (c == x) w = see[x];
#pragma unroll
            for (int j = 0; j < 32; ++j)
              if (!(w >> j & 1)) s[j] = 0xff800000u;
          }
        };
        // the row's reference moves to the tile's maximum where that is higher, and with it what
        // was summed
        auto move_reference = [&] {
          float mx = -INFINITY;
#pragma unroll 1
          for (int c = 0; c < kWords; ++c) {
            uint32_t s[32];
            tmem_load(ts + copy * C::kCols + 32 * c, s);
            hide(c, s);
#pragma unroll
            for (int j = 0; j < 32; j += 2) mx = max3(mx, __uint_as_float(s[j]), __uint_as_float(s[j + 1]));
          }
          const float now = fmaxf(m_ref, mx * sl), f = m_ref == -INFINITY ? 0.f : ex2(m_ref - now);
          m_ref = now;
          l *= f;
          if (t >= 3 - kQ) {  // the group's PV of the tile before is done: S came after it
#pragma unroll 1
            for (int c = 0; c < kDim; c += 32) {
              uint32_t o[32];
              tmem_load(to + kDim * g + c, o);
#pragma unroll
              for (int j = 0; j < 32; ++j) o[j] = __float_as_uint(__uint_as_float(o[j]) * f);
              tmem_store(to + kDim * g + c, o);
            }
          }
        };
        if (__any_sync(0xffffffffu, m_ref == -INFINITY)) move_reference();
        // weights relative to the reference; where their sum passes 2^16 (seldom), once more
        // relative to the tile's maximum
        uint32_t pw[C::kCols / 2];
        float sum[4];
#pragma unroll 1
        for (bool again = false;; again = true) {
          const float sub = m_ref == -INFINITY ? 0.f : -m_ref;
#pragma unroll
          for (int j = 0; j < 4; ++j) sum[j] = 0.f;
          // (32 scores at a time left gaps at their waits: a turn took 1430 cycles for 1203; 128: 1315)
          constexpr int kAtOnce = kWords < 2 ? 1 : 2;
#pragma unroll
          for (int c0 = 0; c0 < kWords; c0 += kAtOnce) {
            uint32_t s[kAtOnce][32];
#pragma unroll
            for (int c = 0; c < kAtOnce; ++c) tmem_load_begin(ts + copy * C::kCols + 32 * (c0 + c), s[c]);
#pragma unroll
            for (int c = 0; c < kAtOnce; ++c) {
              tmem_wait_load(s[c]);
              hide(c0 + c, s[c]);
            }
#pragma unroll
            for (int c = 0; c < kAtOnce; ++c)
#pragma unroll
              for (int j = 0; j < 32; j += 2) {
                const float2 y = fma2(make_float2(__uint_as_float(s[c][j]), __uint_as_float(s[c][j + 1])),
                                      make_float2(sl, sl), make_float2(sub, sub));
                const uint32_t w = cvt_bf16x2(ex2(y.x), ex2(y.y));
                pw[16 * (c0 + c) + j / 2] = w;
                add_pair(w, sum[j & 2], sum[(j & 2) + 1]);
              }
          }
          if (again || !__any_sync(0xffffffffu, (sum[0] + sum[1]) + (sum[2] + sum[3]) > 0x1p16f)) break;
          move_reference();
        }
        l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
        tmem_store(ts + copy * (C::kCols / 2), pw);
        if (kCopies > 1) {
          const uint32_t none[C::kCols / 2] = {};
#pragma unroll
          for (int c = 1; c < kCopies; ++c) tmem_store(ts + (copy ^ c) * (C::kCols / 2), none);
        }
        __syncwarp();
        tmem_wait_store();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(PFULL(g));
        if (kQ == 2 && (g == 0 || t + 1 < r.n_tiles)) named_bar_arrive(3 - g, kSoft);
      }
      // ---- the run's end: the groups and copies join
      const int own = kQ == 2 ? r.n_tiles : (r.n_tiles + 1 - g) / 2;
      if (own > 0) mbar_wait(PVDONE(g), (n - 1) & 1);
      s_ml[threadIdx.x] = make_float2(m_ref, l);
      tc_fence_before();
      __syncwarp();
      named_bar_sync(1, kSoft);
      tc_fence_after();
      const bool whole = r.n_tiles == r.tiles, both = kQ == 1 && r.n_tiles > 1;
      uint32_t any_bad = 0;
      if (masked_run)
        for (int w = 0; w < 8; ++w) any_bad |= bad_rows[w];
      const bool page_bad = *bad_page >> (run & 31) & 1;
      // a row's maximum over groups and copies, and its sum relative to that
      auto joined_ml = [&](int rr, float& mm, float& ll) {
        mm = -INFINITY, ll = 0.f;
#pragma unroll
        for (int c = 0; c < 2 * kCopies; ++c) mm = fmaxf(mm, s_ml[c * C::kRows + rr].x);
        const float sub = mm == -INFINITY ? 0.f : mm;
#pragma unroll
        for (int c = 0; c < 2 * kCopies; ++c) ll += s_ml[c * C::kRows + rr].y * ex2(s_ml[c * C::kRows + rr].x - sub);
        if (page_bad) ll = NAN;
        if (!tree_ok) mm = NAN;  // says so to the joining kernel
        return sub;
      };
      float top, total, ref = 0.f;
      if (kQ == 2) {
        top = tree_ok ? m_ref : NAN;
        total = page_bad ? NAN : l;
      } else {
        ref = joined_ml(rl % C::kRows, top, total);
      }
      const float f0 = kQ == 2 ? 1.f : ex2(s_ml[rl].x - ref), f1 = both ? ex2(s_ml[kTile + rl].x - ref) : 0.f;
      if (!tree_ok && threadIdx.x == 0) sd_set_error(SD_DEVERR_TREE);
      float* part = a.part + (2 * static_cast<size_t>(blockIdx.x) + (r.tile0 == 0 ? 1 : 0)) * part_floats(a.rows, kDim);
      // (in a cluster: rows in this CTA's K and V slots, whose products are done)
      auto put_o = [&](int rr, int c, const float4& v) {
        if (kCluster) *reinterpret_cast<float4*>(smem + cluster_o<kDim>(rr, c >> 2)) = v;
        else *(reinterpret_cast<float4*>(part) + static_cast<size_t>(c >> 2) * a.rows + rr) = v;
      };
      auto put_ml = [&](int rr, const float2& v) {
        if (kCluster) *reinterpret_cast<float2*>(smem + cluster_ml<kDim>(a.rows, rr)) = v;
        else *(reinterpret_cast<float2*>(part + static_cast<size_t>(a.rows) * kDim) + rr) = v;
      };
      auto out_of = [&](int pr) {  // packed row pr's output
        const int i = gdiv(pr);
        return a.out + ((static_cast<long long>(r.b) * a.R + i) * a.Hq + r.kvh * a.G + pr - i * a.G) * kDim;
      };
      // 32 columns of the lane's row, the groups' O joined
      auto joined = [&](int c, float (&x)[32]) {
        uint32_t o[32];
        __syncwarp();
        tmem_load(to + (kQ == 2 ? kDim * g : 0) + c, o);
#pragma unroll
        for (int j = 0; j < 32; ++j) x[j] = f0 * __uint_as_float(o[j]);
        if (both) {
          tmem_load(to + kDim + c, o);
#pragma unroll
          for (int j = 0; j < 32; ++j) x[j] = fmaf(f1, __uint_as_float(o[j]), x[j]);
        }
        if (any_bad && live && tree_ok && copy == 0)
#pragma unroll 1
          for (int j = 0; j < 32; ++j) {
            const float v = bad_values(a, s_parent, bad_rows, r.b, r.kvh, prefix, node, c + j, kDim);
#pragma unroll
            for (int k = 0; k < 32; ++k) x[k] += k == j ? v : 0.f;
          }
      };
      if (kCopies == 1) {
        // whole rows go out through the query tile (its products are done), a warp's own lanes
        const float inv = 1.f / total;
        const uint32_t stage = base + C::kOffQ + (kQ == 2 ? g * C::kTileBytes : 0);
        constexpr int kWide = kQ == 2 ? kDim : kDim / 2;  // columns a group
        const int c0 = kQ == 2 ? 0 : g * kWide;
#pragma unroll 1
        for (int c = c0; c < c0 + kWide; c += 32) {
          float x[32];
          joined(c, x);
          if (!whole) {
            if (live)
#pragma unroll
              for (int j = 0; j < 32; j += 4) put_o(row, c + j, make_float4(x[j], x[j + 1], x[j + 2], x[j + 3]));
          } else {
#pragma unroll
            for (int j = 0; j < 32; j += 8)
              st_shared_v4(stage + (c >> 6) * C::kHalf + rl * 128 + (((((c & 63) + j) >> 3) ^ (rl & 7)) << 4),
                           cvt_bf16x2(x[j] * inv, x[j + 1] * inv), cvt_bf16x2(x[j + 2] * inv, x[j + 3] * inv),
                           cvt_bf16x2(x[j + 4] * inv, x[j + 5] * inv), cvt_bf16x2(x[j + 6] * inv, x[j + 7] * inv));
          }
        }
        __syncwarp();
        if (!whole) {
          if (live && (kQ == 2 || g == 0)) put_ml(row, make_float2(top, total));
        } else if (tree_ok) {
          constexpr int kPer = kWide / 8;  // 16-byte chunks a row
#pragma unroll 4
          for (int x = lane; x < 32 * kPer; x += 32) {
            const int at = (warp & 3) * 32 + x / kPer, c = c0 / 8 + x % kPer, pr = r.mb * a.rows + (kQ == 2 ? g * kTile : 0) + at;
            if (pr >= M) continue;
            uint4 v;
            asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];"
                         : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
                         : "r"(stage + (c >> 3) * C::kHalf + at * 128 + (((c & 7) ^ (at & 7)) << 4))
                         : "memory");
            *reinterpret_cast<uint4*>(out_of(pr) + c * 8) = v;
          }
        }
      } else {
        // the copies' sums through shared memory: [128 lanes][columns of a round]; the query tile
        // (its products are done) holds half of them, a cluster's slots all, behind the part
        constexpr int kRounds = kCluster ? 1 : 2, kWide = kDim / kRounds;
        static_assert(!kCluster || C::kRows * (kDim + 2) * 4 + kTile * kDim * 4 <= C::kOffQ, "part and columns");
        float* stage = reinterpret_cast<float*>(smem + (kCluster ? (C::kRows * (kDim + 2) * 4 + 127) / 128 * 128 : C::kOffQ));
#pragma unroll 1
        for (int round = 0; round < kRounds; ++round) {
#pragma unroll 1
          for (int c = g * 32; c < kWide; c += 64) {  // 32 columns a group
            float x[32];
            joined(round * kWide + c, x);
            if (live)
#pragma unroll
            for (int j = 0; j < 8; ++j)
              *reinterpret_cast<float4*>(stage + rl * kWide + ((((c >> 2) + j) ^ (rl & 7)) << 2)) =
                  make_float4(x[4 * j], x[4 * j + 1], x[4 * j + 2], x[4 * j + 3]);
          }
          __syncwarp();
          named_bar_sync(1, kSoft);
          const bool wide = kCluster || whole;
          for (int x = threadIdx.x; x < (wide ? min(C::kRows, M - r.mb * a.rows) : C::kRows) * (kWide / 4); x += kSoft) {
            // (rows along the lanes for the workspace's parts, else columns)
            const int rr = wide ? x / (kWide / 4) : x % C::kRows, c4 = wide ? x % (kWide / 4) : x / C::kRows;
            const int pr = r.mb * a.rows + rr, d = round * kWide + c4 * 4;
            if (pr >= M) continue;
            float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int cp = 0; cp < kCopies; ++cp) {
              const int at = cp * C::kRows + rr;
              const float4 y = *reinterpret_cast<const float4*>(stage + at * kWide + ((c4 ^ (at & 7)) << 2));
              v.x += y.x, v.y += y.y, v.z += y.z, v.w += y.w;
            }
            if (!whole) {
              put_o(rr, d, v);
              if (d == 0) {
                float2 fin;
                joined_ml(rr, fin.x, fin.y);
                put_ml(rr, fin);
              }
            } else if (tree_ok) {
              float mm, ll;
              joined_ml(rr, mm, ll);
              const float inv = 1.f / ll;
              *reinterpret_cast<uint2*>(out_of(pr) + d) = make_uint2(cvt_bf16x2(v.x * inv, v.y * inv), cvt_bf16x2(v.z * inv, v.w * inv));
            }
          }
          __syncwarp();
          named_bar_sync(1, kSoft);
        }
      }
      tc_fence_before();
      __syncwarp();
      named_bar_sync(1, kSoft);
      if (threadIdx.x == 0 && page_bad) atomicAnd(const_cast<uint32_t*>(bad_page), ~(1u << (run & 31)));
      ++run;
    }
  }
  tc_fence_before();
  const int cs = gridDim.x, parts = kCluster ? min(cs, walk.s.tiles) : 1;  // CTAs that had tiles: the first ones
  __syncwarp();
  if (parts > 1) asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");  // (the same for the whole cluster)
  else __syncthreads();
  if (parts > 1) cluster_wait();
  if (warp == kProduct) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512) : "memory");
  }
  if (kCluster && parts > 1) {
    // ---- the cluster's parts: a CTA joins its share of the rows, a thread four columns of one
    const int n = parts;
    const int M = walk.s.m * a.G, mb = unit_block, rows = min(a.rows, M - mb * a.rows), each = (rows + cs - 1) / cs;
    const int row0 = blockIdx.x * each, mine = min(each, rows - row0);
    for (int x = threadIdx.x; x < mine * (kDim / 4); x += kThreads) {
      const int row = row0 + x / (kDim / 4), c4 = x % (kDim / 4);
      const uint32_t at = base + cluster_o<kDim>(row, c4), at_ml = base + cluster_ml<kDim>(a.rows, row);
      Joined j;
      constexpr int kBatch = 4;  // (in a loop: 16 at once, in line, took 13.8 for 13.6 us)
#pragma unroll 1
      for (int k0 = 0; k0 < n; k0 += kBatch) {
        float4 v[kBatch];
        float2 ml[kBatch];
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
          ml[u] = make_float2(-INFINITY, 0.f);
          v[u] = make_float4(0.f, 0.f, 0.f, 0.f);
          if (k0 + u < n) {
            asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(ml[u].x), "=f"(ml[u].y) : "r"(cluster_map(at_ml, k0 + u)));
            asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];"
                         : "=f"(v[u].x), "=f"(v[u].y), "=f"(v[u].z), "=f"(v[u].w)
                         : "r"(cluster_map(at, k0 + u)));
          }
        }
        j.add(ml, v);
      }
      const int pr = mb * a.rows + row, i = pr / a.G;
      j.store(a.out + ((static_cast<long long>(blockIdx.z) * a.R + i) * a.Hq + unit_head * a.G + pr - i * a.G) * kDim + c4 * 4);
    }
    __syncwarp();
    cluster_arrive_relaxed();  // (its reads are done; nobody's memory goes before)
    cluster_wait();
  }
}

// The units that a share's border cuts: border c lies between shares c - 1 and c, and the
// first one that cuts a unit joins its parts. A thread takes four columns of a row, rows along
// the lanes (as the parts lie), and eight parts, or four rows of two, at once: with 39 MB of parts
// of two (32 scenes, 61 rows) it waits for memory, 15 us cold, 22 with one row at a time.
template <int kDim>
__global__ void __launch_bounds__(kJoin) tree_join_kernel(const __grid_constant__ TreeArgs a, int ctas) {
  constexpr int kRowsJ = kJoin / (kDim / 4);
  sd_pdl_enter();
  const int lane = threadIdx.x & 31, c = blockIdx.x + 1;
  Walk walk;
  const Plan plan = walk.begin<true>(a, c, ctas, lane);
  Run r;
  if (!walk.next(a, r)) return;
  if (r.first == plan.begin(c) || plan.begin(c - 1) > r.first) return;
  const int share = c - 1, n = plan.cta_of(r.first + r.tiles - 1) - share + 1;  // its first share, its parts
  const int c4 = threadIdx.x / kRowsJ, rows = min(a.rows, r.m * a.G - r.mb * a.rows);
  const size_t pf = part_floats(a.rows, kDim);
  // (the unit begins in its first share's second part, and goes on in the others' first)
  const float* part0 = a.part + 2 * static_cast<size_t>(share) * pf;
  const int step = gridDim.y * kRowsJ;
  auto out_of = [&](int row) {
    const int p = r.mb * a.rows + row, i = p / a.G;
    return a.out + ((static_cast<long long>(r.b) * a.R + i) * a.Hq + r.kvh * a.G + p - i * a.G) * kDim + c4 * 4;
  };
  // kRows rows and kParts parts at once
  auto join = [&](auto rows_at, auto parts_at) {
    constexpr int kRows = decltype(rows_at)::value, kParts = decltype(parts_at)::value;
    for (int row0 = blockIdx.y * kRowsJ + threadIdx.x % kRowsJ; row0 < rows; row0 += kRows * step) {
      Joined j[kRows];
      for (int k0 = 0; k0 < n; k0 += kParts) {
        float4 v[kRows][kParts];
        float2 ml[kRows][kParts];
#pragma unroll
        for (int i = 0; i < kRows; ++i)
#pragma unroll
          for (int u = 0; u < kParts; ++u) {
            const int row = row0 + i * step, k = k0 + u;
            ml[i][u] = make_float2(-INFINITY, 0.f);
            v[i][u] = make_float4(0.f, 0.f, 0.f, 0.f);
            if (k < n && row < rows) {
              const float* part = part0 + (2 * static_cast<size_t>(k) + (k == 0 ? 1 : 0)) * pf;
              ml[i][u] = __ldcg(reinterpret_cast<const float2*>(part + static_cast<size_t>(a.rows) * kDim) + row);
              v[i][u] = __ldcg(reinterpret_cast<const float4*>(part) + static_cast<size_t>(c4) * a.rows + row);
            }
          }
#pragma unroll
        for (int i = 0; i < kRows; ++i) j[i].add(ml[i], v[i]);
      }
#pragma unroll
      for (int i = 0; i < kRows; ++i)
        if (row0 + i * step < rows) j[i].store(out_of(row0 + i * step));
    }
  };
  // (a unit cut once has two parts: then more rows instead)
  if (n == 2) join(std::integral_constant<int, 4>(), std::integral_constant<int, 2>());
  else join(std::integral_constant<int, 1>(), std::integral_constant<int, 8>());
}

// ------------------------------------------------------------------ host
constexpr int kSizes[] = {1, 2, 3, 4, 5, 6, 7, 8, 10, 12, 14, 16};  // CTAs a cluster
constexpr int kNumSizes = sizeof(kSizes) / sizeof(int);

cudaLaunchConfig_t config(dim3 grid, int smem, int cs, cudaStream_t st, cudaLaunchAttribute (&attr)[2]) {
  cudaLaunchConfig_t cfg = {};
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = cs;
  attr[1].val.clusterDim.y = 1;
  attr[1].val.clusterDim.z = 1;
  cfg.gridDim = grid;
  cfg.blockDim = dim3(kThreads, 1, 1);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cfg.attrs = attr;
  cfg.numAttrs = cs > 0 ? 2 : 1;
  return cfg;
}

// The kernel of a shape: even shares over `grid` CTAs (cs = 0) or clusters of cs.
template <int kDim, int kCopies, int kQ>
cudaError_t launch(const CUtensorMap& k, const CUtensorMap& v, const TreeArgs& a, dim3 grid, int cs, cudaStream_t st) {
  cudaLaunchAttribute attr[2];
  const cudaLaunchConfig_t cfg = config(grid, Cfg<kDim, kCopies, kQ>::kSmem, cs, st, attr);
  return cs > 0 ? cudaLaunchKernelEx(&cfg, tree_attention_kernel<kDim, kCopies, kQ, true>, k, v, a)
                : cudaLaunchKernelEx(&cfg, tree_attention_kernel<kDim, kCopies, kQ, false>, k, v, a);
}

template <int kDim, int kCopies, int kQ>
bool prepare(int* active) {
  const void* even = reinterpret_cast<const void*>(tree_attention_kernel<kDim, kCopies, kQ, false>);
  const void* cluster = reinterpret_cast<const void*>(tree_attention_kernel<kDim, kCopies, kQ, true>);
  constexpr int smem = Cfg<kDim, kCopies, kQ>::kSmem;
  if (cudaFuncSetAttribute(even, cudaFuncAttributeMaxDynamicSharedMemorySize, smem) != cudaSuccess ||
      cudaFuncSetAttribute(cluster, cudaFuncAttributeMaxDynamicSharedMemorySize, smem) != cudaSuccess ||
      cudaFuncSetAttribute(cluster, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) != cudaSuccess)
    return false;
  for (int i = 0; i < kNumSizes; ++i) {
    cudaLaunchAttribute attr[2];
    cudaLaunchConfig_t cfg = config(dim3(kSizes[i], 1, 1), smem, kSizes[i], nullptr, attr);
    attr[0] = attr[1];  // (the occupancy query takes the cluster alone)
    cfg.numAttrs = 1;
    if (cudaOccupancyMaxActiveClusters(&active[i], cluster, &cfg) != cudaSuccess) {
      (void)cudaGetLastError();
      active[i] = 0;
    }
  }
  return true;
}

// Per device, once: the kernels' shared memory, and the clusters of each size that fit at once.
struct DevState {
  std::once_flag once;
  bool ok = false;
  int active[2][4][kNumSizes] = {};  // [head dim 64, 128][copies 4, 2, 1, two row tiles]
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
    s.ok = prepare<64, 4, 1>(s.active[0][0]) && prepare<64, 2, 1>(s.active[0][1]) && prepare<64, 1, 1>(s.active[0][2]) &&
           prepare<64, 1, 2>(s.active[0][3]) && prepare<128, 4, 1>(s.active[1][0]) && prepare<128, 2, 1>(s.active[1][1]) &&
           prepare<128, 1, 1>(s.active[1][2]) && prepare<128, 1, 2>(s.active[1][3]);
    if (!s.ok) (void)cudaGetLastError();
  });
  return s.ok ? &s : nullptr;
}

struct HostPlan {
  int variant, rows, mblocks;  // copies 4, 2, 1, two row tiles; packed rows of an m-block
  int cs, ctas;                // CTAs a cluster; 0: even shares over ctas
  long long units, tiles;
  size_t ws_bytes;             // what even shares leave to the joining kernel
};

// What does not hang on the way that is chosen, for a device of `sms` SMs. ws_bytes grows with
// each of B, R and cap.
sd_status host_shape(int B, int R, int Hq, int Hkv, int D, int cap, int sms, HostPlan* p) {
  const long long M = static_cast<long long>(Hq / Hkv) * R;
  p->tiles = (static_cast<long long>(cap) + kTile - 1) / kTile;
  if (cap > 0x7fffff00) return SD_ERR_UNSUPPORTED;
  // copies where they fit (4096 keys, 4 packed rows: 10.8 -> 10.2 us; 131072 keys, 32: 98.6 ->
  // 93.7), two row tiles past one (32 scenes, 244 rows: 209 us, as two m-blocks 263; 205 now)
  p->variant = M <= 32 ? 0 : M <= 64 ? 1 : M <= 128 ? 2 : 3;
  p->rows = 32 << p->variant;
  const long long blocks = (M + p->rows - 1) / p->rows;
  p->units = blocks * B * Hkv;
  if (p->units > 0x7fffffffll / p->tiles) return SD_ERR_UNSUPPORTED;
  p->mblocks = static_cast<int>(blocks);
  p->ctas = static_cast<int>(std::min<long long>(std::min(sms, kMaxCtas), p->units * p->tiles));
  // (one tile a unit: no share's border cuts one)
  p->ws_bytes = p->tiles > 1 ? 2 * static_cast<size_t>(p->ctas) * part_floats(p->rows, D) * sizeof(float) : 0;
  return SD_OK;
}

sd_status host_plan(int B, int R, int Hq, int Hkv, int D, int cap, HostPlan* p) {
  const sd_status s = host_shape(B, R, Hq, Hkv, D, cap, sd_num_sms(), p);
  if (s != SD_OK) return s;
  const long long units = p->units, tiles = p->tiles, blocks = p->mblocks;
  DevState* dev = state();
  if (!dev) return SD_ERR_CUDA;
  // The way of least estimated time, in us, from what each took over 1 to 32 scenes of 512 to
  // 8192 keys: a CTA's tile, its first queries to its last output, the exchange in a cluster,
  // the joining kernel; and never less than all tiles' bytes take. (32 query / 8 KV heads x 128,
  // clusters / even shares: 26 rows and 4096 keys, 1 scene 16 / 37, 12 scenes 43 / 50, 20
  // scenes 81 / 71; 61 rows, 32 scenes of 512 keys 46 / 65, of 8192 232 / 205; 8 rows, 131072
  // keys 94 / 100, where clusters of 8 take 129, of 16 146.) The keys are not known here, so it
  // is the table's width that counts: measured for tables as wide as their longest scene. In one
  // 16 times as wide few scenes take even shares too: 1 row over 4096 keys 7.4 -> 12.1 us, 26
  // rows 11.9 -> 25.9, 32 scenes of 512 keys with 61 rows 33.7 -> 45.2.
  struct Cost {
    double tile, unit, exchange, join;
  };
  static constexpr Cost kCosts[2][4] = {{{0.7, 7.5, 1.0, 2.0}, {0.7, 7.5, 1.5, 3.0}, {0.72, 9.0, 1.5, 5.0}, {1.3, 12.0, 4.0, 10.0}},
                                        {{0.93, 7.5, 2.0, 2.0}, {0.95, 7.5, 3.0, 4.0}, {1.0, 8.0, 4.5, 7.0}, {1.64, 12.5, 6.0, 15.0}}};
  const Cost& c = kCosts[D == 128][p->variant];
  const int* active = dev->active[D == 128][p->variant];
  const double all = static_cast<double>(units) * tiles, stream = all * (4.0 * kTile * D / 6.7e6);
  const double runs = static_cast<double>((units + p->ctas - 1) / p->ctas);  // that a share begins beside its first
  double best = std::max(stream, all / p->ctas * c.tile + runs * c.unit) + c.unit + (tiles > 1 ? c.join : 0.0);
  p->cs = 0;
  if (blocks * Hkv <= 65535)
    for (int i = 0; i < kNumSizes; ++i) {
      const int cs = kSizes[i];
      if (active[i] <= 0 || cs > tiles) continue;
      const double waves = static_cast<double>((units + active[i] - 1) / active[i]);
      const double cost = std::max(stream + c.unit, waves * ((tiles + cs - 1) / cs * c.tile + c.unit + (cs > 1 ? c.exchange : 0.0)));
      if (cost < best) best = cost, p->cs = cs;
    }
  if (p->cs > 0) p->ws_bytes = 0;
  return SD_OK;
}

}  // namespace

extern "C" size_t sd_tree_attention_workspace(int B, int R, int Hq, int Hkv, int D, int capacity) {
  if (B <= 0 || R <= 0 || R > kMaxRows || Hkv <= 0 || Hq <= 0 || Hq % Hkv || Hq / Hkv > 4095 || (D != 64 && D != 128) || capacity <= 0)
    return 0;
  // enough for even shares, whatever the way: the estimate goes from one to the other and back as B
  // and R grow, and a workspace of the largest call has to serve the smaller ones
  HostPlan p = {};
  return host_shape(B, R, Hq, Hkv, D, capacity, state() ? sd_num_sms() : kMaxCtas, &p) == SD_OK ? p.ws_bytes : 0;
}

extern "C" sd_status sd_tree_attention(const void* q, long long q_stride, const sd_paged_cache* cache,
                                       const int32_t* parents, const int32_t* n_new, void* out, int R, int Hq,
                                       float scale, void* workspace, size_t ws_bytes, sd_stream_t stream) {
  const sd_status s = sd_internal_paged_check(cache);
  if (s != SD_OK) return s;
  const int B = cache->batch, Hkv = cache->n_kv_heads, D = cache->head_dim;
  if (R <= 0 || Hq <= 0 || Hq % Hkv) return SD_ERR_INVALID_ARG;
  if (!(scale >= 0.f) || !isfinite(scale)) return SD_ERR_INVALID_ARG;
  if (q_stride < static_cast<long long>(Hq) * D || q_stride % 8) return SD_ERR_INVALID_ARG;
  if (R > kMaxRows || Hq / Hkv > 4095) return SD_ERR_UNSUPPORTED;
  if (B == 0) return SD_OK;
  if (!q || !out || !sd_aligned16(q) || !sd_aligned16(out)) return SD_ERR_INVALID_ARG;
  if (workspace && !sd_aligned16(workspace)) return SD_ERR_INVALID_ARG;
  const double sc = scale > 0.f ? scale : 1.0 / sqrt(static_cast<double>(D));
  const float scale_log2 = static_cast<float>(sc * 1.4426950408889634);
  if (!isfinite(scale_log2)) return SD_ERR_INVALID_ARG;
  const int cap = cache->max_pages * cache->page;
  HostPlan p = {};
  const sd_status planned = host_plan(B, R, Hq, Hkv, D, cap, &p);
  if (planned != SD_OK) return planned;
  if (p.ws_bytes > 0 && (!workspace || ws_bytes < p.ws_bytes)) return SD_ERR_WORKSPACE;
  TreeArgs a = {};
  a.q = static_cast<const __nv_bfloat16*>(q);
  a.out = static_cast<__nv_bfloat16*>(out);
  a.v = static_cast<const __nv_bfloat16*>(cache->v);
  a.table = cache->table;
  a.len = cache->len;
  a.parents = parents;
  a.n_new = n_new;
  a.q_stride = q_stride;
  a.part = static_cast<float*>(workspace);
  a.B = B;
  a.R = R;
  a.Hq = Hq;
  a.Hkv = Hkv;
  a.G = Hq / Hkv;
  a.n_pages = cache->n_pages;
  a.shift = cache->page == 16 ? 4 : cache->page == 32 ? 5 : cache->page == 64 ? 6 : 7;
  a.max_pages = cache->max_pages;
  a.cap = cap;
  a.rows = p.rows;
  a.row_shift = 5 + p.variant;
  a.mblocks = p.mblocks;
  a.scale_log2 = scale_log2;
  a.inv_g = 1.0f / static_cast<float>(a.G);
  CUtensorMap k, v;
  if (!make_map(&k, cache->k, cache->page, cache->n_pages * Hkv, cache->page, D) ||
      !make_map(&v, cache->v, cache->page, cache->n_pages * Hkv, cache->page, D))
    return SD_ERR_CUDA;
  const cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  const auto run = D == 128 ? (p.variant == 0 ? launch<128, 4, 1> : p.variant == 1 ? launch<128, 2, 1>
                               : p.variant == 2 ? launch<128, 1, 1> : launch<128, 1, 2>)
                            : (p.variant == 0 ? launch<64, 4, 1> : p.variant == 1 ? launch<64, 2, 1>
                               : p.variant == 2 ? launch<64, 1, 1> : launch<64, 1, 2>);
  cudaError_t e = run(k, v, a, p.cs > 0 ? dim3(p.cs, Hkv * p.mblocks, B) : dim3(p.ctas), p.cs, st);
  if (e == cudaSuccess && p.ws_bytes > 0 && p.ctas > 1) {
    const long long rows = std::min<long long>(p.rows, static_cast<long long>(a.G) * R);
    e = sd_launch_pdl(D == 128 ? tree_join_kernel<128> : tree_join_kernel<64>,
                      dim3(p.ctas - 1, static_cast<unsigned>(std::min<long long>((rows * (D / 4) + kJoin - 1) / kJoin, 4))), dim3(kJoin), 0,
                      st, a, p.ctas);
  }
  if (e != cudaSuccess) {
    (void)cudaGetLastError();
    return SD_ERR_CUDA;
  }
  return SD_OK;
}
