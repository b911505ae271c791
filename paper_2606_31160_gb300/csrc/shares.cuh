// Even shares of a batch's key tiles (sm_103a): the tiles of all units (a scene's KV heads,
// or their m-blocks), one unit after the other, cut into one contiguous share a CTA. Fewer
// than 2^31 tiles; a scene that is not valid has none.
#pragma once
#include "common.cuh"

namespace {

constexpr int kShareTile = 128;  // keys a tile

struct Scenes {
  const int32_t* len;
  const int32_t* committed;  // or nullptr
  int B, R, cap, units;      // units a scene
};
// The keys of scene b, 0 where its length, or its committed rows, are not valid.
__device__ __forceinline__ int keys_of(const Scenes& s, int b) {
  const int n = __ldcg(s.len + b), c = s.committed ? __ldcg(s.committed + b) : 0;
  return n >= s.R && n <= s.cap && c >= 0 && c <= s.R ? n : 0;
}
__device__ __forceinline__ int tiles_of(int n_keys) { return (n_keys + kShareTile - 1) / kShareTile; }

struct Shares {
  int total, each, rest;  // all tiles, tiles a share, shares with one more
  int n_keys;             // of scene `lane`
  __device__ __forceinline__ int begin(int cta) const { return cta * each + min(cta, rest); }
  // the CTA with tile `pos` in its share
  __device__ __forceinline__ int cta_of(int pos) const {
    const int more = rest * (each + 1);  // tiles of the shares with one more
    return pos < more ? pos / (each + 1) : rest + (pos - more) / each;
  }
};

__device__ __forceinline__ Shares shares_of(const Scenes& sc, int lane, int ctas) {
  Shares s;
  s.n_keys = lane < sc.B ? keys_of(sc, lane) : 0;
  int n = tiles_of(s.n_keys);
  for (int b = lane + 32; b < sc.B; b += 32) n += tiles_of(keys_of(sc, b));
  s.total = static_cast<int>(__reduce_add_sync(0xffffffffu, static_cast<uint32_t>(n))) * sc.units;
  s.each = s.total / ctas;
  s.rest = s.total - s.each * ctas;
  return s;
}

// Tile `tile` of unit `unit` of scene b, which has so many keys, and tiles a unit; the unit's
// first tile is `first` of all.
struct Place {
  int b, unit, tile, n_keys, tiles, first;
};
__device__ __forceinline__ Place locate(const Scenes& sc, const Shares& s, int pos, int lane) {  // pos < total
  Place p = {};
  int n_keys = s.n_keys, before = 0;
  for (int b0 = 0; b0 < sc.B; b0 += 32) {
    if (b0 > 0) n_keys = b0 + lane < sc.B ? keys_of(sc, b0 + lane) : 0;
    const int mine = tiles_of(n_keys) * sc.units;
    int upto = mine;
#pragma unroll
    for (int x = 1; x < 32; x <<= 1) {
      const int y = __shfl_up_sync(0xffffffffu, upto, x);
      if (lane >= x) upto += y;
    }
    const uint32_t past = __ballot_sync(0xffffffffu, before + upto > pos);
    if (past) {
      const int at = __ffs(past) - 1;
      p.b = b0 + at;
      p.n_keys = __shfl_sync(0xffffffffu, n_keys, at);
      p.tiles = tiles_of(p.n_keys);
      const int in = pos - before - __shfl_sync(0xffffffffu, upto - mine, at);
      p.unit = in / p.tiles;
      p.tile = in - p.unit * p.tiles;
      p.first = pos - p.tile;
      break;
    }
    before += __shfl_sync(0xffffffffu, upto, 31);
  }
  return p;
}

// A run of one unit's tiles in a CTA's share.
struct Span {
  int b, unit, first, n_keys, key_begin, key_end, n_tiles;
  bool whole;  // all the unit's tiles
};
// The runs of this CTA's share (of a grid of one dimension), from the first on, or from the last.
template <bool kBack>
struct Walk {
  Place at;
  int left;  // tiles
  __device__ __forceinline__ void begin(const Scenes& sc, const Shares& s, int lane) {
    const int first = s.begin(blockIdx.x);
    left = s.begin(blockIdx.x + 1) - first;
    at = Place{};
    if (left > 0) at = locate(sc, s, kBack ? first + left - 1 : first, lane);
  }
  __device__ __forceinline__ Span next(const Scenes& sc) {
    Span r;
    r.b = at.b;
    r.unit = at.unit;
    r.first = at.first;
    r.n_keys = at.n_keys;
    r.n_tiles = min(kBack ? at.tile + 1 : at.tiles - at.tile, left);
    r.whole = r.n_tiles == at.tiles;
    const int from = kBack ? at.tile + 1 - r.n_tiles : at.tile;
    r.key_begin = from * kShareTile;
    r.key_end = from + r.n_tiles == at.tiles ? at.n_keys : r.key_begin + r.n_tiles * kShareTile;
    left -= r.n_tiles;
    if (left > 0) {
      at.unit += kBack ? -1 : 1;
      if (!kBack) at.first += at.tiles;
      if (at.unit == (kBack ? -1 : sc.units)) {
        at.unit = kBack ? sc.units - 1 : 0;
        at.tiles = 0;
        at.b += kBack ? -1 : 1;
        for (; at.tiles == 0 && (kBack ? at.b >= 0 : at.b < sc.B); at.b += kBack ? -1 : 1) {
          at.n_keys = keys_of(sc, at.b);
          at.tiles = tiles_of(at.n_keys);
          if (at.tiles > 0) break;
        }
        if (at.tiles == 0) left = 0;  // (only if a length changed under the kernel)
      }
      if (kBack) at.first -= at.tiles;
      at.tile = kBack ? at.tiles - 1 : 0;
    }
    return r;
  }
};

}  // namespace
