// The paged KV cache: rows appended with the rotation on the way, and the rows that a
// tree's acceptance kept, moved together (sm_103a).
//
// A pool is [n_pages][Hkv][page][D]: row n of scene b and head g lies at
//     ((table[b][n / page] Hkv + g) page + n % page) D
// so that a page's rows of one head are contiguous (what the attention reads as one box).
//
// Append. Each 16-byte chunk of a new row is read once and written once; query and key
// chunks are rotated between (the angles as in the rotation kernel, bit for bit). A scene
// with a page out of range is left untouched, so every CTA looks at all the pages that the
// scene's new rows take before it writes. The scene's last CTA (a ticket) moves the length.
// Long calls are bound by the bytes: 8192 rows of 32 + 8 + 8 heads x 128, 201 MB, 36.2 us, 0.83 of
// a copy's rate. 8 rows take 4.4 us: length, pages, rows, ticket.
//
// Commit. Row first + path[i] moves to first + i. The path ascends, so path[i] >= i, and a
// thread that takes one 16-byte column of a head's rows in order, some at a time, never
// reads a row that it has written. 36 caches at once: one scene 7.8 us, 32 scenes of up to 61
// rows 13 us; round trips (length, path, pages, rows, ticket), not bytes (0.9 and 18 MB), and
// 1152 CTAs of 58 registers, four an SM, go through them in two waves.
#include "common.cuh"

#include <math.h>
#include <algorithm>

SD_DEFINE_ERROR_ACCESSOR(sd_take_error_paged)

namespace {

constexpr int kThreads = 128;  // of an append
constexpr int kCtas = 14;      // CTAs an SM of a long append

struct Paged {
  const int32_t* table;
  int Hkv, n_pages, shift, max_pages;  // page = 1 << shift
};
__device__ __forceinline__ long long paged_row(const Paged& p, int page_id, int g, int n) {
  return ((static_cast<long long>(page_id) * p.Hkv + g) << p.shift) + (n & ((1 << p.shift) - 1));
}

struct AppendArgs {
  Paged pg;
  uint4 *k, *v;            // pools
  const uint4 *k_new, *v_new;
  uint4 *q, *q_out;
  long long ks, vs, qs, qos;  // row strides in 16-byte chunks
  int32_t* len;
  uint32_t* ticket;
  const int32_t* n_new;
  const int32_t* pos;
  int R, Hq;
};

// Whether the pages of rows [first, first + n) of scene b are all valid, over the CTA.
__device__ __forceinline__ bool pages_ok(const Paged& p, int b, int first, int n) {
  bool ok = true;
  if (n > 0) {
    const int32_t* t = p.table + static_cast<long long>(b) * p.max_pages;
    for (int i = (first >> p.shift) + static_cast<int>(threadIdx.x); i <= ((first + n - 1) >> p.shift); i += kThreads) {
      const int id = __ldcg(t + i);
      ok &= id >= 0 && id < p.n_pages;
    }
  }
  return __syncthreads_and(ok) != 0;
}

// Grid (CTAs of a scene, scenes). A thread takes the same 16-byte chunk of kPer heads of one
// row, queries first, then keys, then values, and then of the row so many further on.
template <int D, int kPer>
__global__ void __launch_bounds__(kThreads) paged_append_kernel(const __grid_constant__ AppendArgs a,
                                                                const __grid_constant__ RopeTable tab) {
  constexpr int kVec = D / 8, kItems = kThreads / kVec;  // items (a row's kPer heads) of a CTA at once
  const int b = blockIdx.y, vec = threadIdx.x % kVec;
  const RopeChunk chunk = sd_rope_chunk(vec, tab);
  const int heads = a.Hq + 2 * a.pg.Hkv, rotated = a.pos ? a.Hq + a.pg.Hkv : 0, groups = (heads + kPer - 1) / kPer;
  sd_pdl_enter();
  const int l0 = __ldcg(a.len + b), n = a.n_new ? __ldcg(a.n_new + b) : a.R;
  const bool count_ok = n >= 0 && n <= a.R && l0 >= 0;
  const bool fits = count_ok && static_cast<long long>(l0) + n <= static_cast<long long>(a.pg.max_pages) << a.pg.shift;
  uint4 x[kPer];
  int page = 0, p[3] = {0, 0, 0};
  auto place = [&](long long item, int& r, int& h0) {
    r = static_cast<int>(item / groups);
    h0 = static_cast<int>(item - static_cast<long long>(r) * groups) * kPer;
  };
  auto load = [&](int r, int h0) {
    const long long row = static_cast<long long>(b) * a.R + r;
#pragma unroll
    for (int u = 0; u < kPer; ++u) {
      const int h = h0 + u;
      const uint4* src = h < a.Hq ? a.q + row * a.qs + h * kVec
                         : h < a.Hq + a.pg.Hkv ? a.k_new + row * a.ks + (h - a.Hq) * kVec
                                               : a.v_new + row * a.vs + (h - a.Hq - a.pg.Hkv) * kVec;
      if (h < heads) x[u] = __ldcg(src + vec);
    }
    page = __ldcg(a.pg.table + static_cast<long long>(b) * a.pg.max_pages + ((l0 + r) >> a.pg.shift));
    if (h0 < rotated)
#pragma unroll
      for (int j = 0; j < 3; ++j) p[j] = __ldcg(a.pos + row * 3 + j);
  };
  // the first row travels while the CTA looks at the pages
  const long long step = static_cast<long long>(gridDim.x) * kItems, items = fits ? static_cast<long long>(n) * groups : 0;
  long long item = blockIdx.x * static_cast<long long>(kItems) + threadIdx.x / kVec;
  int r = 0, h0 = 0;
  if (item < items) {
    place(item, r, h0);
    load(r, h0);
  }
  // (also the barrier between this CTA's reads of the length and its ticket)
  const bool paged = pages_ok(a.pg, b, l0, fits ? n : 0);
  if (threadIdx.x == 0) {
    __threadfence();
    if (atomicAdd(&a.ticket[b], 1u) == gridDim.x - 1) {
      a.ticket[b] = 0;
      if (fits && paged) a.len[b] = l0 + n;
      else sd_set_error(!count_ok ? SD_DEVERR_LENGTH : (fits ? SD_DEVERR_PAGE : SD_DEVERR_KV_OVERFLOW));
    }
  }
  if (!paged) return;
  while (item < items) {
    if (h0 < rotated) {
      float c[4], s[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float t = static_cast<float>(chunk.axis[j] == 0 ? p[0] : (chunk.axis[j] == 1 ? p[1] : p[2]));
        sincospif(2.0f * sd_frac_turns(t, chunk.hi[j], chunk.lo[j]), &s[j], &c[j]);
      }
#pragma unroll
      for (int u = 0; u < kPer; ++u)
        if (h0 + u < rotated)
          x[u] = make_uint4(sd_rope_pair(x[u].x, c[0], s[0]), sd_rope_pair(x[u].y, c[1], s[1]),
                            sd_rope_pair(x[u].z, c[2], s[2]), sd_rope_pair(x[u].w, c[3], s[3]));
    }
    const long long row = static_cast<long long>(b) * a.R + r;
#pragma unroll
    for (int u = 0; u < kPer; ++u) {
      const int h = h0 + u;
      if (h >= heads) break;
      if (h < a.Hq) {
        a.q_out[row * a.qos + h * kVec + vec] = x[u];
      } else {
        const bool key = h < a.Hq + a.pg.Hkv;
        const int g = h - a.Hq - (key ? 0 : a.pg.Hkv);
        (key ? a.k : a.v)[paged_row(a.pg, page, g, l0 + r) * kVec + vec] = x[u];
      }
    }
    item += step;
    if (item < items) {
      place(item, r, h0);
      load(r, h0);
    }
  }
}

// ------------------------------------------------------------------ commit
constexpr int kCaches = 48;  // caches a launch
constexpr int kRows = 256;   // threads, and rows of a path looked at together

struct CommitArgs {
  struct {
    uint4 *k, *v;
    const int32_t* table;
    int32_t* len;
    uint32_t* ticket;
    int n_pages, max_pages;
  } c[kCaches];
  const int32_t *path, *n_emit, *n_new;
  int R, Hkv, shift;
};

// Grid (columns of one cache's keys and values, scenes, caches). A CTA takes kRows rows of
// the path at a time: their places into shared memory, checked, then the rows.
template <int D>
__global__ void __launch_bounds__(kRows) paged_commit_kernel(const __grid_constant__ CommitArgs a) {
  constexpr int kVec = D / 8;
  constexpr int kBatch = 8;  // rows a thread has in flight
  __shared__ long long s_src[kRows], s_dst[kRows];  // rows of the pools; s_src -1: in its place
  const int b = blockIdx.y;
  const auto& c = a.c[blockIdx.z];
  const Paged pg = {c.table, a.Hkv, c.n_pages, a.shift, c.max_pages};
  sd_pdl_enter();
  const int32_t* path = a.path + static_cast<long long>(b) * a.R;
  const int32_t* table = c.table + static_cast<long long>(b) * c.max_pages;
  const int l = __ldcg(c.len + b), n = a.n_new ? __ldcg(a.n_new + b) : a.R, m = __ldcg(a.n_emit + b);
  // (the first rows of the path travel with the lengths)
  int from = static_cast<int>(threadIdx.x) < a.R ? __ldcg(path + threadIdx.x) : 0;
  int before = threadIdx.x > 0 && static_cast<int>(threadIdx.x) < a.R ? __ldcg(path + threadIdx.x - 1) : -1;
  const bool len_ok = n >= 0 && n <= a.R && l >= n && l <= static_cast<long long>(c.max_pages) << a.shift;
  const bool m_ok = m >= 0 && m <= n;
  const int first = l - n, rows = len_ok && m_ok ? m : 0;
  bool path_ok = true, page_ok = true;
  // where row i of the path comes from and goes to
  auto place = [&](int i) {
    const bool ok = from > before && from < n;
    path_ok &= ok;
    const int src = __ldcg(table + ((first + (ok ? from : 0)) >> a.shift)), dst = __ldcg(table + ((first + i) >> a.shift));
    page_ok &= src >= 0 && src < c.n_pages && dst >= 0 && dst < c.n_pages;
    s_src[threadIdx.x] = from == i ? -1 : paged_row(pg, src, 0, first + from);
    s_dst[threadIdx.x] = paged_row(pg, dst, 0, first + i);
  };
  auto load = [&](int i) {
    from = __ldcg(path + i);
    before = i > 0 ? __ldcg(path + i - 1) : -1;
  };
  for (int i = static_cast<int>(threadIdx.x) + kRows; i < rows; i += kRows) {  // (long paths: checked first)
    load(i);
    place(i);
  }
  if (static_cast<int>(threadIdx.x) < rows) {
    if (rows > kRows) load(threadIdx.x);
    place(threadIdx.x);
  }
  path_ok = __syncthreads_and(path_ok) != 0;
  page_ok = __syncthreads_and(page_ok) != 0;
  const bool ok = len_ok && m_ok && path_ok && page_ok;
  if (threadIdx.x == 0) {
    __threadfence();
    if (atomicAdd(&c.ticket[b], 1u) == gridDim.x - 1) {
      c.ticket[b] = 0;
      if (ok) c.len[b] = first + m;
      else sd_set_error(!len_ok ? SD_DEVERR_LENGTH : (m_ok && path_ok ? SD_DEVERR_PAGE : SD_DEVERR_ROLLBACK));
    }
  }
  if (!ok) return;
  const int col = blockIdx.x * kRows + threadIdx.x;  // [k, v][head][chunk]
  const int vec = col % kVec, h = col / kVec, g = h % a.Hkv;
  uint4* pool = (h < a.Hkv ? c.k : c.v) + ((static_cast<long long>(g) << a.shift) * kVec + vec);
  for (int i0 = 0; i0 < m; i0 += kRows) {
    if (i0 > 0) {
      __syncthreads();
      if (i0 + static_cast<int>(threadIdx.x) < m) {
        load(i0 + threadIdx.x);
        place(i0 + threadIdx.x);
      }
      __syncthreads();
    }
    const int here = min(m - i0, kRows);
    if (h >= 2 * a.Hkv) continue;
    for (int i = 0; i < here; i += kBatch) {
      uint4 x[kBatch];
#pragma unroll
      for (int u = 0; u < kBatch; ++u)
        if (i + u < here && s_src[i + u] >= 0) x[u] = __ldcg(pool + s_src[i + u] * kVec);
#pragma unroll
      for (int u = 0; u < kBatch; ++u)
        if (i + u < here && s_src[i + u] >= 0) pool[s_dst[i + u] * kVec] = x[u];
    }
  }
}

// The rotation's table, kept from call to call of a thread with the same numbers (64 powers take
// 3 us).
const RopeTable* table_of(int D, const int32_t* sections, int interleaved, float base) {
  struct Kept {
    bool valid = false;
    int D, sections[3], interleaved;
    float base;
    RopeTable tab;
  };
  static thread_local Kept k;
  if (!k.valid || k.D != D || k.sections[0] != sections[0] || k.sections[1] != sections[1] || k.sections[2] != sections[2] ||
      k.interleaved != interleaved || k.base != base) {
    k.valid = sd_internal_rope_table(D, sections, interleaved, base, &k.tab);
    k.D = D, k.interleaved = interleaved, k.base = base;
    for (int i = 0; i < 3; ++i) k.sections[i] = sections[i];
  }
  return k.valid ? &k.tab : nullptr;
}

int log2_of(int page) { return page == 16 ? 4 : page == 32 ? 5 : page == 64 ? 6 : 7; }

}  // namespace

sd_status sd_internal_paged_check(const sd_paged_cache* c) {
  if (!c || c->batch < 0 || c->n_kv_heads <= 0 || c->n_pages <= 0 || c->max_pages <= 0) return SD_ERR_INVALID_ARG;
  if (c->head_dim != 64 && c->head_dim != 128) return SD_ERR_UNSUPPORTED;
  if (c->page != 16 && c->page != 32 && c->page != 64 && c->page != 128) return SD_ERR_UNSUPPORTED;
  if (c->batch > 65535 || c->n_kv_heads > 32767) return SD_ERR_UNSUPPORTED;
  if (static_cast<long long>(c->max_pages) * c->page > 0x7fffffffll) return SD_ERR_UNSUPPORTED;
  if (static_cast<long long>(c->n_pages) * c->n_kv_heads > 0x7fffffffll) return SD_ERR_UNSUPPORTED;
  if (c->batch == 0) return SD_OK;
  if (!c->k || !c->v || !c->table || !c->len || !c->ticket) return SD_ERR_INVALID_ARG;
  if (!sd_aligned16(c->k) || !sd_aligned16(c->v)) return SD_ERR_INVALID_ARG;
  return SD_OK;
}

extern "C" sd_status sd_paged_append(const sd_paged_cache* cache, const void* k_new, long long k_stride,
                                     const void* v_new, long long v_stride, void* q, long long q_stride, void* q_out,
                                     int R, int Hq, const int32_t* pos, const int32_t sections[3], int interleaved,
                                     float base, const int32_t* n_new, sd_stream_t stream) {
  const sd_status s = sd_internal_paged_check(cache);
  if (s != SD_OK) return s;
  const int B = cache->batch, Hkv = cache->n_kv_heads, D = cache->head_dim;
  if (R < 0 || Hq < 0) return SD_ERR_INVALID_ARG;
  if (interleaved != 0 && interleaved != 1) return SD_ERR_INVALID_ARG;
  static const RopeTable kNone = {};
  const RopeTable* tab = &kNone;
  if (pos) {
    if (!sections || !(base > 1.0f) || !isfinite(base)) return SD_ERR_INVALID_ARG;
    tab = table_of(D, sections, interleaved, base);
    if (!tab) return SD_ERR_INVALID_ARG;
  }
  if (k_stride < static_cast<long long>(Hkv) * D || v_stride < static_cast<long long>(Hkv) * D || k_stride % 8 || v_stride % 8 ||
      (q && (q_stride < static_cast<long long>(Hq) * D || q_stride % 8)))
    return SD_ERR_INVALID_ARG;
  if (B == 0 || R == 0) return SD_OK;  // (the addresses of nothing may be NULL)
  if ((Hq > 0) != (q != nullptr) || (q_out && !q) || (q && !pos)) return SD_ERR_INVALID_ARG;
  if (!k_new || !v_new || !sd_aligned16(k_new) || !sd_aligned16(v_new) || !sd_aligned16(q) || !sd_aligned16(q_out))
    return SD_ERR_INVALID_ARG;
  AppendArgs a = {};
  a.pg = {cache->table, Hkv, cache->n_pages, log2_of(cache->page), cache->max_pages};
  a.k = static_cast<uint4*>(cache->k);
  a.v = static_cast<uint4*>(cache->v);
  a.k_new = static_cast<const uint4*>(k_new);
  a.v_new = static_cast<const uint4*>(v_new);
  a.q = static_cast<uint4*>(q);
  a.q_out = static_cast<uint4*>(q_out ? q_out : q);
  a.ks = k_stride / 8;
  a.vs = v_stride / 8;
  a.qs = q_stride / 8;
  a.qos = q_out ? static_cast<long long>(Hq) * D / 8 : a.qs;
  a.len = cache->len;
  a.ticket = cache->ticket;
  a.n_new = n_new;
  a.pos = pos;
  a.R = R;
  a.Hq = Hq;
  // heads a thread: one where the call is short, so that many threads share its latency; four
  // or eight where it is long: the angles of a row are taken once for them (1, 4, 8 heads: 8 rows
  // of 48 heads 4.4, 5.1, 5.6 us; 32 ragged trees of 36 heads x 64 10.0, 7.4, 7.8; 8192 rows of 48 92, 38.2, 36.2)
  const long long heads = Hq + 2ll * Hkv, per_cta = kThreads / (D / 8), sms = sd_num_sms();
  const long long ctas = static_cast<long long>(B) * R * heads / per_cta;
  const int per = ctas >= 16 * sms ? 8 : ctas >= 4 * sms ? 4 : 1;
  // as many CTAs as are resident (seven an SM, at 72 registers), twice, and each goes on from
  // there. 201 MB: 36.2 us; one CTA for each 128 items 43.9, CTAs of 256 threads, three an SM, 38.4
  const long long blocks = std::min((R * ((heads + per - 1) / per) + per_cta - 1) / per_cta, std::max<long long>((kCtas * sms + B - 1) / B, 1));
  const auto kernel = D == 64 ? (per == 8 ? paged_append_kernel<64, 8> : per == 4 ? paged_append_kernel<64, 4> : paged_append_kernel<64, 1>)
                              : (per == 8 ? paged_append_kernel<128, 8> : per == 4 ? paged_append_kernel<128, 4> : paged_append_kernel<128, 1>);
  if (sd_launch_pdl(kernel,
                    dim3(static_cast<unsigned>(blocks), B), dim3(kThreads), 0, reinterpret_cast<cudaStream_t>(stream), a,
                    *tab) != cudaSuccess) {
    (void)cudaGetLastError();
    return SD_ERR_CUDA;
  }
  return SD_OK;
}

extern "C" sd_status sd_paged_commit(const sd_paged_cache* caches, int count, const int32_t* path, const int32_t* n_emit,
                                     const int32_t* n_new, int R, sd_stream_t stream) {
  if (!caches || count <= 0 || R <= 0) return SD_ERR_INVALID_ARG;
  if (R > 65535) return SD_ERR_UNSUPPORTED;
  for (int i = 0; i < count; ++i) {
    const sd_status s = sd_internal_paged_check(&caches[i]);
    if (s != SD_OK) return s;
    if (caches[i].batch != caches[0].batch || caches[i].n_kv_heads != caches[0].n_kv_heads ||
        caches[i].page != caches[0].page || caches[i].head_dim != caches[0].head_dim)
      return SD_ERR_INVALID_ARG;
    for (int j = 0; j < i; ++j)  // the same cache twice would move its rows twice
      if (caches[0].batch > 0 && (caches[i].k == caches[j].k || caches[i].v == caches[j].v || caches[i].len == caches[j].len ||
                                  caches[i].ticket == caches[j].ticket))
        return SD_ERR_INVALID_ARG;
  }
  if (caches[0].batch == 0) return SD_OK;
  if (!path || !n_emit) return SD_ERR_INVALID_ARG;
  const int D = caches[0].head_dim;
  CommitArgs a = {};
  a.path = path;
  a.n_emit = n_emit;
  a.n_new = n_new;
  a.R = R;
  a.Hkv = caches[0].n_kv_heads;
  a.shift = log2_of(caches[0].page);
  const int blocks = (2 * a.Hkv * (D / 8) + kRows - 1) / kRows;
  for (int i0 = 0; i0 < count; i0 += kCaches) {
    const int n = count - i0 < kCaches ? count - i0 : kCaches;
    for (int i = 0; i < n; ++i) {
      const sd_paged_cache& c = caches[i0 + i];
      a.c[i] = {static_cast<uint4*>(c.k), static_cast<uint4*>(c.v), c.table, c.len, c.ticket, c.n_pages, c.max_pages};
    }
    if (sd_launch_pdl(D == 64 ? paged_commit_kernel<64> : paged_commit_kernel<128>, dim3(blocks, caches[0].batch, n),
                      dim3(kRows), 0, reinterpret_cast<cudaStream_t>(stream), a) != cudaSuccess) {
      (void)cudaGetLastError();
      return SD_ERR_CUDA;
    }
  }
  return SD_OK;
}
