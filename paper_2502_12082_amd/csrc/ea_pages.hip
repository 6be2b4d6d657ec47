// ea_pages.hip -- a cache of keys and values in pages and in 4 bits: rows go in
// and come back (append, read), and page tables go from step to step (update,
// compaction) with the pages that have to be copied.
//
// Blocks of 32 values share the scale 2^e, the smallest that leaves the largest
// magnitude at most 7: with a = max |x| = m 2^E, 1 <= m < 2, that is e = E - 2, or
// E - 1 where m > 1.75; x / 2^e is rounded to the nearest of 0, 0.5, 1, 1.5, 2, 3, 4
// and 6, ties to the even code (v_cvt_scalef32_pk_fp4, which takes the scale).  e is
// -125 at least and 125 at most, so that every number there is is a normal fp32 one.
#include "ea_common.h"
#include "ea_internal.h"

namespace ea {

namespace {

// ------------------------------------------------------------ rows in, rows out

// A thread takes 8 values of one token's key and value head: 16 (bf16) or 32
// bytes, 4 bytes of codes.  LPR lanes are a row; a wave's rows are tokens in order,
// whose rows of codes lie in one piece.  Bound by HBM where tokens are many.
constexpr int CR_NT = 256, CR_VALS = 8;
template <typename E>
struct Vals {
  float x[CR_VALS];
  __device__ __forceinline__ void load(const E* p) {
    if constexpr (sizeof(E) == 2) {
      const u32x4 w = *reinterpret_cast<const u32x4*>(p);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        x[2 * i] = __uint_as_float(w[i] << 16);
        x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
      }
    } else {
      const f32x4 a = reinterpret_cast<const f32x4*>(p)[0], b = reinterpret_cast<const f32x4*>(p)[1];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        x[i] = a[i];
        x[4 + i] = b[i];
      }
    }
  }
  // (a code's number times a power of two has two significant bits: no rounding in bf16.
  // Stores that pass the caches by: contexts of 8 requests of up to 8192 tokens, 8 heads, d
  // = 128, 29.6 us, 6.4 TB/s, against 40.2.)
  __device__ __forceinline__ void store(E* p) const {
    if constexpr (sizeof(E) == 2) {
      u32x4 w;
#pragma unroll
      for (int i = 0; i < 4; ++i)
        w[i] = __float_as_uint(x[2 * i]) >> 16 | (__float_as_uint(x[2 * i + 1]) & 0xFFFF0000u);
      __builtin_nontemporal_store(w, reinterpret_cast<u32x4*>(p));
    } else {
      f32x4 a, b;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        a[i] = x[i];
        b[i] = x[4 + i];
      }
      __builtin_nontemporal_store(a, reinterpret_cast<f32x4*>(p));
      __builtin_nontemporal_store(b, reinterpret_cast<f32x4*>(p) + 1);
    }
  }
};

// (control words: lanes of a quad exchange, 8 lanes mirrored, 16 rotated by 4 and by 8)
constexpr int QUAD_1032 = 0xB1, QUAD_2301 = 0x4E, HALF_MIRROR = 0x141, ROW_ROR_4 = 0x124, ROW_ROR_8 = 0x128;
template <int CTRL>
__device__ __forceinline__ uint32_t dpp_of(uint32_t v) {
#if defined(__HIP_DEVICE_COMPILE__)
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xf, 0xf, true);
#else
  return v;
#endif
}

// Scale byte of the block of 32 values whose four lanes call this, 255 where one
// of them is not finite.  (Magnitudes compare as the integers that their bits are.)
__device__ __forceinline__ uint32_t scale_of(const float (&x)[CR_VALS]) {
  uint32_t a = 0;
#pragma unroll
  for (int i = 0; i < CR_VALS; ++i) a = max(a, __float_as_uint(x[i]) & 0x7FFFFFFFu);
  a = max(a, dpp_of<QUAD_1032>(a));
  a = max(a, dpp_of<QUAD_2301>(a));
  const int e = (int)(a >> 23);
  return e == 255 ? 255u : (uint32_t)min(max(e - 2 + ((a & 0x7FFFFFu) > 0x600000u ? 1 : 0), 2), 252);
}

// The scale bytes of all blocks of a row, in all of its lanes.
template <int D>
__device__ __forceinline__ uint32_t row_scales(uint32_t scale, int sub) {
  uint32_t v = scale << (8 * (sub / 4));
  if constexpr (D == 64) return v | dpp_of<HALF_MIRROR>(v);
  v |= dpp_of<ROW_ROR_4>(v);
  return v | dpp_of<ROW_ROR_8>(v);
}

__device__ __forceinline__ uint32_t codes_of(const float (&x)[CR_VALS], uint32_t scale) {
  uint32_t w = 0;
#if defined(__HIP_DEVICE_COMPILE__)
  if (scale == 255) return 0;
  const float s = __uint_as_float(scale << 23);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[0], x[1], s, 0);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[2], x[3], s, 1);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[4], x[5], s, 2);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[6], x[7], s, 3);
#endif
  return w;
}
__device__ __forceinline__ void values_of(uint32_t w, uint32_t scale, float (&x)[CR_VALS]) {
#if defined(__HIP_DEVICE_COMPILE__)
  const float s = scale == 255 ? __builtin_nanf("") : __uint_as_float(scale << 23);
  auto pair = [&](int at, auto v) {
    x[at] = v[0] * s;
    x[at + 1] = v[1] * s;
  };
  pair(0, __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.f, 0));
  pair(2, __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.f, 1));
  pair(4, __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.f, 2));
  pair(6, __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.f, 3));
#endif
}

// Rows that a thread takes one after another, all loads first.
constexpr int CR_ROWS = 2;

template <typename E, int D, bool APPEND>
__global__ __launch_bounds__(CR_NT) void cache_rows_kernel(CacheRowsArgs a, int token_tiles) {
  constexpr int LPR = D / CR_VALS, STEP = CR_NT / LPR;
  const int sub = threadIdx.x % LPR, head = blockIdx.x / token_tiles;
  const int t0 = blockIdx.x % token_tiles * (STEP * CR_ROWS) + threadIdx.x / LPR;
  E* const K = static_cast<E*>(a.k) + head * a.k_head + sub * CR_VALS;
  E* const V = static_cast<E*>(a.v) + head * a.v_head + sub * CR_VALS;
  int32_t at[CR_ROWS], page[CR_ROWS];
#pragma unroll
  for (int u = 0; u < CR_ROWS; ++u) {
    const int t = t0 + u * STEP;
    at[u] = t < a.tokens ? a.positions[t] : -1;
    page[u] = t < a.tokens ? page_of(a.c, a.t, a.rows[t], at[u]) : -1;
  }
  if constexpr (APPEND) {
    Vals<E> k[CR_ROWS], v[CR_ROWS];
#pragma unroll
    for (int u = 0; u < CR_ROWS; ++u) {
      const int64_t t = min(t0 + u * STEP, a.tokens - 1);
      k[u].load(K + t * a.k_row);
      v[u].load(V + t * a.v_row);
    }
#pragma unroll
    for (int u = 0; u < CR_ROWS; ++u) {
      const uint32_t ks = scale_of(k[u].x), vs = scale_of(v[u].x);
      const uint32_t ks_row = row_scales<D>(ks, sub), vs_row = row_scales<D>(vs, sub);
      if (page[u] < 0) continue;
      const int r = at[u] & (PAGE_TILE - 1);
      uint8_t* const kt = a.cache + tile_at(a.c, page[u], head, false, at[u]);
      uint8_t* const vt = kt + part_bytes(a.c);
      const int to = r * (D / 2) + 4 * sub;
      *reinterpret_cast<uint32_t*>(kt + to) = codes_of(k[u].x, ks);
      *reinterpret_cast<uint32_t*>(vt + to) = codes_of(v[u].x, vs);
      if (sub < 2) {  // (the keys' scales by one lane, the values' by another)
        uint8_t* const st = (sub ? vt : kt) + PAGE_TILE * (D / 2) + r * (D / 32);
        const uint32_t scales = sub ? vs_row : ks_row;
        if constexpr (D == 64)
          *reinterpret_cast<uint16_t*>(st) = (uint16_t)scales;
        else
          *reinterpret_cast<uint32_t*>(st) = scales;
      }
    }
  } else {
    uint32_t k[CR_ROWS], v[CR_ROWS], ks[CR_ROWS], vs[CR_ROWS];
#pragma unroll
    for (int u = 0; u < CR_ROWS; ++u) {
      // (a row without a page reads the first one, and writes 0)
      const int r = at[u] & (PAGE_TILE - 1);
      const uint8_t* const kt = a.cache + tile_at(a.c, max(page[u], 0), head, false, at[u]);
      const uint8_t* const vt = kt + part_bytes(a.c);
      const int from = r * (D / 2) + 4 * sub, st = PAGE_TILE * (D / 2) + r * (D / 32) + sub / 4;
      k[u] = *reinterpret_cast<const uint32_t*>(kt + from);
      v[u] = *reinterpret_cast<const uint32_t*>(vt + from);
      ks[u] = kt[st];
      vs[u] = vt[st];
    }
#pragma unroll
    for (int u = 0; u < CR_ROWS; ++u) {
      const int64_t t = t0 + u * STEP;
      if (t >= a.tokens) continue;
      if (page[u] < 0) k[u] = v[u] = ks[u] = vs[u] = 0;
      Vals<E> x;
      values_of(k[u], ks[u], x.x);
      x.store(K + t * a.k_row);
      values_of(v[u], vs[u], x.x);
      x.store(V + t * a.v_row);
    }
  }
}

template <bool APPEND>
hipError_t launch_rows(const CacheRowsArgs& a, int dtype, hipStream_t s) {
  void (*kernel)(CacheRowsArgs, int) =
      a.c.head_dim == 64 ? (dtype == 0 ? cache_rows_kernel<__bf16, 64, APPEND> : cache_rows_kernel<float, 64, APPEND>)
                         : (dtype == 0 ? cache_rows_kernel<__bf16, 128, APPEND> : cache_rows_kernel<float, 128, APPEND>);
  const int step = CR_NT / (a.c.head_dim / CR_VALS) * CR_ROWS;
  int tiles = (a.tokens + step - 1) / step;
  CacheRowsArgs args = a;
  void* params[] = {&args, &tiles};
  return hipLaunchKernel(reinterpret_cast<const void*>(kernel), dim3((unsigned)(tiles * a.c.kv_heads)), dim3(CR_NT),
                         params, 0, s);
}

// ------------------------------------------------------------------ tables

constexpr int UP_NT = 1024, UP_WAVES = UP_NT / 64;

// Sums of `mine` over the threads before this one, from `base` on; base grows by
// all of them.  Counts stop at 2^30 (no pool has as many pages).
__device__ __forceinline__ int count_up(int a, int b) { return min(a + b, 1 << 30); }
__device__ __forceinline__ int place_of(int mine, int& base, int (&sums)[2][UP_WAVES], int& turn) {
  const int lane = lane_id(), w = wave_id();
  // (a wave's sum is small; the VALU alone: rows of 16 lanes, then from row to row)
  int incl = mine;
  incl += (int)dpp_of<0x111>(incl);  // row_shr 1, 2, 4, 8
  incl += (int)dpp_of<0x112>(incl);
  incl += (int)dpp_of<0x114>(incl);
  incl += (int)dpp_of<0x118>(incl);
#if defined(__HIP_DEVICE_COMPILE__)
  incl += __builtin_amdgcn_update_dpp(0, incl, 0x142, 0xa, 0xf, false);  // lane 15 to rows 1 and 3
  incl += __builtin_amdgcn_update_dpp(0, incl, 0x143, 0xc, 0xf, false);  // lane 31 to rows 2 and 3
#endif
  const int excl = incl - mine;
  auto& m = sums[turn];
  turn ^= 1;
  if (lane == 63) m[w] = incl;
  __syncthreads();
  int at = base;
#pragma unroll
  for (int x = 0; x < UP_WAVES; ++x) {
    if (x < w) at = count_up(at, m[x]);
    base = count_up(base, m[x]);
  }
  return count_up(at, excl);
}

__device__ __forceinline__ int row_length(const CacheUpdateArgs& a, int row) {
  return row < 0 || row >= a.t.rows ? 0 : a.lengths[row];
}
__device__ __forceinline__ RowPlan plan_of(const CacheUpdateArgs& a, int r) {
  return plan_row(row_length(a, a.parents[r]), a.counts[r], a.t.width, a.c.shift);
}
// The page that a row which `writes` has in part filled, or -1.
__device__ __forceinline__ int last_page(const CacheUpdateArgs& a, int r, const RowPlan& p) {
  return p.writes ? page_of(a.c, a.t, a.parents[r], p.old) : -1;
}
__device__ __forceinline__ RowPlan kept_of(const CacheUpdateArgs& a, int r) {
  return plan_row(row_length(a, r), 0, a.t.width, a.c.shift);
}

// Small tables (small_tables): one workgroup plans, with a bit in LDS for every page
// that is held, and the rows that are about to write to a page in a hash table.  (Counts of
// all holders there took a look for every entry: 64 rows of up to 256 pages 12.5 us against
// 9.1.)  It is bound by its chain of loads and barriers: a row's parent, its length, its
// entries.
constexpr int PL_ROWS = 256, PL_WORDS = 4096, PL_SLOTS = 2 * PL_ROWS, PL_FREE = 2048;

struct PageSet {
  uint32_t* word;  // a bit for each page
  int pages;
  __device__ __forceinline__ int words() const { return (pages + 31) / 32; }
  __device__ __forceinline__ void clear() const {
    for (int i = threadIdx.x; i < words(); i += UP_NT) word[i] = 0;
  }
  // pages [32 i, 32 i + 32) that are in the set
  __device__ __forceinline__ uint32_t held(int i) const { return i < words() ? word[i] : 0; }
  __device__ __forceinline__ uint32_t free(int i) const {
    return i >= words() ? 0 : ~word[i] & (32 * i + 32 > pages ? (1u << (pages & 31)) - 1 : ~0u);
  }
};

// Marks the pages that the entries [0, kept[r]) of the table's rows from[r] name: BATCH rows of a
// wave, and LOADS entries of a lane of each, are in flight.
template <int BATCH, int LOADS>
__device__ __forceinline__ void mark_rows(const CacheUpdateArgs& a, uint32_t* held, const int* from, const int* kept,
                                          int rows) {
  const int lane = lane_id();
  for (int r0 = wave_id(); r0 < rows; r0 += BATCH * UP_WAVES) {
    int n[BATCH], most = 0;
    const int32_t* in[BATCH];
#pragma unroll
    for (int j = 0; j < BATCH; ++j) {
      const int r = r0 + j * UP_WAVES;
      n[j] = r < rows ? kept[r] : 0;
      in[j] = a.t.ids + (n[j] ? from[r] : 0) * a.t.stride;
      most = max(most, n[j]);
    }
    for (int e0 = lane; e0 < most; e0 += 64 * LOADS) {
      int id[BATCH][LOADS];
#pragma unroll
      for (int j = 0; j < BATCH; ++j)
#pragma unroll
        for (int u = 0; u < LOADS; ++u) id[j][u] = e0 + 64 * u < n[j] ? in[j][e0 + 64 * u] : -1;
#pragma unroll
      for (int j = 0; j < BATCH; ++j)
#pragma unroll
        for (int u = 0; u < LOADS; ++u)
          if (id[j][u] >= 0 && id[j][u] < a.c.pages) atomicOr(&held[id[j][u] >> 5], 1u << (id[j][u] & 31));
    }
  }
}
// (64 rows of 128 pages 7.3 us with four rows and two entries, 9.1 with eight and one; 256 beams
// of 30 11.2 and 10.3.  Pieces of 64 entries, whichever rows they are of: 9.3 and 11.0.)
__device__ __forceinline__ void mark_held(const CacheUpdateArgs& a, uint32_t* held, const int* from, const int* kept,
                                          int rows) {
  if (rows <= 64)
    mark_rows<4, 2>(a, held, from, kept, rows);
  else
    mark_rows<8, 1>(a, held, from, kept, rows);
}

// Workgroup 0 plans; workgroup 1 + r writes those entries of row r that need no plan.
__global__ __launch_bounds__(UP_NT) void update_small_kernel(CacheUpdateArgs a) {
  __shared__ uint32_t held_words[PL_WORDS];
  __shared__ int key[PL_SLOTS], writers[PL_SLOTS], lowest[PL_SLOTS];
  __shared__ int from[PL_ROWS], kept[PL_ROWS], before[PL_ROWS + 1];
  __shared__ int sums[2][UP_WAVES], free_pages[PL_FREE];
  const int t = threadIdx.x;
  if (blockIdx.x) {
    const int r = blockIdx.x - 1;
    const RowPlan p = plan_of(a, r);
    int32_t* const out = a.table_out + r * a.out_stride;
    const int32_t* const in = a.t.ids + (p.old ? a.parents[r] : 0) * a.t.stride;
    const int open = p.writes ? p.old >> a.c.shift : -1;
    for (int i = t; i < a.t.width; i += UP_NT)
      if (i != open && (i < p.kept || i >= p.kept + p.grown)) out[i] = i < p.kept ? in[i] : -1;
    return;
  }
  const PageSet held{held_words, a.c.pages};
  held.clear();
  for (int i = t; i < PL_SLOTS; i += UP_NT) {
    key[i] = -1;
    writers[i] = 0;
    lowest[i] = INT32_MAX;
  }
  __syncthreads();
  RowPlan p{};
  int last = -1, slot = 0;
  if (t < a.rows_out) {
    p = plan_of(a, t);
    from[t] = a.parents[t];
    kept[t] = p.kept - (p.writes ? 1 : 0);  // (the page that it writes to is looked at below)
    last = last_page(a, t, p);
  }
  auto first = [](int page) { return (int)((uint32_t)page * 0x9E3779B1u >> 23); };
  static_assert(PL_SLOTS == 1 << 9, "a hash is 9 bits");
  if (last >= 0) {
    for (slot = first(last);; slot = (slot + 1) % PL_SLOTS) {  // (at most half of the slots are taken)
      const int was = atomicCAS(&key[slot], -1, last);
      if (was == -1 || was == last) break;
    }
    atomicAdd(&writers[slot], 1);
    atomicMin(&lowest[slot], t);
  }
  __syncthreads();
  mark_held(a, held_words, from, kept, a.rows_out);
  __syncthreads();
  // ---- pages needed before each row.  A page that rows are about to write to is held by
  // these, and by others if it is marked by now.
  int turn = 0, needed = 0;
  const int others = last >= 0 ? (int)(held_words[last >> 5] >> (last & 31) & 1) : 0;
  auto copy_with = [&](int keeper) {
    return last >= 0 && copies(writers[slot] + others, writers[slot], keeper, t) ? 1 : 0;
  };
  int copy = copy_with(lowest[slot]);
  int need = t < a.rows_out ? p.grown + copy : 0;
  int at = place_of(need, needed, sums, turn);
  if (last >= 0) atomicOr(&held_words[last >> 5], 1u << (last & 31));
  if (t < PL_ROWS) {
    before[t] = at;
    kept[t] = p.kept | copy << 30;
  }
  if (t == 0) before[PL_ROWS] = needed;
  __syncthreads();
  // ---- as many free pages, the lowest first
  int* const free_list = needed <= PL_FREE ? free_pages : a.free_list;
  int found = 0;
  for (int w0 = 0; w0 < held.words() && found < needed; w0 += UP_NT) {
    uint32_t bits = held.free(w0 + t);
    int to = place_of(__popc(bits), found, sums, turn);
    for (; bits && to < needed; bits &= bits - 1) free_list[to++] = 32 * (w0 + t) + __ffs(bits) - 1;
  }
  if (found < needed) {  // as many in all, of other rows
    int* const furthest = key;  // (which have served)
    for (int i = t; i < PL_SLOTS; i += UP_NT) furthest[i] = INT32_MAX;
    __syncthreads();
    if (last >= 0) atomicMin(&furthest[slot], keeper_key(p.old, a.c.shift, t));
    __syncthreads();
    copy = copy_with(keeper_row(furthest[slot]));
    need = t < a.rows_out ? p.grown + copy : 0;
    int again = 0;
    at = place_of(need, again, sums, turn);
    if (t < PL_ROWS) {
      before[t] = at;
      kept[t] = p.kept | copy << 30;
    }
  }
  __syncthreads();
  // ---- to the rows that can have all of theirs
  if (t < a.rows_out) {
    const bool done = need == 0 || at + need <= found;
    const int to = done && copy ? free_list[at] : -1;
    // (the entry that the row is about to write to; an entry that names no page stays)
    if (p.writes) {
      const int e = p.old >> a.c.shift;
      a.table_out[t * a.out_stride + e] = to >= 0 ? to : a.t.ids[from[t] * a.t.stride + e];
    }
    a.source[t] = last;
    a.target[t] = to;
    a.lengths_out[t] = done ? p.wanted : p.old;
    a.missing[t] = !p.fits ? -1 : done ? 0 : need;
  }
  for (int k = t; k < needed; k += UP_NT) {
    int lo = 0, hi = PL_ROWS;  // before[lo] <= k < before[hi]: the row that needs page k
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      (before[mid] <= k ? lo : hi) = mid;
    }
    const int i = k - before[lo] - (kept[lo] >> 30);
    if (i >= 0)
      a.table_out[lo * a.out_stride + (kept[lo] & 0x3FFFFFFF) + i] = before[lo + 1] <= found ? free_list[k] : -1;
  }
}

// Pages in use are marked; those behind the first `used` are paired with the free
// ones among these.
__device__ __forceinline__ void pair_pages(const CacheUpdateArgs& a, const PageSet& held, int (&sums)[2][UP_WAVES]) {
  const int t = threadIdx.x;
  int turn = 0, used = 0;
  for (int w0 = 0; w0 < held.words(); w0 += UP_NT) place_of(__popc(held.held(w0 + t)), used, sums, turn);
  // free pages below `used`, and pages in use from there on: as many
  int holes = 0, moves = 0;
  for (int w0 = 0; w0 < held.words(); w0 += UP_NT) {
    const int first = 32 * (w0 + t);
    const uint32_t below = used <= first ? 0u : used >= first + 32 ? ~0u : (1u << (used - first)) - 1;
    uint32_t hole = held.free(w0 + t) & below, move = held.held(w0 + t) & ~below;
    int h = place_of(__popc(hole), holes, sums, turn), m = place_of(__popc(move), moves, sums, turn);
    for (; hole; hole &= hole - 1) a.target[h++] = first + __ffs(hole) - 1;
    for (; move; move &= move - 1) a.source[m++] = first + __ffs(move) - 1;
  }
  __syncthreads();
  for (int m = t; m < moves; m += UP_NT) a.lowest[a.source[m]] = a.target[m];
  if (t == 0) {
    a.marks[0] = moves;
    a.missing[0] = used;
  }
}

__global__ __launch_bounds__(UP_NT) void compact_small_kernel(CacheUpdateArgs a) {
  __shared__ uint32_t held_words[PL_WORDS];
  __shared__ int from[PL_ROWS], kept[PL_ROWS];
  __shared__ int sums[2][UP_WAVES];
  const int t = threadIdx.x;
  const PageSet held{held_words, a.c.pages};
  held.clear();
  if (t < a.t.rows) {
    from[t] = t;
    kept[t] = kept_of(a, t).kept;
  }
  __syncthreads();
  mark_held(a, held_words, from, kept, a.t.rows);
  __syncthreads();
  pair_pages(a, held, sums);
}

// Any tables: counts of every page in memory, by a workgroup per row, and then one
// workgroup that plans.
__global__ __launch_bounds__(256) void clear_kernel(CacheUpdateArgs a) {
  const int i = blockIdx.x * 256 + threadIdx.x;
  if (i >= a.c.pages) return;
  a.holders[i] = 0;
  if (a.parents) {
    a.writers[i] = 0;
    a.lowest[i] = a.furthest[i] = INT32_MAX;
  }
}

__global__ __launch_bounds__(256) void update_rows_kernel(CacheUpdateArgs a) {
  const int t = threadIdx.x, r = blockIdx.x;
  const RowPlan p = plan_of(a, r);
  int32_t* const out = a.table_out + r * a.out_stride;
  const int32_t* const in = a.t.ids + (p.old ? a.parents[r] : 0) * a.t.stride;
  for (int i = t; i < a.t.width; i += 256) {
    int id = -1;
    if (i < p.kept) {
      id = in[i];
      if (id >= 0 && id < a.c.pages) atomicAdd(a.holders + id, 1);
    }
    out[i] = id;
  }
  if (t == 0) {
    const int last = last_page(a, r, p);
    if (last >= 0) {
      atomicAdd(a.writers + last, 1);
      atomicMin(a.lowest + last, r);
      atomicMin(a.furthest + last, keeper_key(p.old, a.c.shift, r));
    }
  }
}

__global__ __launch_bounds__(UP_NT) void update_plan_kernel(CacheUpdateArgs a) {
  __shared__ int sums[2][UP_WAVES];
  __shared__ int many, grown_row[UP_NT], grown_kept[UP_NT], grown_pages[UP_NT], grown_at[UP_NT];
  const int t = threadIdx.x, lane = lane_id(), w = wave_id();
  bool few = false;  // fewer pages are free than are needed
  auto row_copies = [&](int r, int last) {
    return last >= 0 && copies(a.holders[last], a.writers[last], few ? keeper_row(a.furthest[last]) : a.lowest[last], r);
  };
  int turn = 0, needed = 0;
  auto count_needs = [&]() {  // (of each row by the thread that gives it its pages below)
    needed = 0;
    for (int r0 = 0; r0 < a.rows_out; r0 += UP_NT) {
      const int r = r0 + t;
      int need = 0;
      if (r < a.rows_out) {
        const RowPlan p = plan_of(a, r);
        need = p.grown + (row_copies(r, last_page(a, r, p)) ? 1 : 0);
      }
      const int at = place_of(need, needed, sums, turn);
      if (r < a.rows_out) a.before[r] = at;
    }
  };
  count_needs();
  const int want = min(needed, a.c.pages);
  int found = 0;
  for (int p0 = 0; p0 < a.c.pages && found < want; p0 += 4 * UP_NT) {
    int32_t h[4];
    int mine = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int p = p0 + 4 * t + e;
      h[e] = p < a.c.pages ? a.holders[p] : 1;
      mine += h[e] == 0 ? 1 : 0;
    }
    int at = place_of(mine, found, sums, turn);
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (h[e] == 0) a.free_list[at++] = p0 + 4 * t + e;
  }
  if (found < needed) {  // as many in all, of other rows
    few = true;
    count_needs();
  }
  __syncthreads();
  // (a thread to a row; rows that grow by many pages have them from a wave each)
  for (int r0 = 0; r0 < a.rows_out; r0 += UP_NT) {
    const int r = r0 + t;
    if (t == 0) many = 0;
    __syncthreads();
    if (r < a.rows_out) {
      const RowPlan p = plan_of(a, r);
      const int last = last_page(a, r, p), copy = row_copies(r, last) ? 1 : 0;
      const int need = p.grown + copy, at = a.before[r];
      const bool done = need == 0 || count_up(at, need) <= found;
      int32_t* const out = a.table_out + r * a.out_stride;
      const int to = done && copy ? a.free_list[at] : -1;
      if (to >= 0) out[p.old >> a.c.shift] = to;
      a.source[r] = last;
      a.target[r] = to;
      a.lengths_out[r] = done ? p.wanted : p.old;
      a.missing[r] = !p.fits ? -1 : done ? 0 : need;
      if (done && p.grown <= 4) {
        for (int i = 0; i < p.grown; ++i) out[p.kept + i] = a.free_list[at + copy + i];
      } else if (done) {
        const int n = atomicAdd(&many, 1);
        grown_row[n] = r;
        grown_kept[n] = p.kept;
        grown_pages[n] = p.grown;
        grown_at[n] = at + copy;
      }
    }
    __syncthreads();
    for (int n = w; n < many; n += UP_WAVES) {
      int32_t* const out = a.table_out + grown_row[n] * a.out_stride + grown_kept[n];
      for (int i = lane; i < grown_pages[n]; i += 64) out[i] = a.free_list[grown_at[n] + i];
    }
    __syncthreads();
  }
}

__global__ __launch_bounds__(256) void compact_rows_kernel(CacheUpdateArgs a) {
  const int r = blockIdx.x, kept = kept_of(a, r).kept;
  const int32_t* const in = a.t.ids + r * a.t.stride;
  for (int i = threadIdx.x; i < kept; i += 256) {
    const int id = in[i];
    if (id >= 0 && id < a.c.pages) atomicOr(reinterpret_cast<uint32_t*>(a.holders) + (id >> 5), 1u << (id & 31));
  }
}
__global__ __launch_bounds__(UP_NT) void compact_plan_kernel(CacheUpdateArgs a) {
  __shared__ int sums[2][UP_WAVES];
  pair_pages(a, PageSet{reinterpret_cast<uint32_t*>(a.holders), a.c.pages}, sums);
}

constexpr int CP_NT = 256, CP_LOADS = 4, CP_CHUNK = CP_NT * CP_LOADS * 16;

// Stores pass the caches by, and the loads of a compaction (whose pages are read once; those
// that rows share are read again for each copy): 855 MB of pool, 204 MB moved, 80 us, 5.1
// TB/s, against 85 with neither; 256 beams' copies of 33 MB 12.5 us against 13.9, and 16.6
// with both.
// Copies page source[i] to page target[i] (none where that is negative) of every
// layer, i < `pairs` (COMPACT: as many as were found; then the tables too).
template <bool COMPACT>
__global__ __launch_bounds__(CP_NT) void copy_pages_kernel(CacheUpdateArgs a, int chunks) {
  const int t = threadIdx.x;
  const int64_t bytes = page_bytes(a.c), layer = bytes * a.c.pages;
  const int pairs = COMPACT ? a.marks[0] : a.rows_out;
  const int64_t items = (int64_t)pairs * a.layers * chunks;
  for (int64_t x = blockIdx.x; x < items; x += gridDim.x) {
    const int chunk = (int)(x % chunks), l = (int)(x / chunks % a.layers), i = (int)(x / chunks / a.layers);
    const int to = a.target[i];
    if (to < 0) continue;
    const uint8_t* const from = a.cache + l * layer + a.source[i] * bytes;
    uint8_t* const dst = a.cache + l * layer + to * bytes;
    const int64_t at = (int64_t)chunk * CP_CHUNK + 16 * t;
    u32x4 v[CP_LOADS];
#pragma unroll
    for (int u = 0; u < CP_LOADS; ++u)
      if (at + u * CP_NT * 16 < bytes) {
        const u32x4* const p = reinterpret_cast<const u32x4*>(from + at + u * CP_NT * 16);
        v[u] = COMPACT ? __builtin_nontemporal_load(p) : *p;
      }
#pragma unroll
    for (int u = 0; u < CP_LOADS; ++u)
      if (at + u * CP_NT * 16 < bytes)
        __builtin_nontemporal_store(v[u], reinterpret_cast<u32x4*>(dst + at + u * CP_NT * 16));
  }
  if constexpr (COMPACT) {
    for (int r = blockIdx.x; r < a.t.rows; r += gridDim.x) {
      const int kept = kept_of(a, r).kept, used = a.missing[0];
      for (int i = t; i < a.t.width; i += CP_NT) {
        int id = -1;
        if (i < kept) {
          id = a.t.ids[r * a.t.stride + i];
          if (id >= used && id < a.c.pages) id = a.lowest[id];
        }
        a.table_out[r * a.out_stride + i] = id;
      }
    }
  }
}

template <bool COMPACT>
hipError_t launch_copies(const CacheUpdateArgs& a, int64_t pairs, hipStream_t s) {
  int chunks = (int)((page_bytes(a.c) + CP_CHUNK - 1) / CP_CHUNK);
  int64_t wgs = pairs * a.layers * chunks;
  if (COMPACT && wgs < a.t.rows) wgs = a.t.rows;
  if (wgs > 4096) wgs = 4096;
  CacheUpdateArgs args = a;
  void* params[] = {&args, &chunks};
  return hipLaunchKernel(reinterpret_cast<const void*>(copy_pages_kernel<COMPACT>), dim3((unsigned)wgs), dim3(CP_NT),
                         params, 0, s);
}

hipError_t launch_clear(const CacheUpdateArgs& a, hipStream_t s) {
  return launch_kernel(clear_kernel, dim3((unsigned)((a.c.pages + 255) / 256)), dim3(256), s, a);
}

// Tables that one workgroup plans: it reads only what rows hold, and the form for any tables has
// two launches more and counts in memory.  Which is faster at the largest of them depends on
// what they hold, which the host does not know.  us in a graph, this against the other, pages of 16
// tokens, updates: 64 rows of 128 entries 9.0, 12.5; 32 x 4000 a tenth full 10.4, 13.7, half 16.7,
// 17.9, full 25.0, 23.4; 256 x 400 12.8, 13.8; 17.9, 15.3; 21.6, 17.1; but with few pages free,
// all behind those in use, 32 x 4000 full 28.6, 79.6, 256 x 400 25.2, 61.2.  Compactions: 64 x 128
// 7.4, 12.8; 32 x 4000 a tenth full 15.2, 20.6, half 22.1, 24.2, full 30.8, 27.8; 256 x 400
// 15.2, 19.5; 19.9, 21.9; 24.2, 23.0; 16 x 8192 18.4, 22.6; 32.5, 27.8; 50.1, 38.2.
bool small_tables(const CacheUpdateArgs& a, int rows) {
  return rows <= PL_ROWS && a.c.pages <= 32 * PL_WORDS && (int64_t)rows * a.t.width <= 1 << 17;
}

}  // namespace

hipError_t launch_cache_append(const CacheRowsArgs& a, int dtype, hipStream_t s) { return launch_rows<true>(a, dtype, s); }
hipError_t launch_cache_read(const CacheRowsArgs& a, int dtype, hipStream_t s) { return launch_rows<false>(a, dtype, s); }

hipError_t launch_cache_update(const CacheUpdateArgs& a, hipStream_t s) {
  hipError_t e;
  if (small_tables(a, a.rows_out)) {
    e = launch_kernel(update_small_kernel, dim3((unsigned)a.rows_out + 1), dim3(UP_NT), s, a);
  } else {
    e = launch_clear(a, s);
    if (e == hipSuccess) e = launch_kernel(update_rows_kernel, dim3((unsigned)a.rows_out), dim3(256), s, a);
    if (e == hipSuccess) e = launch_kernel(update_plan_kernel, dim3(1), dim3(UP_NT), s, a);
  }
  return e == hipSuccess ? launch_copies<false>(a, a.rows_out, s) : e;
}

hipError_t launch_cache_compact(const CacheUpdateArgs& a, hipStream_t s) {
  hipError_t e;
  if (small_tables(a, a.t.rows)) {
    e = launch_kernel(compact_small_kernel, dim3(1), dim3(UP_NT), s, a);
  } else {
    e = launch_clear(a, s);
    if (e == hipSuccess) e = launch_kernel(compact_rows_kernel, dim3((unsigned)a.t.rows), dim3(256), s, a);
    if (e == hipSuccess) e = launch_kernel(compact_plan_kernel, dim3(1), dim3(UP_NT), s, a);
  }
  return e == hipSuccess ? launch_copies<true>(a, a.c.pages / 2 + 1, s) : e;
}

}  // namespace ea
