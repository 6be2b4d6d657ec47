// ea_paged.hip -- alpha-entmax attention of single tokens over a cache in pages
// and in 4 bits (ea_pages.h), 1 < alpha <= 2.
//
// For head h of query i, with keys k_j of its row of the table:
//   x_j = (alpha - 1) scale <q, k_j>,  tau: sum_j [x_j - tau]_+^gamma = 1,
//   o = sum_j [x_j - tau]_+^gamma v_j.
// Two kernels, or for short rows one that does both:
//
// Scores.  <q, k> comes from the matrix cores' product of 8-bit and 4-bit
// operands with a scale for every 32 values: K's codes and scales are its operands
// as they lie in the cache.  Its 8-bit operand has four significant bits, and it
// keeps products of 8 values 13 bits below the largest of them (measured; 23 bits
// between such groups), so q is taken apart into digits: of a block of 32 values with
// the largest magnitude in [8, 16) units, digit 0 is the nearest whole number
// of units, digit 1 that of 32nds of what is left, and so on, each a whole number of at
// most 16.  A product of a digit and a code has 8 bits, and the sums of a
// block are exact.  Four digits are within 2^-19 of the largest magnitude (bf16),
// six within 2^-29 (fp32).  Only scores that can matter are written: the largest scores of
// a region's lanes are scores of distinct keys, so f restricted to them lies below f,
// and its root is a lower bound of tau.  (Those within 1 of the largest, as
// tau is at least max x - 1, were ten times as many: 64 requests of up to 9216 keys,
// 32/8 heads, d = 128, this step 42.2 us against 38.0, the next 21.5 against 12.5.)
//
// Solve.  One workgroup per query row.  The regions' bounds, and in the same way the
// largest scores of its regions, bound tau from below; the listed scores above that go to LDS, tau is solved on them
// (Algorithm 1's iteration), and the rows of V with a probability are gathered.  From
// the bound on, x and tau are taken against the row's largest x, as c (s - max s): the 24
// bits of a tau by itself are too few where scores are far from 0 (1300 alike at
// x = 2^18 had probabilities with the sum 77, and from 2^24 on rows could come out as 0).
// Rows with more scores than fit read their lists for every evaluation.  Lists have an
// order that depends on the scores alone, and sums one that depends on the lists.
#include "ea_common.h"
#include "ea_internal.h"

namespace ea {

namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));

// v and its neighbours in other lanes of 16, by the VALU alone.
template <int CTRL>
__device__ __forceinline__ float dpp(float v) {
#if defined(__HIP_DEVICE_COMPILE__)
  return __uint_as_float(
      (uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(v), CTRL, 0xf, 0xf, true));
#else
  return v;
#endif
}
constexpr int QUAD_1032 = 0xB1, QUAD_2301 = 0x4E, HALF_MIRROR = 0x141, MIRROR = 0x140;
constexpr int ROW_ROR_4 = 0x124, ROW_ROR_8 = 0x128;
template <typename F>
__device__ __forceinline__ float fold8(float v, F&& f) {
  v = f(v, dpp<QUAD_1032>(v));
  v = f(v, dpp<QUAD_2301>(v));
  return f(v, dpp<HALF_MIRROR>(v));
}
template <typename F>
__device__ __forceinline__ float fold16(float v, F&& f) {
  v = fold8(v, f);
  return f(v, dpp<MIRROR>(v));
}
// over the four lanes that are 16 apart
template <typename F>
__device__ __forceinline__ float fold_rows(float v, F&& f) {
#if defined(__HIP_DEVICE_COMPILE__)
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = f(__uint_as_float(r[0]), __uint_as_float(r[1]));
#endif
  float lo, hi;
  wave_halves(v, lo, hi);
  return f(lo, hi);
}
template <typename F>
__device__ __forceinline__ float fold64(float v, F&& f) {
  return fold_rows(fold16(v, f), f);
}
__device__ __forceinline__ float addf(float a, float b) { return a + b; }
__device__ __forceinline__ float maxf(float a, float b) { return fmaxf(a, b); }

__device__ __forceinline__ int query_length(const PagedArgs& a, int i) {
  return min(max(((const ci32*)a.lengths)[i], 0), a.longest);
}
__device__ __forceinline__ int query_row(const PagedArgs& a, int i) {
  return a.rows ? ((const ci32*)a.rows)[i] : i;
}

// ------------------------------------------------------------------ scores

constexpr int PS_NT = 256, PS_WAVES = 4;
constexpr int PS_KEYS = PAGED_REGION / PS_WAVES;  // of a wave
constexpr int PS_TILES = PS_KEYS / PAGE_TILE;
// Tiles in flight, each place taken again once its tile's scores are there.  (All 16 at
// once leave registers for three waves instead of four: 64 requests of up to 9216 keys,
// 32/8 heads, d = 128, 40.5 us against 38.0; four 38.6.)
constexpr int PS_AHEAD = 8;
constexpr int PS_CHUNK = 4;  // tiles that are left out together where a row ends before them
constexpr int PS_HEADS = 16;  // query heads of a workgroup, the rows of a product
constexpr int PS_STEPS = 4;   // Newton's steps of a region's bound

template <typename E>
constexpr int digits() {
  return sizeof(E) == 2 ? 4 : 6;
}

// The rows of a product that heads have: a lane holds four rows of it, and a group of
// up to four heads fills one of them in every lane.
__device__ __forceinline__ int row_of_head(int j) { return (j & 3) * 4 + (j >> 2); }

template <int CTRL>
__device__ __forceinline__ int dpp_int(int v) {
#if defined(__HIP_DEVICE_COMPILE__)
  return __builtin_amdgcn_update_dpp(0, v, CTRL, 0xf, 0xf, true);
#else
  return v;
#endif
}

// A lower bound of tau: the root of f restricted to the scores v of 16 lanes, `top`
// the largest of them, by Newton's steps from c top - 1 on, which stay below it.  It is
// less by the sums' rounding, and NaN where the largest is not finite.
template <int GK>
__device__ __forceinline__ float region_bound_of(const float (&v)[PS_WAVES], float top, float c, float gamma) {
  float lo = c * top - 1.f;
#pragma unroll 1
  for (int it = 0; it < PS_STEPS; ++it) {
    float s0 = 0.f, s1 = 0.f;
#pragma unroll
    for (int y = 0; y < PS_WAVES; ++y) {
      float p, u;
      Gamma<GK>::pu(relu_z(c, v[y], lo), gamma, p, u);
      s0 += p;
      s1 += u;
    }
    s0 = fold16(s0, addf);
    s1 = fold16(s1, addf);
    lo += fmaxf((s0 - 1.f) * __builtin_amdgcn_rcpf(gamma * s1), 0.f);
  }
  return lo - 4e-6f * fmaxf(1.f, fabsf(lo));
}
__device__ __forceinline__ float region_bound(const PagedArgs& a, const float (&v)[PS_WAVES], float top) {
  switch (a.gk) {
    case 1: return region_bound_of<1>(v, top, a.scale_c, a.gamma);
    case 2: return region_bound_of<2>(v, top, a.scale_c, a.gamma);
    case 4: return region_bound_of<4>(v, top, a.scale_c, a.gamma);
  }
  return region_bound_of<0>(v, top, a.scale_c, a.gamma);
}

// Queries in digits: `heads` of them from head h0 of query i on.
template <typename E, int D>
struct Digits {
  static constexpr int T = digits<E>();
  uint8_t digit[T][PS_HEADS][D];
  uint8_t unit[T][PS_HEADS][D / 32];

  template <int NT>
  __device__ __forceinline__ void take(const PagedArgs& a, int i, int h0, int heads) {
    for (int c = threadIdx.x; c < heads * (D / 4); c += NT) {
      const int j = c / (D / 4), at = c % (D / 4) * 4;
      const E* const p = static_cast<const E*>(a.q) + i * a.q_row + (h0 + j) * a.q_head + at;
      float y[4];
      if constexpr (sizeof(E) == 2) {
        const u32x2 v = *reinterpret_cast<const u32x2*>(p);
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          y[2 * e] = __uint_as_float(v[e] << 16);
          y[2 * e + 1] = __uint_as_float(v[e] & 0xFFFF0000u);
        }
      } else {
        const f32x4 v = *reinterpret_cast<const f32x4*>(p);
#pragma unroll
        for (int e = 0; e < 4; ++e) y[e] = v[e];
      }
      // (non-negative floats compare as integers do; NaN is the largest)
      uint32_t m = 0;
#pragma unroll
      for (int e = 0; e < 4; ++e) m = max(m, __float_as_uint(y[e]) & 0x7FFFFFFFu);
      m = __float_as_uint(fold8(__uint_as_float(m), [](float p, float q) {
        return __uint_as_float(max(__float_as_uint(p), __float_as_uint(q)));
      }));
      const int e0 = (int)(m >> 23);  // units of 2^(e0 - 127 - 3)
      const bool finite = e0 != 255;
#pragma unroll
      for (int e = 0; e < 4; ++e) y[e] = finite ? ldexpf(y[e], 130 - e0) : 0.f;
      const int r = row_of_head(j);
#pragma unroll
      for (int d = 0; d < T; ++d) {
        float n[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          n[e] = rintf(y[e]);
          y[e] = (y[e] - n[e]) * 32.f;
        }
        int word = 0;
#if defined(__HIP_DEVICE_COMPILE__)
        word = __builtin_amdgcn_cvt_pk_fp8_f32(n[0], n[1], word, false);
        word = __builtin_amdgcn_cvt_pk_fp8_f32(n[2], n[3], word, true);
#endif
        const int scale = e0 - 3 - 5 * d;  // (digits under 2^-127 are dropped)
        *reinterpret_cast<int*>(&digit[d][r][at]) = scale < 0 ? 0 : word;
        if ((c & 7) == 0) unit[d][r][at / 32] = finite ? (uint8_t)max(scale, 0) : 255;
      }
    }
  }
};

// A wave's TILES tiles of keys, tile u from key k0 + u step on, against up to 16 heads:
// R4 registers of scores to a tile, heads 4 at a time.
template <typename E, int D, int R4, int TILES>
struct WaveKeys {
  static constexpr int T = digits<E>(), NM = T * D / 128;  // products of a tile
  static constexpr int SB = D / 32, AHEAD = TILES < PS_AHEAD ? TILES : PS_AHEAD;
  static_assert(TILES <= 16 && TILES % PS_CHUNK == 0, "a lane of 16 for each tile's page");
  const PagedArgs& a;
  const int kv, k0, step, len, col, g;
  int ids;  // page of tile `col`, -1 where there is none
  i32x4 kf[AHEAD];
  int ks[AHEAD];

  __device__ __forceinline__ WaveKeys(const PagedArgs& args, int i, int kv_head, int first, int apart, int length)
      : a(args), kv(kv_head), k0(first), step(apart), len(length), col(lane_id() & 15), g(lane_id() >> 4) {
    const int key = k0 + col * step;
    ids = col < TILES && key < len ? page_of(a.c, a.t, query_row(a, i), key) : -1;
#pragma unroll
    for (int c = 0; c < AHEAD; c += PS_CHUNK) load(c);
  }
  __device__ __forceinline__ void load(int c) {  // chunk c of the tiles
    if (k0 + c * step >= len) return;
#pragma unroll
    for (int u = c; u < c + PS_CHUNK; ++u) {
      // (a tile without a page reads the first one's, and its scores are dropped)
      const int page = max(__builtin_amdgcn_readlane(ids, u), 0);
      const uint8_t* const tile = a.cache + tile_at(a.c, page, kv, false, k0 + u * step);
      const int part = D == 128 ? g : g & 1;
      kf[u % AHEAD] = __builtin_nontemporal_load(reinterpret_cast<const i32x4*>(tile + (uint32_t)(col * (D / 2) + part * 16)));
      ks[u % AHEAD] = tile[(uint32_t)(PAGE_TILE * (D / 2) + col * SB + part)];
    }
  }
  // s: of head g + 4 r and the tiles' key `col` (-inf: none); top: the lane's largest
  __device__ __forceinline__ void scores(const Digits<E, D>& q, float (&s)[TILES][R4], float (&top)[R4]) {
    // A operands: of 128 values a lane holds 16 g .. and 64 + 16 g .., and the scale
    // of block g; at D = 64 two digits are one operand, K's row twice the other
    i32x8 qf[NM];
    int qs[NM];
#pragma unroll
    for (int m = 0; m < NM; ++m) {
      const i32x4 lo = *reinterpret_cast<const i32x4*>(D == 128 ? &q.digit[m][col][16 * g] : &q.digit[2 * m][col][16 * g]);
      const i32x4 hi = *reinterpret_cast<const i32x4*>(D == 128 ? &q.digit[m][col][64 % D + 16 * g]
                                                                : &q.digit[(2 * m + 1) % T][col][16 * g]);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        qf[m][e] = lo[e];
        qf[m][4 + e] = hi[e];
      }
      qs[m] = D == 128 ? q.unit[m][col][g % SB] : q.unit[(2 * m + (g >> 1)) % T][col][g & 1];
    }
#pragma unroll
    for (int u = 0; u < TILES; ++u)
#pragma unroll
      for (int r = 0; r < R4; ++r) s[u][r] = -INFINITY;
#pragma unroll
    for (int r = 0; r < R4; ++r) top[r] = -INFINITY;
#pragma unroll
    for (int c = 0; c < TILES; c += PS_CHUNK) {
      if (k0 + c * step >= len) break;
#pragma unroll
      for (int u = c; u < c + PS_CHUNK; ++u) {
        f32x4 v = {0.f, 0.f, 0.f, 0.f};
#if defined(__HIP_DEVICE_COMPILE__)
        const i32x4 kw = kf[u % AHEAD];
        const i32x8 k = {kw[0], kw[1], kw[2], kw[3], 0, 0, 0, 0};
#pragma unroll
        for (int m = NM - 1; m >= 0; --m)  // (the smallest first)
          v = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(qf[m], k, v, 0, 4, 0, qs[m], 0, ks[u % AHEAD]);
#endif
        const bool ok = k0 + u * step + col < len && __builtin_amdgcn_readlane(ids, u) >= 0;
#pragma unroll
        for (int r = 0; r < R4; ++r) {
          s[u][r] = ok ? v[r] : -INFINITY;
          top[r] = fmaxf(top[r], s[u][r]);  // (a NaN is left out)
        }
      }
      if (c + AHEAD < TILES) load(c + AHEAD);
    }
  }
  // where the lane's key of tile u lies in the pool
  __device__ __forceinline__ uint32_t slot(int u) const {
    return ((uint32_t)__builtin_amdgcn_readlane(ids, u) << a.c.shift) +
           (uint32_t)((k0 + u * step) & ((1 << a.c.shift) - 1)) + col;
  }
  // The lane's scores above `bound`, a bit for each tile; where they go among those of the
  // 16 lanes of its row, and how many these have (in the last of them).
  __device__ __forceinline__ static int above(const float (&s)[TILES][R4], int r, float c, float bound, int& to, int& all) {
    int mine = 0;
#pragma unroll
    for (int u = 0; u < TILES; ++u) mine |= relu_z(c, s[u][r], bound) > 0.f ? 1 << u : 0;
    const int n = __popc(mine);
    all = n;
    all += dpp_int<0x111>(all);  // row_shr 1, 2, 4, 8: sums over the lanes up to each
    all += dpp_int<0x112>(all);
    all += dpp_int<0x114>(all);
    all += dpp_int<0x118>(all);
    to = all - n;
    return mine;
  }
  __device__ __forceinline__ void write(const float (&s)[TILES][R4], int r, int mine, u32x2_t* at) const {
#pragma unroll
    for (int u = 0; u < TILES; ++u)
      if (mine & 1 << u) *at++ = u32x2_t{__float_as_uint(s[u][r]), slot(u)};
  }
};

// A workgroup per region of keys, query, key head and 16 of its query heads.
template <typename E, int D, int R4>
__global__ __launch_bounds__(PS_NT) void paged_scores_kernel(PagedArgs a, int head_tiles) {
  using W = WaveKeys<E, D, R4, PS_TILES>;
  __shared__ __attribute__((aligned(16))) Digits<E, D> q;
  __shared__ float lane_top[PS_WAVES][PS_HEADS][16];
  __shared__ int wave_count[PS_WAVES][PS_HEADS];
  __shared__ float head_top[PS_HEADS], head_bound[PS_HEADS];
  const int lane = lane_id(), w = wave_id(), col = lane & 15, g = lane >> 4;
  int x = blockIdx.x;
  const int kv = x % a.c.kv_heads;
  x /= a.c.kv_heads;
  const int ht = x % head_tiles;
  x /= head_tiles;
  const int region = x % a.regions, i = x / a.regions;
  const int len = query_length(a, i), first = region * PAGED_REGION;
  if (first >= len) return;
  const int heads = min(PS_HEADS, a.group - ht * PS_HEADS), h0 = kv * a.group + ht * PS_HEADS;
  W keys(a, i, kv, first + w * PS_KEYS, PAGE_TILE, len);
  q.template take<PS_NT>(a, i, h0, heads);
  __syncthreads();
  float s[PS_TILES][R4], top[R4];
  keys.scores(q, s, top);
  // ---- a lower bound of tau from the largest scores of the lanes, which are scores of
  // 64 keys of the region, and what is above it
#pragma unroll
  for (int r = 0; r < R4; ++r) lane_top[w][g + 4 * r][col] = top[r];
  __syncthreads();
  // A wave bounds the four heads of its lane groups: each four by a wave of their own and
  // a barrier more, but up to four heads by every wave for itself. Whole calls: 8 rows of
  // 30000 keys, 40/2 heads, 33.3 us, and 35.8 with every wave bounding all; 16 of 8000,
  // 16/1 heads, 18.7 and 20.1; 64 of 9000, 32/4 heads, 39.5 and 40.5. With four heads the
  // barrier costs more than it saves: this kernel took 33.6 us so on 65536 keys, 32.5
  // without.
  auto bound_of = [&](int j, float& largest) {
    float v[PS_WAVES];
#pragma unroll
    for (int y = 0; y < PS_WAVES; ++y) v[y] = lane_top[y][j][col];
    largest = fold16(fmaxf(fmaxf(v[0], v[1]), fmaxf(v[2], v[3])), maxf);
    const float lo = region_bound(a, v, largest);
    return j < heads ? lo : INFINITY;
  };
  float bound[R4];
  if constexpr (R4 == 1) {
    bound[0] = bound_of(g, top[0]);
  } else {
    if (w < R4) {
      float largest;
      const float lo = bound_of(g + 4 * w, largest);
      if (col == 0) {
        head_top[g + 4 * w] = largest;
        head_bound[g + 4 * w] = lo;
      }
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < R4; ++r) {
      top[r] = head_top[g + 4 * r];
      bound[r] = head_bound[g + 4 * r];
    }
  }
  int mine[R4], to[R4];
#pragma unroll
  for (int r = 0; r < R4; ++r) {
    int all;
    mine[r] = W::above(s, r, a.scale_c, bound[r], to[r], all);
    if (col == 15) wave_count[w][g + 4 * r] = all;
  }
  __syncthreads();
#pragma unroll
  for (int r = 0; r < R4; ++r) {
    const int j = g + 4 * r;
    const int64_t list = ((int64_t)i * a.heads + h0 + min(j, heads - 1)) * a.regions + region;
    int all = 0;
#pragma unroll
    for (int y = 0; y < PS_WAVES; ++y) {
      const int n = wave_count[y][j];
      to[r] += y < w ? n : 0;
      all += n;
    }
    if (w == 0 && col == 0 && j < heads)
      a.tops[list] = u32x4_t{__float_as_uint(top[r]), __float_as_uint(bound[r]), (uint32_t)all, 0};
    keys.write(s, r, mine[r], a.list + list * PAGED_REGION + to[r]);
  }
}

// ------------------------------------------------------------------- solve

constexpr int MAX_REGIONS = MAX_SEQLEN / PAGED_REGION;
constexpr int PV_VALS = 16;   // values of V that a lane takes of a row
constexpr int PV_BATCH = 8;   // rows of V of a lane in flight

// z^gamma, z^(gamma-1), z^(gamma-2) summed over z > 0
template <int GK>
__device__ __forceinline__ void add_z(float z, float gamma, float& s0, float& s1, float& s2) {
  if (z > 0.f) {
    float p, u;
    Gamma<GK>::pu(z, gamma, p, u);
    s0 += p;
    s1 += u;
    if constexpr (GK == 2) s2 += 1.f;
    if constexpr (GK == 4) s2 += z * z;
    if constexpr (GK == 0) s2 += u / z;
  }
}

// tau - max x of a row of `len` keys from its bound lo on: Algorithm 1's iteration.
// sums(tau, s0, s1, s2): of all of the row's scores.
template <typename F>
__device__ __forceinline__ float solve_tau(const PagedArgs& a, float lo, int len, F&& sums) {
  const float gm = a.gamma;
  // (all keys alike, and a little more for the functions' rounding)
  float hi = -0.999998f * exp2f((1.f - a.alpha) * __log2f((float)len));
  float low = fminf(lo, hi), tau = low;
  for (int it = 0;; ++it) {
    float s0 = 0.f, s1 = 0.f, s2 = 0.f;
    sums(tau, s0, s1, s2);
    const float f = s0 - 1.f;
    const bool stop = fabsf(f) <= a.tol || it >= a.max_iter;
    // B_f, Newton's bound, H_f: the update rules of the attention solver
    const float f1 = -gm * s1, f2 = gm * (gm - 1.f) * s2;
    if (f < 0.f)
      hi = tau;
    else
      low = tau;
    const float slack = 1e-6f * fmaxf(1.f, fmaxf(fabsf(low), fabsf(hi)));
    if (f1 < 0.f) low = fminf(fmaxf(low, tau - f * __builtin_amdgcn_rcpf(f1) - 10.f * slack), hi);
    const float th = tau - 2.f * f * f1 * __builtin_amdgcn_rcpf(2.f * f1 * f1 - f * f2);
    const bool take = th >= low - slack && th <= hi + slack;
    // (the update from the last evaluation is taken too)
    tau = take ? fminf(fmaxf(th, low), hi) : th < low ? low : 0.5f * (low + hi);
    if (stop) return tau;
  }
}

// The sum of rows of V times their probabilities: LPK lanes to a row, each 16 values of it
// (half a block).
template <int D>
struct RowSum {
  static constexpr int LPK = D / PV_VALS, KPW = 64 / LPK;  // lanes of a row, rows of a wave
  float o[PV_VALS];
  const uint8_t* V;  // the values of the key head in page 0
  int64_t page_step;
  int shift, sub, grp;

  __device__ __forceinline__ RowSum(const PagedArgs& a, int kv)
      : o{}, V(a.cache + tile_at(a.c, 0, kv, true, 0)), page_step(page_bytes(a.c)), shift(a.c.shift),
        sub(lane_id() % LPK), grp(lane_id() / LPK) {}
  // Adds entries (p, place in the pool) list[first], list[first + 1] .. KPW at a time, and then those
  // `step` behind, up to n.
  __device__ __forceinline__ void add(const u32x2_t* list, int first, int step, int n) {
    for (int e0 = first; e0 < n; e0 += step * PV_BATCH) {
      u32x2 codes[PV_BATCH];
      float p[PV_BATCH];
      uint32_t scale[PV_BATCH];
#pragma unroll
      for (int u = 0; u < PV_BATCH; ++u) {
        const u32x2_t v = list[min(e0 + u * step + grp, n - 1)];
        p[u] = __uint_as_float(v[0]);
        const int at = (int)(v[1] & ((1u << shift) - 1));
        const uint8_t* const tile = V + (int64_t)(v[1] >> shift) * page_step + (at >> 4) * tile_bytes(D);
        codes[u] = *reinterpret_cast<const u32x2*>(tile + (at & 15) * (D / 2) + 8 * sub);
        scale[u] = tile[PAGE_TILE * (D / 2) + (at & 15) * (D / 32) + sub / 2];
      }
#pragma unroll
      for (int u = 0; u < PV_BATCH; ++u) {
        if (e0 + u * step >= n) break;
        // (a row again in the place of none: whatever it holds is not used)
#if defined(__HIP_DEVICE_COMPILE__)
        const float ps = e0 + u * step + grp >= n ? 0.f
                         : scale[u] == 255        ? __builtin_nanf("")
                                                  : p[u] * __uint_as_float(scale[u] << 23);
        auto two = [&](int at, auto v) {
          o[at] = fmaf(ps, v[0], o[at]);
          o[at + 1] = fmaf(ps, v[1], o[at + 1]);
        };
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          two(8 * x, __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes[u][x], 1.f, 0));
          two(8 * x + 2, __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes[u][x], 1.f, 1));
          two(8 * x + 4, __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes[u][x], 1.f, 2));
          two(8 * x + 6, __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes[u][x], 1.f, 3));
        }
#endif
      }
    }
  }
  // the wave's sums
  __device__ __forceinline__ void store(float (&sums)[D]) {
#pragma unroll
    for (int d = 0; d < PV_VALS; ++d) {
      // (lanes rotate inside 16, then rows and halves swap: no LDS)
      if constexpr (LPK == 4) o[d] += dpp<ROW_ROR_4>(o[d]);
      o[d] = fold_rows(o[d] + dpp<ROW_ROR_8>(o[d]), addf);
    }
    if (grp == 0)
#pragma unroll
      for (int d = 0; d < PV_VALS; d += 4)
        *reinterpret_cast<f32x4*>(&sums[sub * PV_VALS + d]) = f32x4{o[d], o[d + 1], o[d + 2], o[d + 3]};
  }
};

// How far an entry's score lies from the largest one.
__device__ __forceinline__ float below(const u32x2_t& v, float top) { return __uint_as_float(v[0]) - top; }

// Of n entries with scores, the largest of them `top`, those with a probability move to the
// front, p in place of the score (a wave; no entry is overwritten before it has been read).
// Their number.
template <int GK>
__device__ __forceinline__ int keep_probable(const PagedArgs& a, u32x2_t* list, int n, float top, float tau) {
  const int lane = lane_id();
  int np = 0;
  for (int e0 = 0; e0 < n; e0 += 64) {
    u32x2_t v = {0xFF800000u, 0};
    if (e0 + lane < n) v = list[e0 + lane];
    const float p = Gamma<GK>::p_only(relu_z(a.scale_c, below(v, top), tau), a.gamma);
    const uint64_t k = __ballot(p > 0.f);
    if (p > 0.f) {
      v[0] = __float_as_uint(p);
      list[np + __popcll(k & ((1ull << lane) - 1))] = v;
    }
    np += __popcll(k);
  }
  return np;
}

constexpr int SO_LANE = 8;              // scores per lane of a wave that solves a row alone
constexpr int SO_FEW = 64 * SO_LANE;
constexpr int SO_OWN = 16;              // scores per thread of a workgroup that solves one
constexpr int SO_BUFFER = 256;          // entries on their way to a wave's gather

// Rows with few scores above the bound are the first wave's alone, without barriers.
// (With the other waves for a share of the rows of V: one request of 9000 keys, 32 heads,
// 16.1 us against 16.3, 64 requests 53.8 against 49.9.)  Rows with more are solved by all of
// them: each thread keeps SO_OWN scores, and reads the others of its own for every evaluation.
template <typename E, int D, int GK, int NT>
__global__ __launch_bounds__(NT) void paged_solve_kernel(PagedArgs a) {
  constexpr int WAVES = NT / 64, KPW = RowSum<D>::KPW;
  static_assert(WAVES * SO_BUFFER >= SO_FEW, "a wave's scores fit in the place of all buffers");
  __shared__ u32x2_t buffer[WAVES][SO_BUFFER];
  __shared__ __attribute__((aligned(16))) float sums[WAVES][D];
  __shared__ float red[2][3][WAVES];
  __shared__ int starts[MAX_REGIONS + 1];
  __shared__ float row_top, row_bound;
  const int t = threadIdx.x, lane = lane_id(), w = wave_id();
  // (heads of one key head are kv_heads apart: with eight of them, on one XCD)
  const int i = blockIdx.x / a.heads, y = blockIdx.x % a.heads;
  const int kv = y % a.c.kv_heads, h = kv * a.group + y / a.c.kv_heads;
  const int64_t row = ((int64_t)i * a.heads + h) * a.regions;
  E* const O = static_cast<E*>(a.o) + i * a.o_row + h * a.o_head;
  const float c = a.scale_c, gm = a.gamma;

  // ---- the regions' largest scores and bounds, and from them a bound of the row; where each
  // region's listed scores start among all that are looked at (none, where its largest is
  // below the bound)
  if (w == 0) {
    // (read before the length has come: regions behind it are not looked at)
    float top[MAX_REGIONS / 64], m = -INFINITY, lo = -INFINITY;
    u32x4_t found[MAX_REGIONS / 64];
#pragma unroll
    for (int e = 0; e < MAX_REGIONS / 64; ++e) {
      found[e] = u32x4_t{0, 0, 0, 0};
      if (64 * e + lane < a.regions) found[e] = a.tops[row + 64 * e + lane];
    }
    const int regions = (query_length(a, i) + PAGED_REGION - 1) / PAGED_REGION;
#pragma unroll
    for (int e = 0; e < MAX_REGIONS / 64; ++e) {
      const bool there = 64 * e + lane < regions;
      top[e] = there ? __uint_as_float(found[e][0]) : -INFINITY;
      m = fmaxf(m, top[e]);
      if (there) lo = fmaxf(lo, __uint_as_float(found[e][1]));  // (the best of the regions' bounds)
    }
    const float most = fold64(m, maxf);
    m = c * most;
    lo = fmaxf(fold64(lo, maxf) - m, -1.f);  // (from here on against max x)
    const bool any = m > -INFINITY && m < INFINITY;
#pragma unroll
    for (int e = 0; e < MAX_REGIONS / 64; ++e) top[e] -= most;
    for (int it = 0; any && it < 8; ++it) {
      float s0 = 0.f, s1 = 0.f, s2 = 0.f;
#pragma unroll
      for (int e = 0; e < MAX_REGIONS / 64; ++e) add_z<GK>(relu_z(c, top[e], lo), gm, s0, s1, s2);
      s0 = fold64(s0, addf);
      s1 = fold64(s1, addf);
      const float step = (s0 - 1.f) * __builtin_amdgcn_rcpf(gm * s1);
      if (!(step > 1e-3f)) break;  // (no key is above it where s1 is 0)
      lo += step;
      if (!(step > 1e-2f)) break;
    }
    lo = fmaxf(lo - 4e-6f, -1.f);  // (the sums' rounding)
    int base = 0;
#pragma unroll
    for (int e = 0; e < MAX_REGIONS / 64; ++e) {
      const int n = any && relu_z(c, top[e], lo) > 0.f ? (int)found[e][2] : 0;
      int incl = n;
#pragma unroll
      for (int x = 1; x < 64; x <<= 1) {
        const int v = __shfl_up(incl, x);
        if (lane >= x) incl += v;
      }
      starts[64 * e + lane] = base + incl - n;
      base += __builtin_amdgcn_readlane(incl, 63);
    }
    if (lane == 0) {
      starts[MAX_REGIONS] = base;
      row_top = most;
      row_bound = lo;
    }
  }
  __syncthreads();
  const int entries = __builtin_amdgcn_readfirstlane(starts[MAX_REGIONS]);
  if (entries == 0) {  // no keys, or none with a finite score
    for (int d = t; d < D; d += NT) O[d] = (E)0.f;
    return;
  }
  const float top = row_top, lo = row_bound;
  const int len = query_length(a, i);
  auto entry = [&](int e) {  // number e of them
    int x = 0;  // the last region that starts at or before it
#pragma unroll
    for (int step = MAX_REGIONS / 2; step; step >>= 1)
      if (starts[x + step] <= e) x += step;
    return a.list + (row + x) * PAGED_REGION + (e - starts[x]);
  };
  RowSum<D> o(a, kv);

  if (entries <= SO_FEW) {
    if (w) return;
    u32x2_t* const kept = buffer[0];
    float own[SO_LANE];
    u32x2_t v[SO_LANE];
#pragma unroll
    for (int e = 0; e < SO_LANE; ++e) {
      v[e] = u32x2_t{0xFF800000u, 0};  // (-inf)
      if (64 * e + lane < entries) v[e] = *entry(64 * e + lane);
    }
#pragma unroll
    for (int e = 0; e < SO_LANE; ++e) {
      own[e] = below(v[e], top);
      if (64 * e + lane < entries) kept[64 * e + lane] = v[e];
    }
    const float tau = solve_tau(a, lo, len, [&](float tau, float& s0, float& s1, float& s2) {
#pragma unroll
      for (int e = 0; e < SO_LANE; ++e) {
        if (64 * e >= entries) break;
        add_z<GK>(relu_z(c, own[e], tau), gm, s0, s1, s2);
      }
      s0 = fold64(s0, addf);
      s1 = fold64(s1, addf);
      s2 = fold64(s2, addf);
    });
    o.add(kept, 0, KPW, keep_probable<GK>(a, kept, entries, top, tau));
    o.store(sums[0]);
    for (int d = lane; d < D; d += 64) O[d] = (E)sums[0][d];
    return;
  }
  {
    // a thread's entries are t, t + NT ..
    u32x2_t own[SO_OWN];
#pragma unroll
    for (int e = 0; e < SO_OWN; ++e) {
      own[e] = u32x2_t{0xFF800000u, 0};  // (-inf)
      if (e * NT + t < entries) own[e] = *entry(e * NT + t);
      own[e][0] = __float_as_uint(below(own[e], top));
    }
    int turn = 0;
    const float tau = solve_tau(a, lo, len, [&](float tau, float& s0, float& s1, float& s2) {
#pragma unroll
      for (int e = 0; e < SO_OWN; ++e) {
        if (e * NT >= entries) break;
        add_z<GK>(relu_z(c, __uint_as_float(own[e][0]), tau), gm, s0, s1, s2);
      }
#pragma unroll 4
      for (int e = SO_OWN * NT + t; e < entries; e += NT)
        add_z<GK>(relu_z(c, below(*entry(e), top), tau), gm, s0, s1, s2);
      s0 = fold64(s0, addf);
      s1 = fold64(s1, addf);
      s2 = fold64(s2, addf);
      // (two buffers in turn: one barrier)
      auto& r = red[turn];
      turn ^= 1;
      if (lane == 0) {
        r[0][w] = s0;
        r[1][w] = s1;
        r[2][w] = s2;
      }
      __syncthreads();
      s0 = s1 = s2 = 0.f;
#pragma unroll
      for (int x = 0; x < WAVES; ++x) {
        s0 += r[0][x];
        s1 += r[1][x];
        s2 += r[2][x];
      }
    });
    // those with a probability go through the wave's buffer
    int n = 0;
    const uint64_t before = (1ull << lane) - 1;
    auto take = [&](const u32x2_t& v) {  // (against the largest score)
      const float p = Gamma<GK>::p_only(relu_z(c, __uint_as_float(v[0]), tau), gm);
      const uint64_t k = __ballot(p > 0.f);
      if (p > 0.f) buffer[w][n + __popcll(k & before)] = u32x2_t{__float_as_uint(p), v[1]};
      n += __popcll(k);
      if (n > SO_BUFFER - 64) {
        o.add(buffer[w], 0, KPW, n);
        n = 0;
      }
    };
#pragma unroll
    for (int e = 0; e < SO_OWN; ++e) {
      if (e * NT + 64 * w >= entries) break;
      take(own[e]);
    }
    for (int e0 = SO_OWN * NT + 64 * w; e0 < entries; e0 += NT) {
      u32x2_t v = {0xFF800000u, 0};
      if (e0 + lane < entries) v = *entry(e0 + lane);
      v[0] = __float_as_uint(below(v, top));
      take(v);
    }
    o.add(buffer[w], 0, KPW, n);
  }
  // sums over the rows of a wave, then over the waves
  o.store(sums[w]);
  __syncthreads();
  for (int d = t; d < D; d += NT) {
    float sum = 0.f;
#pragma unroll
    for (int x = 0; x < WAVES; ++x) sum += sums[x][d];
    O[d] = (E)sum;
  }
}

// ------------------------------------------------------------- short rows

// Both steps in one workgroup per query, key head and 16 of its query heads, for rows of
// which 16 waves hold all scores at once: no lists in memory (but those of rows with
// more scores above the bound than fit), and one launch.
constexpr int SH_NT = 1024, SH_WAVES = SH_NT / 64;
// Tiles of a wave, which with R4 registers of scores each leave it its 128 registers.  (16
// of four heads fit too, but from 2048 keys on one compute unit's loads take longer than a
// second launch: one request of 4096 keys, 16/4 heads, d = 128, 16.4 us against 13.7.)
constexpr int sh_tiles(int r4) { return r4 <= 2 ? 8 : 4; }
constexpr int SH_LIST = 1024;  // entries of the heads of one register of scores

// tau of one head from its n listed scores, the largest `top`, by one wave; then the list
// holds those with a probability, and their number comes back.
template <int GK>
__device__ __forceinline__ int solve_short(const PagedArgs& a, u32x2_t* list, int n, float lo, float top, int len) {
  constexpr int ALONE = 8;
  const int lane = lane_id();
  float own[ALONE];
#pragma unroll
  for (int e = 0; e < ALONE; ++e) own[e] = 64 * e + lane < n ? below(list[64 * e + lane], top) : -INFINITY;
  const float tau = solve_tau(a, lo, len, [&](float tau, float& s0, float& s1, float& s2) {
#pragma unroll
    for (int e = 0; e < ALONE; ++e) {
      if (64 * e >= n) break;
      add_z<GK>(relu_z(a.scale_c, own[e], tau), a.gamma, s0, s1, s2);
    }
    for (int e = 64 * ALONE + lane; e < n; e += 64)
      add_z<GK>(relu_z(a.scale_c, below(list[e], top), tau), a.gamma, s0, s1, s2);
    s0 = fold64(s0, addf);
    s1 = fold64(s1, addf);
    s2 = fold64(s2, addf);
  });
  return keep_probable<GK>(a, list, n, top, tau);
}

template <typename E, int D, int R4>
__global__ __launch_bounds__(SH_NT) void paged_short_kernel(PagedArgs a, int head_tiles) {
  constexpr int TILES = sh_tiles(R4), HEADS = 4 * R4, CAP = SH_LIST / R4;
  constexpr int WPH = R4 == 1 ? 4 : R4 == 2 ? 2 : 1;  // waves that add up one head's rows of V
  using W = WaveKeys<E, D, R4, TILES>;
  __shared__ __attribute__((aligned(16))) Digits<E, D> q;
  __shared__ float lane_top[SH_WAVES][HEADS][16];
  __shared__ int wave_count[SH_WAVES][HEADS];
  __shared__ u32x2_t lists[HEADS][CAP];
  __shared__ float head_top[HEADS], head_bound[HEADS];
  __shared__ int head_count[HEADS];
  static_assert(sizeof(q) >= SH_WAVES * D * sizeof(float), "the waves' sums fit in place of the digits");
  const int t = threadIdx.x, lane = lane_id(), w = wave_id(), col = lane & 15, g = lane >> 4;
  int x = blockIdx.x;
  const int kv = x % a.c.kv_heads;
  x /= a.c.kv_heads;
  const int ht = x % head_tiles, i = x / head_tiles;
  const int len = query_length(a, i);
  const int heads = min(PS_HEADS, a.group - ht * PS_HEADS), h0 = kv * a.group + ht * PS_HEADS;
  // (a wave's tiles are 16 apart, so that a few tiles are of as many waves)
  W keys(a, i, kv, w * PAGE_TILE, SH_WAVES * PAGE_TILE, len);
  q.template take<SH_NT>(a, i, h0, heads);
  __syncthreads();
  float s[TILES][R4], top[R4];
  keys.scores(q, s, top);
#pragma unroll
  for (int r = 0; r < R4; ++r) lane_top[w][g + 4 * r][col] = top[r];
  __syncthreads();
  // (a wave to each register of heads: the others would repeat its arithmetic)
  if (w < R4) {
    const int j = g + 4 * w;
    float v[PS_WAVES];
#pragma unroll
    for (int y = 0; y < PS_WAVES; ++y) {
      v[y] = lane_top[y][j][col];
#pragma unroll
      for (int z = PS_WAVES; z < SH_WAVES; z += PS_WAVES) v[y] = fmaxf(v[y], lane_top[y + z][j][col]);
    }
    const float m = fold16(fmaxf(fmaxf(v[0], v[1]), fmaxf(v[2], v[3])), maxf);
    const float lo = region_bound(a, v, m);
    if (col == 0) {
      head_top[j] = m;
      head_bound[j] = j < heads ? lo : INFINITY;
    }
  }
  __syncthreads();
  int mine[R4], to[R4];
#pragma unroll
  for (int r = 0; r < R4; ++r) {
    int all;
    mine[r] = W::above(s, r, a.scale_c, head_bound[g + 4 * r], to[r], all);
    if (col == 15) wave_count[w][g + 4 * r] = all;
  }
  __syncthreads();
  bool fits = true;
#pragma unroll
  for (int r = 0; r < R4; ++r) {
    const int n = wave_count[col][g + 4 * r];  // (of wave `col`)
    auto sum16 = [](int v) {  // (counts are exact in fp32)
      return (int)fold16((float)v, addf);
    };
    to[r] += sum16(col < w ? n : 0);
    const int all = sum16(n);
    fits = fits && all <= CAP;
    if (w == 0 && col == 0) head_count[g + 4 * r] = all;
  }
  fits = __all(fits);  // (every wave sees all heads)
  // entry 0 of head j's list
  auto list_of = [&](int j) -> u32x2_t* {
    return fits ? lists[j] : a.list + ((int64_t)i * a.heads + h0 + j) * a.regions * PAGED_REGION;
  };
#pragma unroll
  for (int r = 0; r < R4; ++r) keys.write(s, r, mine[r], list_of(min(g + 4 * r, heads - 1)) + to[r]);
  __syncthreads();
  // ---- a wave to a head: tau, and the keys with a probability
  if (w < heads) {
    const float top = head_top[w], m = a.scale_c * top, lo = fmaxf(head_bound[w] - m, -1.f);
    int n = 0;
    if (m > -INFINITY && m < INFINITY) {  // (else no keys, or none with a finite score)
      const int all = __builtin_amdgcn_readfirstlane(head_count[w]);
      u32x2_t* const list = list_of(w);
      switch (a.gk) {
        case 1: n = solve_short<1>(a, list, all, lo, top, len); break;
        case 2: n = solve_short<2>(a, list, all, lo, top, len); break;
        case 4: n = solve_short<4>(a, list, all, lo, top, len); break;
        default: n = solve_short<0>(a, list, all, lo, top, len);
      }
    }
    if (lane == 0) head_count[w] = n;
  }
  __syncthreads();
  // ---- their rows of V
  float(&sums)[SH_WAVES][D] = reinterpret_cast<float(&)[SH_WAVES][D]>(q);
  const int j = w / WPH;
  if (j < heads) {
    RowSum<D> o(a, kv);
    constexpr int KPW = RowSum<D>::KPW;
    o.add(list_of(j), w % WPH * KPW, WPH * KPW, __builtin_amdgcn_readfirstlane(head_count[j]));
    o.store(sums[w]);
  }
  __syncthreads();
  for (int e = t; e < heads * D; e += SH_NT) {
    const int h = e / D, d = e % D;
    float sum = 0.f;
#pragma unroll
    for (int y = 0; y < WPH; ++y) sum += sums[h * WPH + y][d];
    static_cast<E*>(a.o)[i * a.o_row + (h0 + h) * a.o_head + d] = (E)sum;
  }
}

int head_tiles(const PagedArgs& a) { return (a.group + PS_HEADS - 1) / PS_HEADS; }

int head_registers(const PagedArgs& a) { return a.group >= PS_HEADS ? 4 : (a.group + 3) / 4; }

hipError_t launch_heads(void (*kernel)(PagedArgs, int), int64_t wgs, int threads, const PagedArgs& a, hipStream_t s) {
  PagedArgs args = a;
  int tiles = head_tiles(a);
  void* params[] = {&args, &tiles};
  return hipLaunchKernel(reinterpret_cast<const void*>(kernel), dim3((unsigned)wgs), dim3(threads), params, 0, s);
}

template <typename E, int D>
hipError_t launch_scores(const PagedArgs& a, hipStream_t s) {
  const int r4 = head_registers(a);
  void (*kernel)(PagedArgs, int) = paged_scores_kernel<E, D, 1>;
  if (r4 == 2) kernel = paged_scores_kernel<E, D, 2>;
  if (r4 == 3) kernel = paged_scores_kernel<E, D, 3>;
  if (r4 == 4) kernel = paged_scores_kernel<E, D, 4>;
  return launch_heads(kernel, paged_score_wgs(a), PS_NT, a, s);
}

int64_t short_wgs(const PagedArgs& a) { return (int64_t)a.queries * head_tiles(a) * a.c.kv_heads; }

// Rows that one workgroup each takes, where every one has a compute unit: us in a graph,
// against the two kernels, 32/8 heads, d = 128, 1, 16 and 32 requests (8, 128 and 256
// workgroups) of up to 128 keys 9.3, 9.6, 9.7 against 10.6, 11.0, 11.4, of up to 1000
// 11.0, 11.1, 11.4 against 13.1, 13.2, 13.5, of up to 2000 13.0, 13.0, 13.7 against 13.4,
// 13.4, 15.9; 64 requests (512) of up to 128, 1000 and 2000 17.7, 21.0, 26.3 against 15.8, 19.4,
// 23.7.
bool short_rows(const PagedArgs& a) {
  return a.longest <= SH_WAVES * PAGE_TILE * sh_tiles(head_registers(a)) && short_wgs(a) <= 256;
}

template <typename E, int D>
hipError_t launch_short(const PagedArgs& a, hipStream_t s) {
  const int r4 = head_registers(a);
  void (*kernel)(PagedArgs, int) = paged_short_kernel<E, D, 1>;
  if (r4 == 2) kernel = paged_short_kernel<E, D, 2>;
  if (r4 == 3) kernel = paged_short_kernel<E, D, 3>;
  if (r4 == 4) kernel = paged_short_kernel<E, D, 4>;
  return launch_heads(kernel, short_wgs(a), SH_NT, a, s);
}

template <typename E, int D, int NT>
hipError_t launch_solve(const PagedArgs& a, hipStream_t s) {
  auto kernel = paged_solve_kernel<E, D, 0, NT>;
  if (a.gk == 1) kernel = paged_solve_kernel<E, D, 1, NT>;
  if (a.gk == 2) kernel = paged_solve_kernel<E, D, 2, NT>;
  if (a.gk == 4) kernel = paged_solve_kernel<E, D, 4, NT>;
  return launch_kernel(kernel, dim3((unsigned)(a.queries * a.heads)), dim3(NT), s, a);
}

template <typename E, int D>
hipError_t launch_paged(const PagedArgs& a, hipStream_t s) {
  if (short_rows(a)) return launch_short<E, D>(a, s);
  if (a.regions) {
    const hipError_t e = launch_scores<E, D>(a, s);
    if (e != hipSuccess) return e;
  }
  // Rows that have a compute unit each take 16 waves, for the dense ones: us in a graph, 32/8
  // heads, d = 128, up to 9000 keys, against four waves: 1 and 8 requests, alpha 1.5, c = 1,
  // 16.6 and 20.2 against 16.1 and 19.6; 8, alpha 1.25, c = 0.5, 44 against 74; 16 (512 rows)
  // of those 77 to 86 either way, 64 213 against 170.
  return a.queries * a.heads <= 256 ? launch_solve<E, D, 1024>(a, s) : launch_solve<E, D, 256>(a, s);
}

}  // namespace

int64_t paged_score_wgs(const PagedArgs& a) {
  return (int64_t)a.queries * a.regions * head_tiles(a) * a.c.kv_heads;
}

hipError_t launch_paged_decode(const PagedArgs& a, int dtype, hipStream_t s) {
  if (dtype == 0) return a.c.head_dim == 64 ? launch_paged<__bf16, 64>(a, s) : launch_paged<__bf16, 128>(a, s);
  return a.c.head_dim == 64 ? launch_paged<float, 64>(a, s) : launch_paged<float, 128>(a, s);
}

}  // namespace ea
