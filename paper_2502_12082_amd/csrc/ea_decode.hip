// ea_decode.hip -- alpha-entmax attention of one new token per request, over a
// prefix that all requests share and each request's own cache.
//
// For head h of request b, with keys k_j of the prefix and of the cache:
//   x_j = (alpha - 1) scale <q, k_j>,  tau: sum_j [x_j - tau]_+^gamma = 1,
//   o = sum_j [x_j - tau]_+^gamma v_j.
// tau couples all keys, so there is no sum to carry along while the keys
// stream by, as a softmax has; but few keys have a probability, so that after
// the scores only those rows of V have to be read.  Two kernels:
//
// Scores.  The queries of every request that share a key head form one matrix,
// so a prefix key is read once for all of them; a request's own cache meets
// the queries of its group.  A wave holds 32 RT queries as MFMA B operands in
// registers and streams key blocks of 32 from memory straight into A operands
// (no LDS: each key row is used by one wave).  Bound by HBM: the keys are read
// once, a score is 4 bytes written against 2 D bytes of key read for all
// queries of the head.  The maximum of every (query, key block) is written too.
//
// Solve.  One workgroup per query row.  The maxima of its blocks are scores of
// distinct keys, so f restricted to them lies below f, and its root b is a
// lower bound of tau (as the bound of the attention solver, over every block):
// only blocks with a larger maximum are read, and of those only the scores
// above b are kept, in LDS.  tau is solved on the kept scores (Algorithm 1's
// iteration), and the rows of V with a probability are gathered, 16 bytes a
// lane.  Rows that keep more than fit are solved by reading the scores of
// those blocks again for every evaluation, and gather V part by part.
// Every list keeps the order of the keys, so results do not depend on timing.
#include "ea_common.h"
#include "ea_internal.h"

namespace ea {

namespace {

constexpr int SC_NT = 256;
constexpr int SC_WAVES = SC_NT / 64;

// ------------------------------------------------------------------ scores

// Scores of DEC_RUN key blocks from block kb0 on (`blocks` in all, `keys`
// keys) against the wave's 32 RT rows from r0 on (`rows` in all):
// s[(kb * rows + r) * 32 + key], and maxima m[r * blocks + kb].
template <typename E, int D, int RT>
__device__ __forceinline__ void score_run(const E* K, int64_t ldk, int keys, int blocks, int kb0, int r0, int rows,
                                          const typename Mma<E>::frag (&qf)[RT][D / Mma<E>::KW], float* s, float* m) {
  using M = Mma<E>;
  constexpr int KS = D / M::KW;
  const int lane = lane_id(), half = lane >> 5;
  typename M::frag kf[2][KS];
  auto load = [&](int kb, typename M::frag (&f)[KS]) {
    // (rows past the end repeat the last one; their scores become -inf)
    const E* row = K + (int64_t)min(kb * DEC_KEYS + (lane & 31), keys - 1) * ldk;
#pragma unroll
    for (int kk = 0; kk < KS; ++kk) f[kk] = load_row_frag_global<E, D>(row, 0, 1, kk);
  };
  float top[RT][DEC_RUN];
  load(kb0, kf[0]);
#pragma unroll
  for (int x = 0; x < DEC_RUN; ++x) {
    const int kb = kb0 + x;
#pragma unroll
    for (int t = 0; t < RT; ++t) top[t][x] = -INFINITY;
    if (kb >= blocks) continue;
    if (x + 1 < DEC_RUN && kb + 1 < blocks) load(kb + 1, kf[(x + 1) & 1]);
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      f32x16 v = zero16();
#pragma unroll
      for (int kk = 0; kk < KS; ++kk) v = M::mma(kf[x & 1][kk], qf[t][kk], v);
      if ((kb + 1) * DEC_KEYS > keys) {
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (kb * DEC_KEYS + crow(r) >= keys) v[r] = -INFINITY;
      }
      float mx = v[0];
#pragma unroll
      for (int r = 1; r < 16; ++r) mx = fmaxf(mx, v[r]);
      float lo, hi;
      wave_halves(mx, lo, hi);
      top[t][x] = fmaxf(lo, hi);
      const int row = r0 + 32 * t + (lane & 31);
      if (row < rows) {
        float* out = s + ((int64_t)kb * rows + row) * DEC_KEYS + 4 * half;
#pragma unroll
        for (int r = 0; r < 16; r += 4) *reinterpret_cast<f32x4*>(out + 2 * r) = f32x4{v[r], v[r + 1], v[r + 2], v[r + 3]};
      }
    }
  }
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    const int row = r0 + 32 * t + (lane & 31);
    if (row < rows && half == 0) {
#pragma unroll
      for (int x = 0; x < DEC_RUN; ++x)
        if (kb0 + x < blocks) m[(int64_t)row * blocks + kb0 + x] = top[t][x];
    }
  }
}

__device__ __forceinline__ int blocks_of(int keys) { return (keys + DEC_KEYS - 1) / DEC_KEYS; }
__device__ __forceinline__ int own_length(const DecodeArgs& a, int b) {
  return min(max(((const ci32*)a.lengths)[b], 0), a.capacity);
}

// Workgroups of the prefix first: per key head, row tile and chunk of
// `per_wave` runs a wave; then one wave per request, key head, row tile and run.
template <typename E, int D, int RT>
__global__ __launch_bounds__(SC_NT, 2) void decode_scores_kernel(DecodeArgs a, int row_tiles, int per_wave, int prefix_wgs) {
  using M = Mma<E>;
  constexpr int KS = D / M::KW;
  const int lane = lane_id(), w = wave_id();
  int x = blockIdx.x;
  if (x < prefix_wgs) {
    const int rows = a.requests * a.group;
    // row tiles of the same keys are next to each other in time
    const int chunks = (a.prefix_runs + SC_WAVES * per_wave - 1) / (SC_WAVES * per_wave);
    const int rt = x % row_tiles, chunk = x / row_tiles % chunks, kv = x / row_tiles / chunks;
    const int r0 = rt * 32 * RT, blocks = blocks_of(a.prefix);
    typename M::frag qf[RT][KS];
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      const int r = min(r0 + 32 * t + (lane & 31), rows - 1), b = r / a.group, g = r - b * a.group;
      const E* row = static_cast<const E*>(a.q) + b * a.q_row + (kv * a.group + g) * a.q_head;
#pragma unroll
      for (int kk = 0; kk < KS; ++kk) qf[t][kk] = load_row_frag_global<E, D>(row, 0, 1, kk);
    }
    const E* K = static_cast<const E*>(a.pk) + kv * a.pk_head;
    float* s = a.ps + (int64_t)kv * blocks * rows * DEC_KEYS;
    float* m = a.pm + (int64_t)kv * rows * blocks;
    for (int y = 0; y < per_wave; ++y) {
      const int run = (chunk * per_wave + y) * SC_WAVES + w;
      if (run >= a.prefix_runs) break;
      score_run<E, D, RT>(K, a.pk_row, a.prefix, blocks, run * DEC_RUN, r0, rows, qf, s, m);
    }
    return;
  }
  x = (x - prefix_wgs) * SC_WAVES + w;
  const int tiles = (a.group + 31) / 32;
  const int run = x % a.own_runs, rt = x / a.own_runs % tiles, rest = x / a.own_runs / tiles;
  const int kv = rest % a.kv_heads, b = rest / a.kv_heads;
  if (b >= a.requests) return;
  const int keys = own_length(a, b), blocks = blocks_of(a.capacity);
  if (run * DEC_RUN * DEC_KEYS >= keys) return;
  typename M::frag qf[1][KS];
  const int g = min(rt * 32 + (lane & 31), a.group - 1);
  const E* row = static_cast<const E*>(a.q) + b * a.q_row + (kv * a.group + g) * a.q_head;
#pragma unroll
  for (int kk = 0; kk < KS; ++kk) qf[0][kk] = load_row_frag_global<E, D>(row, 0, 1, kk);
  const int64_t bk = (int64_t)b * a.kv_heads + kv;
  score_run<E, D, 1>(static_cast<const E*>(a.k) + b * a.k_batch + kv * a.k_head, a.k_row, keys, blocks, run * DEC_RUN,
                     rt * 32, a.group, qf, a.os + bk * blocks * a.group * DEC_KEYS, a.om + bk * a.group * blocks);
}

// ------------------------------------------------------------------- solve

constexpr int SO_NT = 256;
constexpr int SO_WAVES = SO_NT / 64;
constexpr int SO_CAP = 2048;     // scores kept in LDS
constexpr int SO_BLOCKS = MAX_SEQLEN / DEC_KEYS + 2;  // block numbers kept in LDS
constexpr int SO_LANE = 8;       // scores per lane that every wave solves on its own

// The wave's and the workgroup's sums and counts.  All threads.
__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) v += __shfl_xor(v, o);
  return v;
}
__device__ __forceinline__ float wave_maxf(float v) {
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) v = fmaxf(v, __shfl_xor(v, o));
  return v;
}

// A row's scores: blocks 0 .. prefix blocks - 1, then its own.
struct RowScores {
  const float *ps, *os, *pm, *om;  // of the row
  int64_t p_step, o_step;          // block to block in the scores
  int p_blocks, blocks;
  __device__ __forceinline__ float top(int b) const { return b < p_blocks ? pm[b] : om[b - p_blocks]; }
  __device__ __forceinline__ const float* block(int b) const {
    return b < p_blocks ? ps + b * p_step : os + (b - p_blocks) * o_step;
  }
};

template <typename E, int D, int GK>
__global__ __launch_bounds__(SO_NT) void decode_solve_kernel(DecodeArgs a) {
  using R = RowGroup<E, D>;
  constexpr int VPL = R::VPL, LPR = R::LPR, NG = SO_NT / LPR;
  __shared__ float kept[SO_CAP];     // scores above the bound, in the order of the keys
  __shared__ int kept_key[SO_CAP];   // 32 block + key in the block
  __shared__ uint16_t chosen[SO_BLOCKS];  // blocks with such a score
  __shared__ float red[3][SO_WAVES];
  __shared__ int cnt[SO_WAVES];
  static_assert(sizeof(kept) >= NG * D * sizeof(float), "the groups' sums fit in place of the scores");
  const int t = threadIdx.x, lane = lane_id(), w = wave_id();
  const int b = blockIdx.x / a.heads, h = blockIdx.x % a.heads, kv = h / a.group, g = h % a.group;
  const int len = own_length(a, b);
  const int p_blocks = blocks_of(a.prefix), own_cap = blocks_of(a.capacity);
  RowScores row;
  row.p_blocks = p_blocks;
  row.blocks = p_blocks + blocks_of(len);
  const int64_t rows = (int64_t)a.requests * a.group, r = (int64_t)b * a.group + g, bk = (int64_t)b * a.kv_heads + kv;
  row.ps = a.ps + ((int64_t)kv * p_blocks * rows + r) * DEC_KEYS;
  row.p_step = rows * DEC_KEYS;
  row.pm = a.pm + ((int64_t)kv * rows + r) * p_blocks;
  row.os = a.os + (bk * own_cap * a.group + g) * DEC_KEYS;
  row.o_step = (int64_t)a.group * DEC_KEYS;
  row.om = a.om + (bk * a.group + g) * own_cap;
  E* const O = static_cast<E*>(a.o) + b * a.o_row + h * a.o_head;
  const float c = a.c, gm = a.gamma;

  // Sums over the workgroup of three values, in all threads.
  auto sum3 = [&](float& x, float& y, float& z) {
    x = wave_sum(x);
    y = wave_sum(y);
    z = wave_sum(z);
    __syncthreads();
    if (lane == 0) {
      red[0][w] = x;
      red[1][w] = y;
      red[2][w] = z;
    }
    __syncthreads();
    x = (red[0][0] + red[0][1]) + (red[0][2] + red[0][3]);
    y = (red[1][0] + red[1][1]) + (red[1][2] + red[1][3]);
    z = (red[2][0] + red[2][1]) + (red[2][2] + red[2][3]);
  };
  // Where the thread's `mine` items go among those of all threads, from
  // `base` on; base grows by all of them.
  auto place = [&](int mine, int& base) {
    int incl = mine;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int v = __shfl_up(incl, o);
      if (lane >= o) incl += v;
    }
    __syncthreads();
    if (lane == 63) cnt[w] = incl;
    __syncthreads();
    int at = base + incl - mine;
#pragma unroll
    for (int x = 0; x < SO_WAVES; ++x) {
      if (x < w) at += cnt[x];
      base += cnt[x];
    }
    return at;
  };

  // ---- the largest score, and the bound from the blocks' maxima
  float m = -INFINITY;
  for (int x = t; x < row.blocks; x += SO_NT) m = fmaxf(m, row.top(x));
  m = wave_maxf(m);
  if (lane == 0) red[0][w] = m;
  __syncthreads();
  m = c * fmaxf(fmaxf(red[0][0], red[0][1]), fmaxf(red[0][2], red[0][3]));
  __syncthreads();
  if (!(m > -INFINITY)) {  // no keys (or none with a finite score): nothing to add up
    for (int x = t; x < D; x += SO_NT) O[x] = (E)0.f;
    return;
  }
  // z^gamma, z^(gamma-1), z^(gamma-2) summed over z > 0
  auto add = [&](float z, float& s0, float& s1, float& s2) {
    if (z > 0.f) {
      float p, u;
      Gamma<GK>::pu(z, gm, p, u);
      s0 += p;
      s1 += u;
      if constexpr (GK == 2) s2 += 1.f;
      if constexpr (GK == 4) s2 += z * z;
      if constexpr (GK == 0) s2 += u / z;
    }
  };
  const bool convex = gm >= 1.f;
  float lo = m - 1.f;
  if (convex) {
    for (int it = 0; it < 8; ++it) {
      float s0 = 0.f, s1 = 0.f, s2 = 0.f;
      for (int x = t; x < row.blocks; x += SO_NT) add(relu_z(c, row.top(x), lo), s0, s1, s2);
      sum3(s0, s1, s2);
      const float step = (s0 - 1.f) / (gm * s1);
      if (!(step > 1e-3f)) break;
      lo += step;
    }
  }
  // less the rounding of the sums (a lower bound serves as well)
  lo -= 4e-6f * fmaxf(1.f, fabsf(lo));

  // ---- the blocks with a score above the bound, and those scores
  int nb = 0;
  for (int x0 = 0; x0 < row.blocks; x0 += SO_NT) {
    const int x = x0 + t;
    const bool take = x < row.blocks && relu_z(c, row.top(min(x, row.blocks - 1)), lo) > 0.f;
    const int at = place(take ? 1 : 0, nb);
    if (take) chosen[at] = (uint16_t)x;
  }
  __syncthreads();
  // Scores of the chosen blocks in turn: eight threads to a block, four
  // scores each.  use(score vector, first key, 0 <= thread's block < nb).
  constexpr int BPS = SO_NT / 8;  // blocks a step
  auto scores_of = [&](int x) { return *reinterpret_cast<const f32x4*>(row.block(chosen[x]) + 4 * (t & 7)); };
  // Keeps the scores of chosen blocks [x0, x1) with z > 0 at `at_tau`, up to
  // SO_CAP of them; returns their number (more: the rest are not kept).
  auto collect = [&](int x0, int x1, float at_tau) {
    int n = 0;
    for (int s0 = x0; s0 < x1; s0 += BPS) {
      const int x = s0 + (t >> 3);
      f32x4 v = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
      if (x < x1) v = scores_of(x);
      int mine = 0;
      bool in[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        in[e] = relu_z(c, v[e], at_tau) > 0.f;
        mine += in[e] ? 1 : 0;
      }
      int at = place(mine, n);
      const int key = x < x1 ? chosen[x] * DEC_KEYS + 4 * (t & 7) : 0;
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (in[e]) {
          if (at < SO_CAP) {
            kept[at] = v[e];
            kept_key[at] = key + e;
          }
          ++at;
        }
    }
    __syncthreads();
    return n;
  };
  const int total = collect(0, nb, lo);
  const bool wide = total > SO_CAP;

  // ---- tau: Algorithm 1's iteration on the kept scores
  float hi = m - powf((float)max(a.prefix + len, 1), 1.f - a.alpha);
  float low = fminf(lo, hi);
  float tau = convex ? low : 0.5f * (low + hi), f_prev = INFINITY;
  const bool alone = total <= 64 * SO_LANE;  // every wave by itself: no barriers
  float x[SO_LANE];
  if (alone) {
#pragma unroll
    for (int e = 0; e < SO_LANE; ++e) x[e] = 64 * e + lane < total ? kept[64 * e + lane] : -INFINITY;
  }
  for (int it = 0;; ++it) {
    float s0 = 0.f, s1 = 0.f, s2 = 0.f;
    if (alone) {
#pragma unroll
      for (int e = 0; e < SO_LANE; ++e) add(relu_z(c, x[e], tau), s0, s1, s2);
      s0 = wave_sum(s0);
      s1 = wave_sum(s1);
      s2 = wave_sum(s2);
    } else if (!wide) {
      for (int y = t; y < total; y += SO_NT) add(relu_z(c, kept[y], tau), s0, s1, s2);
      sum3(s0, s1, s2);
    } else {
      for (int y = t >> 3; y < nb; y += BPS) {
        const f32x4 v = scores_of(y);
#pragma unroll
        for (int e = 0; e < 4; ++e) add(relu_z(c, v[e], tau), s0, s1, s2);
      }
      sum3(s0, s1, s2);
    }
    const float f = s0 - 1.f;
    const bool stop = fabsf(f) <= a.tol || it >= a.max_iter;
    if (stop && !convex) break;  // (the update would leave a root that has been found)
    // B_f, Newton's bound, H_f: the update rules of the attention solver
    const float f1 = -gm * s1, f2 = gm * (gm - 1.f) * s2;
    if (f < 0.f)
      hi = tau;
    else
      low = tau;
    const float slack = 1e-6f * fmaxf(1.f, fmaxf(fabsf(low), fabsf(hi)));
    if (convex && f1 < 0.f) low = fminf(fmaxf(low, tau - f / f1 - 10.f * slack), hi);
    const float th = tau - 2.f * f * f1 / (2.f * f1 * f1 - f * f2);
    bool take = th >= low - slack && th <= hi + slack;
    if (!convex && fabsf(f) > 0.5f * f_prev) take = false;
    f_prev = fabsf(f);
    // (the update from the last evaluation is taken too)
    tau = take ? fminf(fmaxf(th, low), hi) : convex && th < low ? low : 0.5f * (low + hi);
    if (stop) break;
  }

  // ---- O: the rows of V with a probability
  const int sub = lane % LPR, grp = t / LPR;
  float o[VPL] = {};
  const char* const own_v = reinterpret_cast<const char*>(static_cast<const E*>(a.v) + b * a.v_batch + kv * a.v_head);
  const char* const pre_v = reinterpret_cast<const char*>(static_cast<const E*>(a.pv) + kv * a.pv_head);
  auto gather = [&](int n) {
    constexpr int BATCH = 4;
    for (int y0 = grp; y0 < n; y0 += NG * BATCH) {
      u32x4 v[BATCH];
      float p[BATCH];
#pragma unroll
      for (int u = 0; u < BATCH; ++u) {
        const int y = y0 + u * NG;
        p[u] = 0.f;
        v[u] = u32x4{0, 0, 0, 0};
        if (y < n) {
          p[u] = Gamma<GK>::p_only(relu_z(c, kept[y], tau), gm);
          if (p[u] > 0.f) {  // (a key without a probability is not read)
            const int key = kept_key[y], blk = key / DEC_KEYS;
            const char* v_row = blk < p_blocks ? pre_v + key * a.pv_row * (int64_t)sizeof(E)
                                               : own_v + (key - p_blocks * DEC_KEYS) * a.v_row * (int64_t)sizeof(E);
            v[u] = *reinterpret_cast<const u32x4*>(v_row + sub * 16);
          }
        }
      }
#pragma unroll
      for (int u = 0; u < BATCH; ++u) {
        float e[VPL];
        R::unpack(v[u], e);
#pragma unroll
        for (int d = 0; d < VPL; ++d) o[d] = fmaf(p[u], e[d], o[d]);
      }
    }
  };
  if (!wide) {
    gather(total);
  } else {
    constexpr int PART = SO_CAP / DEC_KEYS;  // blocks whose scores all fit
    for (int x0 = 0; x0 < nb; x0 += PART) {
      __syncthreads();
      gather(collect(x0, min(x0 + PART, nb), tau));
    }
  }
  __syncthreads();
  // the groups' sums, in place of the kept scores
#pragma unroll
  for (int d = 0; d < VPL; ++d) kept[grp * D + sub * VPL + d] = o[d];
  __syncthreads();
  for (int d = t; d < D; d += SO_NT) {
    float sum = 0.f;
    for (int x2 = 0; x2 < NG; ++x2) sum += kept[x2 * D + d];
    O[d] = (E)sum;
  }
}

template <typename E, int D, int RT>
hipError_t launch_scores(const DecodeArgs& a, hipStream_t s) {
  const int row_tiles = (a.requests * a.group + 32 * RT - 1) / (32 * RT);
  // runs of a wave: as few as give every wave of the device work (eight waves
  // to each of 256 compute units), so that queries are loaded seldom
  int64_t waves = (int64_t)a.kv_heads * row_tiles * a.prefix_runs;
  int per_wave = (int)(waves / 2048);
  per_wave = per_wave < 1 ? 1 : per_wave > 8 ? 8 : per_wave;
  const int chunks = (a.prefix_runs + SC_WAVES * per_wave - 1) / (SC_WAVES * per_wave);
  const int64_t prefix_wgs = a.prefix ? (int64_t)a.kv_heads * row_tiles * chunks : 0;
  const int64_t own = (int64_t)a.requests * a.kv_heads * ((a.group + 31) / 32) * a.own_runs;
  const int64_t wgs = prefix_wgs + (own + SC_WAVES - 1) / SC_WAVES;
  if (wgs == 0) return hipSuccess;
  if (wgs > INT32_MAX) return hipErrorInvalidConfiguration;
  DecodeArgs args = a;
  int rt = row_tiles, pw = per_wave, pg = (int)prefix_wgs;
  void* params[] = {&args, &rt, &pw, &pg};
  return hipLaunchKernel(reinterpret_cast<const void*>(decode_scores_kernel<E, D, RT>), dim3((unsigned)wgs), dim3(SC_NT),
                         params, 0, s);
}

template <typename E, int D>
hipError_t launch_decode_d(const DecodeArgs& a, hipStream_t s) {
  const int rows = a.requests * a.group;
  hipError_t e;
  if (sizeof(E) == 2 && rows > 64)
    e = launch_scores<E, D, sizeof(E) == 2 ? 4 : 1>(a, s);
  else if (sizeof(E) == 2 && rows > 32)
    e = launch_scores<E, D, sizeof(E) == 2 ? 2 : 1>(a, s);
  else
    e = launch_scores<E, D, 1>(a, s);
  if (e != hipSuccess) return e;
  auto kernel = decode_solve_kernel<E, D, 0>;
  if (a.gk == 1) kernel = decode_solve_kernel<E, D, 1>;
  if (a.gk == 2) kernel = decode_solve_kernel<E, D, 2>;
  if (a.gk == 4) kernel = decode_solve_kernel<E, D, 4>;
  return launch_kernel(kernel, dim3((unsigned)(a.requests * a.heads)), dim3(SO_NT), s, a);
}

}  // namespace

hipError_t launch_decode(const DecodeArgs& a, int dtype, int head_dim, hipStream_t s) {
  if (dtype == 0) return head_dim == 64 ? launch_decode_d<__bf16, 64>(a, s) : launch_decode_d<__bf16, 128>(a, s);
  return head_dim == 64 ? launch_decode_d<float, 64>(a, s) : launch_decode_d<float, 128>(a, s);
}

}  // namespace ea
