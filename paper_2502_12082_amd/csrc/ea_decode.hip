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
// Maxima.  The queries of every request that share a key head form one matrix,
// so a prefix key is read once for all of them; a request's own cache meets
// the queries of its group.  A wave holds up to 64 queries as MFMA B operands in
// registers and streams key blocks of 32 through LDS of its own, whole rows by
// one instruction (read straight into A operands, every lane of a load is in a
// line of its own, and a load takes the address unit 64 cycles: 32 requests,
// 32/8 heads, behind 65536 shared keys, d = 128, 45 us against 37; fp32, 8
// requests behind 32768 keys, the whole call 122 against 78).  Bound by HBM: the
// keys are read once.  The scores themselves are not written (108 us), but the
// largest of every 32 keys, and one byte for every four.
//
// Solve.  One workgroup per query row.  The maxima of its blocks are scores of
// distinct keys, so f restricted to them lies below f, and its root is a
// lower bound of tau (as the bound of the attention solver, over every block):
// only quads of keys whose maximum is above it can have a probability.  Their
// scores are computed again, from K rows that the caches still hold, into LDS,
// tau is solved on them (Algorithm 1's iteration), and the rows of V with a
// probability are gathered, 16 bytes a lane.  Rows with more quads than fit
// compute the scores of whole blocks into memory and read them for every
// evaluation, and gather V part by part.  Every list has an order that depends
// on the scores alone, not on timing.
//
// fp32 inputs with alpha > 2: p = z^gamma, gamma < 1, has no bounded slope at z
// = 0, where an fp32 score off by 1e-6 has p off by 1e-3 (alpha 3).  As in
// attention (ea_common.h), scores within PRECISE_BAND max(1, |tau|) of the edge are
// taken in fp64 there, and tau is finished in fp64; few keys are that near (keys
// put at the edge, alpha 3, queries 20 times as large: O off by 7e-3 without and
// under 5e-5 with; 8 requests, 32/8 heads, 32768 shared keys, alpha 2.5 84 and 94
// us).  For 1 < alpha <= 2 the slope is at most gamma, and fp32 serves.
#include "ea_common.h"
#include "ea_internal.h"

namespace ea {

namespace {

constexpr int SC_NT = 64;
constexpr float QUAD_STEPS = 248.f;             // (255 steps are more than 1, by more than roundings)
constexpr int RUN_BYTES = DEC_RUN * DEC_KEYS / 4;  // of a row's quads in a run

// ------------------------------------------------------------------ maxima

// Key blocks of one wave on their way through LDS, two at once.  (Four of them
// leave room for fewer waves: 57 us against 52 where 64 requests have own caches
// of up to 1024 keys, 55 and 56 where nearly all keys are shared.)
template <typename E, int D>
struct KeyRing {
  using TL = Tile<E, D>;
  static constexpr int BLOCKS = 2;
  static constexpr int ELEMS = DEC_KEYS * D;
  static constexpr int LOADS = DEC_KEYS * TL::CPR / 64;  // wave instructions per block
  static_assert(DEC_RUN % BLOCKS == 0 && (BLOCKS - 1) * LOADS < 64, "a block's place and its wait are constants");
  E* at;
  int ld;                // keys' rows apart, at most 2^24
  uint32_t off[LOADS];  // bytes from the block's first row to the lane's chunks

  __device__ __forceinline__ KeyRing(E* lds, int64_t row_stride) : at(lds), ld((int)row_stride) {
#pragma unroll
    for (int i = 0; i < LOADS; ++i) off[i] = TL::src_off(64 * i + lane_id(), ld) * (uint32_t)sizeof(E);
  }
  // Copies block kb of `keys` rows to place x (rows past the end become 0; their
  // scores are set to -inf).
  __device__ __forceinline__ void copy(const E* K, int keys, int kb, int x) const {
#if defined(__HIP_DEVICE_COMPILE__)
    // (a buffer of the rows that there are)
    kb = __builtin_amdgcn_readfirstlane(kb);
    const int rows = __builtin_amdgcn_readfirstlane(min(keys - kb * DEC_KEYS, DEC_KEYS));
    const auto rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<E*>(K + (int64_t)kb * DEC_KEYS * ld), (short)0,
                                                        ((rows - 1) * ld + D) * (int)sizeof(E), 0x00027000);
    E* const to = at + x * ELEMS;
#pragma unroll
    for (int i = 0; i < LOADS; ++i)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, to_lds(to + 64 * i * TL::VEC), 16, off[i], 0, 0, 0);
#endif
  }
  // Waits until all copies but the latest BLOCKS - 1 (`full`: there are as many) have landed.
  // (Loads complete in the order of their issue; stores among them only make
  // the wait longer.)
  __device__ __forceinline__ static void wait(bool full) {
    constexpr int N = (BLOCKS - 1) * LOADS;
    if (full)
      __builtin_amdgcn_s_waitcnt(0x0F70 | (N & 15) | (N >> 4) << 14);
    else
      dma_wait();
    asm volatile("" ::: "memory");
  }
};

// Maxima of `runs` runs of DEC_RUN key blocks from run `run0` on (`keys` keys in
// all) against the wave's 32 RT rows from r0 on (`rows` in all): of blocks,
// m[r * wide + kb]; and of the quads of four keys, by how much c times each is
// below the block's, in steps of 1 / QUAD_STEPS and rounded down, one byte
// each: qm[(run * rows + r) * RUN_BYTES ..], a wave's in one piece of 2 KB.  A
// quad 255 steps lower is below the largest score less 1, where no key has a
// probability.
template <typename E, int D, int RT>
__device__ __forceinline__ void maxima_runs(const E* K, int keys, int wide, int run0, int runs, int r0,
                                            int rows, float c, const typename Mma<E>::frag (&qf)[RT][D / Mma<E>::KW],
                                            const KeyRing<E, D>& ring, uint8_t* qm, float* m) {
  using M = Mma<E>;
  using R = KeyRing<E, D>;
  constexpr int KS = D / M::KW;
  const int lane = lane_id(), half = lane >> 5;
  const float steps = c * QUAD_STEPS;
  const int first = run0 * DEC_RUN, last = min(first + runs * DEC_RUN, (keys + DEC_KEYS - 1) / DEC_KEYS);
#pragma unroll
  for (int x = 0; x < R::BLOCKS; ++x)
    if (first + x < last) ring.copy(K, keys, first + x, x);
  for (int kb0 = first; kb0 < last; kb0 += DEC_RUN) {
    f32x4 top[RT];
    u32x4 below[RT];
#pragma unroll
    for (int x = 0; x < DEC_RUN; ++x) {
      const int kb = kb0 + x;
#pragma unroll
      for (int t = 0; t < RT; ++t) {
        top[t][x] = -INFINITY;
        below[t][x] = ~0u;
      }
      if (kb >= last) continue;
      R::wait(kb + R::BLOCKS <= last);
      typename M::frag kf[KS];
#pragma unroll
      for (int kk = 0; kk < KS; ++kk) kf[kk] = lds_row_frag<E, D>(ring.at + x % R::BLOCKS * R::ELEMS, lane & 31, kk);
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // (the place is free)
      if (kb + R::BLOCKS < last) ring.copy(K, keys, kb + R::BLOCKS, x % R::BLOCKS);
#pragma unroll
      for (int t = 0; t < RT; ++t) {
        f32x16 v = zero16();
#pragma unroll
        for (int kk = 0; kk < KS; ++kk) v = M::mma(kf[kk], qf[t][kk], v);
        if ((kb + 1) * DEC_KEYS > keys) {
#pragma unroll
          for (int r = 0; r < 16; ++r)
            if (kb * DEC_KEYS + crow(r) >= keys) v[r] = -INFINITY;
        }
        // (the lane's scores 4 i .. 4 i + 3 are keys 8 i + 4 half ..: quad 2 i + half, byte 4 x + i of its half)
        f32x4 gm;
#pragma unroll
        for (int i = 0; i < 4; ++i) gm[i] = fmaxf(fmaxf(v[4 * i], v[4 * i + 1]), fmaxf(v[4 * i + 2], v[4 * i + 3]));
        float lo, hi;
        wave_halves(fmaxf(fmaxf(gm[0], gm[1]), fmaxf(gm[2], gm[3])), lo, hi);
        top[t][x] = fmaxf(lo, hi);
        uint32_t bytes = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) bytes |= (uint32_t)fminf((top[t][x] - gm[i]) * steps, 255.f) << (8 * i);
        below[t][x] = bytes;
      }
    }
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      const int row = r0 + 32 * t + (lane & 31);
      if (row < rows) {
        *reinterpret_cast<u32x4*>(qm + ((int64_t)(kb0 / DEC_RUN) * rows + row) * RUN_BYTES + 16 * half) = below[t];
        if (half == 0) *reinterpret_cast<f32x4*>(m + (int64_t)row * wide + kb0) = top[t];
      }
    }
  }
}
// Quad of a block whose byte is number i of its eight (four to each half).
__device__ __forceinline__ int quad_at(int i) { return 2 * (i & 3) + (i >> 2); }

__device__ __forceinline__ int blocks_of(int keys) { return (keys + DEC_KEYS - 1) / DEC_KEYS; }
__device__ __forceinline__ int own_length(const DecodeArgs& a, int b) {
  return min(max(((const ci32*)a.lengths)[b], 0), a.capacity);
}

// Workgroups of the prefix first: per chunk of `per_wave` runs a wave, row tile
// and key head; then one wave per request, key head, row tile and run.
template <typename E, int D, int RT>
__global__ __launch_bounds__(SC_NT, 2) void decode_maxima_kernel(DecodeArgs a, int row_tiles, int per_wave, int prefix_wgs) {
  using M = Mma<E>;
  constexpr int KS = D / M::KW;
  __shared__ __attribute__((aligned(16))) E keys_lds[KeyRing<E, D>::BLOCKS * KeyRing<E, D>::ELEMS];
  const int lane = lane_id();
  int x = blockIdx.x;
  if (x < prefix_wgs) {
    const int rows = a.requests * a.group;
    // Row tiles of the same keys are next to each other in time, and with eight
    // key heads on one XCD.
    const int kv = x % a.kv_heads, rt = x / a.kv_heads % row_tiles, chunk = x / a.kv_heads / row_tiles;
    const int r0 = rt * 32 * RT;
    typename M::frag qf[RT][KS];
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      const int r = min(r0 + 32 * t + (lane & 31), rows - 1), b = r / a.group, g = r - b * a.group;
      const E* row = static_cast<const E*>(a.q) + b * a.q_row + (kv * a.group + g) * a.q_head;
#pragma unroll
      for (int kk = 0; kk < KS; ++kk) qf[t][kk] = load_row_frag_global<E, D>(row, 0, 1, kk);
    }
    const E* K = static_cast<const E*>(a.pk) + kv * a.pk_head;
    const int wide = a.prefix_runs * DEC_RUN;
    uint8_t* qm = a.pq + (int64_t)kv * a.prefix_runs * rows * RUN_BYTES;
    float* m = a.pm + (int64_t)kv * rows * wide;
    maxima_runs<E, D, RT>(K, a.prefix, wide, chunk * per_wave, min(per_wave, a.prefix_runs - chunk * per_wave),
                          r0, rows, a.c, qf, KeyRing<E, D>(keys_lds, a.pk_row), qm, m);
    return;
  }
  x -= prefix_wgs;
  const int tiles = (a.group + 31) / 32;
  const int run = x % a.own_runs, rt = x / a.own_runs % tiles, rest = x / a.own_runs / tiles;
  const int kv = rest % a.kv_heads, b = rest / a.kv_heads;
  if (b >= a.requests) return;
  const int keys = own_length(a, b);
  if (run * DEC_RUN * DEC_KEYS >= keys) return;
  typename M::frag qf[1][KS];
  const int g = min(rt * 32 + (lane & 31), a.group - 1);
  const E* row = static_cast<const E*>(a.q) + b * a.q_row + (kv * a.group + g) * a.q_head;
#pragma unroll
  for (int kk = 0; kk < KS; ++kk) qf[0][kk] = load_row_frag_global<E, D>(row, 0, 1, kk);
  const int64_t bk = (int64_t)b * a.kv_heads + kv;
  maxima_runs<E, D, 1>(static_cast<const E*>(a.k) + b * a.k_batch + kv * a.k_head, keys, a.own_runs * DEC_RUN,
                       run, 1, rt * 32, a.group, a.c, qf, KeyRing<E, D>(keys_lds, a.k_row), a.oq + bk * a.own_runs * a.group * RUN_BYTES,
                       a.om + bk * a.group * a.own_runs * DEC_RUN);
}

// ------------------------------------------------------------------- solve

constexpr int SO_LONGEST = MAX_SEQLEN / DEC_KEYS + 2;  // most blocks of a row
constexpr int SO_SHORT = 512;    // and of one that a single wave takes
constexpr int SO_LANE = 8;       // scores per lane that a wave solves on its own
constexpr int SO_STEPS = 4;      // blocks that eight threads read at once
constexpr int SO_MAXIMA = 16;    // blocks' maxima that a thread holds in registers

// Sum, and maximum, over the wave, in all lanes (lanes exchange inside quads,
// mirrored inside 8 and 16 lanes, then rows and halves by swaps: no LDS).
template <typename F>
__device__ __forceinline__ float wave_fold(float v, F&& f) {
#if defined(__HIP_DEVICE_COMPILE__)
  auto dpp = [](float x, auto ctrl) {
    return __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(x), decltype(ctrl)::value, 0xf,
                                                                0xf, true));
  };
  v = f(v, dpp(v, std::integral_constant<int, 0xB1>{}));   // quad_perm 1, 0, 3, 2
  v = f(v, dpp(v, std::integral_constant<int, 0x4E>{}));   // quad_perm 2, 3, 0, 1
  v = f(v, dpp(v, std::integral_constant<int, 0x141>{}));  // row_half_mirror
  v = f(v, dpp(v, std::integral_constant<int, 0x140>{}));  // row_mirror
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = f(__uint_as_float(r[0]), __uint_as_float(r[1]));
#endif
  float lo, hi;
  wave_halves(v, lo, hi);
  return f(lo, hi);
}
__device__ __forceinline__ float wave_sum(float v) {
  return wave_fold(v, [](float a, float b) { return a + b; });
}
__device__ __forceinline__ float wave_maxf(float v) {
  return wave_fold(v, [](float a, float b) { return fmaxf(a, b); });
}

// A row's blocks: 0 .. prefix blocks - 1, then its own.
struct RowBlocks {
  const float *pm, *om;  // of the row
  const uint8_t *pq, *oq;
  int64_t p_step, o_step;  // run to run in the quads' bytes
  int p_blocks, blocks;
  __device__ __forceinline__ float top(int b) const { return b < p_blocks ? pm[b] : om[b - p_blocks]; }
  // An upper bound of c times the maximum of quad i of block b.
  __device__ __forceinline__ float quad(float c, int b, int i) const {
    const bool shared = b < p_blocks;
    const int x = shared ? b : b - p_blocks;
    const uint8_t* const run = shared ? pq + x / DEC_RUN * p_step : oq + x / DEC_RUN * o_step;
    return c * top(b) - (float)run[16 * (i >> 2) + x % DEC_RUN * 4 + (i & 3)] * (1.f / QUAD_STEPS);
  }
};

// NT = 64: one wave per row, which waits for no other and repeats no other's
// arithmetic.  NT = 256: four, for few or long rows (see launch_decode_d).
template <typename E, int D, int GK, int NT>
__global__ __launch_bounds__(NT) void decode_solve_kernel(DecodeArgs a) {
  using R = RowGroup<E, D>;
  constexpr int VPL = R::VPL, LPR = R::LPR, NG = NT / LPR, SO_NT = NT, SO_WAVES = NT / 64;
  constexpr int SO_CAP = NT == 64 ? 1024 : 2048;  // scores kept in LDS
  constexpr int SO_QUADS = SO_CAP / 4;
  constexpr int SO_BLOCKS = NT == 64 ? SO_SHORT : SO_LONGEST;
  __shared__ float kept[SO_CAP];          // scores of the quads, four each
  __shared__ uint16_t quad[SO_QUADS];     // quads with a score above the bound (the block's first key / 4 + quad)
  __shared__ uint16_t chosen[SO_BLOCKS];  // blocks with such a score
  __shared__ float red[2][3][SO_WAVES];
  __shared__ int cnt[2][SO_WAVES];
  static_assert(sizeof(kept) >= NG * D * sizeof(float), "the groups' sums fit in place of the scores");
  static_assert(SO_LONGEST * (DEC_KEYS / 4) <= 65536, "a quad's number fits 16 bits");
  const int t = threadIdx.x, lane = lane_id(), w = wave_id(), sub = lane % LPR, grp = t / LPR;
  // (heads of one key head are kv_heads apart: with eight key heads they meet on
  // one XCD, whose L2 then has to hold the rows of that head alone)
  const int b = blockIdx.x / a.heads, y = blockIdx.x % a.heads, kv = y % a.kv_heads, g = y / a.kv_heads;
  const int h = kv * a.group + g;
  const int len = own_length(a, b);
  const int p_blocks = blocks_of(a.prefix), own_cap = blocks_of(a.capacity);
  const int p_wide = a.prefix_runs * DEC_RUN, o_wide = a.own_runs * DEC_RUN;
  RowBlocks row;
  row.p_blocks = p_blocks;
  row.blocks = p_blocks + blocks_of(len);
  const int64_t rows = (int64_t)a.requests * a.group, r = (int64_t)b * a.group + g, bk = (int64_t)b * a.kv_heads + kv;
  row.pm = a.pm + ((int64_t)kv * rows + r) * p_wide;
  row.pq = a.pq + ((int64_t)kv * a.prefix_runs * rows + r) * RUN_BYTES;
  row.p_step = rows * RUN_BYTES;
  row.om = a.om + (bk * a.group + g) * o_wide;
  row.oq = a.oq + (bk * a.own_runs * a.group + g) * RUN_BYTES;
  row.o_step = (int64_t)a.group * RUN_BYTES;
  E* const O = static_cast<E*>(a.o) + b * a.o_row + h * a.o_head;
  const float c = a.c, gm = a.gamma;

  // Sums over the workgroup of three values, in all threads (two buffers in
  // turn: one barrier).
  int turn = 0;
  auto sum3 = [&](float& x, float& y, float& z) {
    x = wave_sum(x);
    y = wave_sum(y);
    z = wave_sum(z);
    if constexpr (SO_WAVES == 1) return;
    auto& m = red[turn];
    turn ^= 1;
    if (lane == 0) {
      m[0][w] = x;
      m[1][w] = y;
      m[2][w] = z;
    }
    __syncthreads();
    x = y = z = 0.f;
#pragma unroll
    for (int i = 0; i < SO_WAVES; ++i) {
      x += m[0][i];
      y += m[1][i];
      z += m[2][i];
    }
  };
  // The largest of a wave-uniform value over the workgroup.
  auto max_waves = [&](float x) {
    if constexpr (SO_WAVES > 1) {
      auto& m = red[turn];
      turn ^= 1;
      if (lane == 0) m[0][w] = x;
      __syncthreads();
#pragma unroll
      for (int i = 0; i < SO_WAVES; ++i) x = fmaxf(x, m[0][i]);
    }
    return x;
  };
  // Where the thread's `mine` items go among those of all threads, from
  // `base` on; base grows by all of them.
  int cturn = 0;
  auto place = [&](int mine, int& base) {
    int incl = mine;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int v = __shfl_up(incl, o);
      if (lane >= o) incl += v;
    }
    if constexpr (SO_WAVES == 1) {
      const int at = base + incl - mine;
      base += __builtin_amdgcn_readlane(incl, 63);
      return at;
    }
    auto& m = cnt[cturn];
    cturn ^= 1;
    if (lane == 63) m[w] = incl;
    __syncthreads();
    int at = base + incl - mine;
#pragma unroll
    for (int x = 0; x < SO_WAVES; ++x) {
      if (x < w) at += m[x];
      base += m[x];
    }
    return at;
  };

  // ---- the maxima of the row's blocks, and the largest score
  float top[SO_MAXIMA], m = -INFINITY;
#pragma unroll
  for (int j = 0; j < SO_MAXIMA; ++j) {
    top[j] = -INFINITY;
    if (j * NT >= row.blocks) break;
    if (j * NT + t < row.blocks) top[j] = row.top(j * NT + t);
  }
  // use(maximum, block) of the thread's blocks; those of longer rows are read again
  auto each_top = [&](auto&& use) {
#pragma unroll
    for (int j = 0; j < SO_MAXIMA; ++j) {
      if (j * NT >= row.blocks) break;
      use(top[j], j * NT + t);
    }
#pragma unroll 4
    for (int x = SO_MAXIMA * NT + t; x < row.blocks; x += NT) use(row.top(x), x);
  };
  each_top([&](float v, int) { m = fmaxf(m, v); });
  m = c * max_waves(wave_maxf(m));
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
  // The bound: Newton's steps on f restricted to the maxima, from max x - 1,
  // stay below its root where f is convex.  First each wave takes its own
  // maxima alone (a bound as well), without waiting for the others; then a
  // step on all of them from the best of those.
  const bool convex = gm >= 1.f;
  float lo = m - 1.f;
  if (convex) {
    auto sums = [&](float& s0, float& s1) {
      float s2 = 0.f;
      each_top([&](float v, int) { add(relu_z(c, v, lo), s0, s1, s2); });
    };
    for (int it = 0; it < 8; ++it) {
      float s0 = 0.f, s1 = 0.f;
      sums(s0, s1);
      s0 = wave_sum(s0);
      s1 = wave_sum(s1);
      const float step = (s0 - 1.f) * __builtin_amdgcn_rcpf(gm * s1);
      if (!(step > 1e-2f)) break;
      lo += step;
    }
    if constexpr (SO_WAVES > 1) {
      lo = max_waves(lo);
      float s0 = 0.f, s1 = 0.f, s2 = 0.f;
      sums(s0, s1);
      sum3(s0, s1, s2);
      const float step = (s0 - 1.f) * __builtin_amdgcn_rcpf(gm * s1);
      if (step > 0.f) lo += step;
    }
  }
  // less the rounding of the sums (a lower bound serves as well)
  lo -= 4e-6f * fmaxf(1.f, fabsf(lo));

  // ---- the blocks with a score above the bound, and those scores
  int nb = 0, mine = 0;
  each_top([&](float v, int) { mine += relu_z(c, v, lo) > 0.f ? 1 : 0; });
  int to = place(mine, nb);
  each_top([&](float v, int x) {
    if (relu_z(c, v, lo) > 0.f) chosen[to++] = (uint16_t)x;
  });
  __syncthreads();
  // ---- the quads with a score above the bound: eight threads to a block
  constexpr int BPS = SO_NT / 8;  // blocks a step
  int nq = 0;
  for (int s0 = 0; s0 < nb; s0 += BPS * SO_STEPS) {
    float q[SO_STEPS];
#pragma unroll
    for (int u = 0; u < SO_STEPS; ++u) {
      const int x = s0 + u * BPS + (t >> 3);
      q[u] = x < nb ? row.quad(c, chosen[x], t & 7) : -INFINITY;
    }
    int mine = 0;
#pragma unroll
    for (int u = 0; u < SO_STEPS; ++u) mine += q[u] > lo ? 1 : 0;
    int at = place(mine, nq);
#pragma unroll
    for (int u = 0; u < SO_STEPS; ++u)
      if (q[u] > lo) {
        if (at < SO_QUADS) quad[at] = (uint16_t)(chosen[s0 + u * BPS + (t >> 3)] * (DEC_KEYS / 4) + quad_at(t & 7));
        ++at;
      }
  }
  __syncthreads();
  const bool wide = nq > SO_QUADS;

  // ---- their scores: a group of lanes per key row
  const E* const own_k = static_cast<const E*>(a.k) + b * a.k_batch + kv * a.k_head;
  const E* const pre_k = static_cast<const E*>(a.pk) + kv * a.pk_head;
  float qv[VPL];
  R::unpack(R::load(static_cast<const E*>(a.q) + b * a.q_row + h * a.q_head, 0u), qv);
  // store(i, scores) of the quads number(i), i < n (four keys each, from key 4
  // number(i) on, counted over all blocks), by the first lane of a group; QB at a time.
  constexpr int QB = NT == 64 ? 4 : 2;
  auto quad_scores = [&](int n, auto&& number, auto&& store) {
    for (int x0 = grp; x0 < n; x0 += QB * NG) {
      u32x4 kw[QB][4];
      int left[QB];  // keys from the quad's first to the end
#pragma unroll
      for (int u = 0; u < QB; ++u) {
        const int q = number(min(x0 + u * NG, n - 1));
        const bool shared = q < p_blocks * (DEC_KEYS / 4);
        const int k0 = 4 * q - (shared ? 0 : p_blocks * DEC_KEYS);
        left[u] = (shared ? a.prefix : len) - k0;
        const E* const base = (shared ? pre_k : own_k) + sub * VPL;
        const int64_t ld = shared ? a.pk_row : a.k_row;
#pragma unroll
        for (int e = 0; e < 4; ++e)
          kw[u][e] = *reinterpret_cast<const u32x4*>(base + (k0 + min(e, left[u] - 1)) * ld);
      }
#pragma unroll
      for (int u = 0; u < QB; ++u) {
        f32x4 s;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          float x2[VPL], dot = 0.f;
          R::unpack(kw[u][e], x2);
#pragma unroll
          for (int d = 0; d < VPL; ++d) dot = fmaf(qv[d], x2[d], dot);
          dot = R::sum(dot);
          s[e] = e < left[u] ? dot : -INFINITY;
        }
        if (sub == 0 && x0 + u * NG < n) store(x0 + u * NG, s);
      }
    }
  };
  float* const spill = a.spill + ((int64_t)b * a.heads + h) * (int64_t)(p_blocks + own_cap) * DEC_KEYS;
  if (!wide)
    quad_scores(nq, [&](int i) { return (int)quad[i]; },
                [&](int i, const f32x4& s) { *reinterpret_cast<f32x4*>(kept + 4 * i) = s; });
  else
    quad_scores(nb * (DEC_KEYS / 4),
                [&](int i) { return chosen[i / (DEC_KEYS / 4)] * (DEC_KEYS / 4) + i % (DEC_KEYS / 4); },
                [&](int i, const f32x4& s) {
                  *reinterpret_cast<f32x4*>(spill + (int64_t)chosen[i / (DEC_KEYS / 4)] * DEC_KEYS +
                                            4 * (i % (DEC_KEYS / 4))) = s;
                });
  __syncthreads();
  const int total = 4 * nq;
  // scores of chosen block x, four to each of eight threads (wide rows)
  auto scores_of = [&](int x) {
    return *reinterpret_cast<const f32x4*>(spill + (int64_t)chosen[x] * DEC_KEYS + 4 * (t & 7));
  };

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
      for (int e = 0; e < SO_LANE; ++e) {
        if (64 * e >= total) break;
        add(relu_z(c, x[e], tau), s0, s1, s2);
      }
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

  // ---- fp32 inputs, alpha > 2: tau in fp64 (see the top of this file)
  [[maybe_unused]] double t64 = tau;
  [[maybe_unused]] const float band = PRECISE_BAND * fmaxf(1.f, fabsf(tau));
  const bool precise = precise_path<E, GK>() && !convex;
  // z of a kept score (-inf or NaN: none), -1 for one below the band
  [[maybe_unused]] auto z64 = [&](float score, int key) -> double {
    const float raw = fmaf(c, score, -tau);
    if (!(raw > -band)) return -1.0;
    if (raw >= band) return a.c64 * (double)score - t64;
    const E* const k_row = key < p_blocks * DEC_KEYS ? pre_k + key * a.pk_row : own_k + (key - p_blocks * DEC_KEYS) * a.k_row;
    const E* const q_row = static_cast<const E*>(a.q) + b * a.q_row + h * a.q_head;
    return exact_x<D>(reinterpret_cast<const float*>(q_row), reinterpret_cast<const float*>(k_row), a.c64) - t64;
  };
  [[maybe_unused]] auto z_of = [&](float score, int key) { return (float)fmin(fmax(z64(score, key), 0.0), 1.0); };
  if constexpr (precise_path<E, GK>()) {
    if (precise) {
      __shared__ double red64[2][2][SO_WAVES];
      const float wider = 1e-5f * fmaxf(1.f, fmaxf(fabsf(low), fabsf(hi)));
      double below = (double)low - wider, above = (double)hi + wider, f_last = INFINITY;
      // Newton's steps inside a bracket, its middle where they leave it or do
      // not halve |f| (f has a kink at every score); the ends meet after 40
      for (int it = 0; it < 40; ++it) {
        double s0 = 0.0, s1 = 0.0;
        auto add64 = [&](double z) {
          if (z > 0.0) {
            const double u = pow(z, a.g64 - 1.0);
            s0 = fma(u, z, s0);
            s1 += u;
          }
        };
        if (!wide) {
          for (int y = t; y < total; y += SO_NT) add64(z64(kept[y], 4 * quad[y >> 2] + (y & 3)));
        } else {
          for (int y = t >> 3; y < nb; y += BPS) {
            const f32x4 v = scores_of(y);
#pragma unroll
            for (int e = 0; e < 4; ++e) add64(z64(v[e], chosen[y] * DEC_KEYS + 4 * (t & 7) + e));
          }
        }
#pragma unroll
        for (int x2 = 32; x2 >= 1; x2 >>= 1) {
          s0 += __shfl_xor(s0, x2);
          s1 += __shfl_xor(s1, x2);
        }
        auto& m64 = red64[it & 1];
        if (lane == 0) {
          m64[0][w] = s0;
          m64[1][w] = s1;
        }
        __syncthreads();
        s0 = s1 = 0.0;
#pragma unroll
        for (int x2 = 0; x2 < SO_WAVES; ++x2) {
          s0 += m64[0][x2];
          s1 += m64[1][x2];
        }
        const double f = s0 - 1.0;
        if (fabs(f) <= 1e-9) break;
        if (f < 0.0)
          above = t64;
        else
          below = t64;
        const double tn = t64 + f / (a.g64 * s1);
        t64 = tn > below && tn < above && fabs(f) <= 0.5 * f_last ? tn : 0.5 * (below + above);
        f_last = fabs(f);
      }
    }
  }

  // ---- O: the rows of V with a probability
  float o[VPL] = {};
  const E* const own_v = static_cast<const E*>(a.v) + b * a.v_batch + kv * a.v_head;
  const E* const pre_v = static_cast<const E*>(a.pv) + kv * a.pv_head;
  // Of n kept scores (or, if precise, z), those at 4 i of the keys from 4 first(i) on: those with a
  // probability move to the front (a score is not overwritten before every
  // thread has read its own), p in place of the score, and their rows of V are
  // added up.
  __shared__ uint16_t from[SO_CAP];
  auto gather = [&](int n, auto&& first) {
    int np = 0;
    for (int y0 = 0; y0 < n; y0 += NT) {
      const float z = y0 + t < n ? (precise ? kept[y0 + t] : relu_z(c, kept[y0 + t], tau)) : 0.f;
      const float p = Gamma<GK>::p_only(z, gm);
      const int at = place(p > 0.f ? 1 : 0, np);
      if (p > 0.f) {
        kept[at] = p;
        from[at] = (uint16_t)(y0 + t);
      }
    }
    __syncthreads();
    constexpr int BATCH = 8;
    for (int y0 = grp; y0 < np; y0 += NG * BATCH) {
      u32x4 v[BATCH];
      float p[BATCH];
#pragma unroll
      for (int u = 0; u < BATCH; ++u) {
        const int y = min(y0 + u * NG, np - 1), i = from[y];
        p[u] = y0 + u * NG < np ? kept[y] : 0.f;
        const int key = 4 * first(i >> 2) + (i & 3);
        const E* const v_row = key < p_blocks * DEC_KEYS ? pre_v + key * a.pv_row
                                                         : own_v + (key - p_blocks * DEC_KEYS) * a.v_row;
        v[u] = *reinterpret_cast<const u32x4*>(v_row + sub * VPL);
      }
#pragma unroll
      for (int u = 0; u < BATCH; ++u) {
        if (y0 + u * NG >= np) break;  // (the last row again, whatever it holds)
        float e[VPL];
        R::unpack(v[u], e);
#pragma unroll
        for (int d = 0; d < VPL; ++d) o[d] = fmaf(p[u], e[d], o[d]);
      }
    }
  };
  if (!wide) {
    if constexpr (precise_path<E, GK>())
      if (precise)
        for (int y = t; y < total; y += SO_NT) kept[y] = z_of(kept[y], 4 * quad[y >> 2] + (y & 3));
    gather(total, [&](int i) { return (int)quad[i]; });
  } else {
    constexpr int PART = SO_CAP / DEC_KEYS;  // blocks whose scores fit
    for (int x0 = 0; x0 < nb; x0 += PART) {
      const int x1 = min(x0 + PART, nb);
      __syncthreads();
      for (int x = x0 + (t >> 3); x < x1; x += BPS) {
        f32x4 v = scores_of(x);
        if constexpr (precise_path<E, GK>())
          if (precise)
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = z_of(v[e], chosen[x] * DEC_KEYS + 4 * (t & 7) + e);
        *reinterpret_cast<f32x4*>(kept + (x - x0) * DEC_KEYS + 4 * (t & 7)) = v;
      }
      __syncthreads();
      gather((x1 - x0) * DEC_KEYS, [&](int i) { return chosen[x0 + i / (DEC_KEYS / 4)] * (DEC_KEYS / 4) + i % (DEC_KEYS / 4); });
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

// Rows of 32 that a wave of the prefix holds.  (64 rows to a wave, with registers
// for two waves more than with 128: 49 us against 45 for 640 rows, 16 requests of
// 40/1 heads behind 65536 keys.)
int row_tile(bool f32, int rows) { return !f32 && rows > 32 ? 2 : 1; }

struct MaximaGrid {
  int row_tiles, per_wave;
  int64_t prefix_wgs, wgs;
};
MaximaGrid maxima_grid(const DecodeArgs& a, bool f32) {
  const int rows = a.requests * a.group, tile = 32 * row_tile(f32, rows);
  MaximaGrid g;
  g.row_tiles = (int)(((int64_t)rows + tile - 1) / tile);
  // runs of a wave: as few as give every wave of the device work (eight waves
  // to each of 256 compute units), so that queries are loaded seldom
  const int64_t each = (int64_t)a.kv_heads * g.row_tiles * a.prefix_runs / 2048;
  g.per_wave = each < 1 ? 1 : each > 8 ? 8 : (int)each;
  const int chunks = (a.prefix_runs + g.per_wave - 1) / g.per_wave;
  g.prefix_wgs = (int64_t)a.kv_heads * g.row_tiles * chunks;
  g.wgs = g.prefix_wgs + (int64_t)a.requests * a.kv_heads * ((a.group + 31) / 32) * a.own_runs;
  return g;
}

template <typename E, int D, int RT>
hipError_t launch_maxima(const DecodeArgs& a, hipStream_t s) {
  MaximaGrid g = maxima_grid(a, sizeof(E) == 4);
  if (g.wgs == 0) return hipSuccess;
  DecodeArgs args = a;
  int pg = (int)g.prefix_wgs;
  void* params[] = {&args, &g.row_tiles, &g.per_wave, &pg};
  return hipLaunchKernel(reinterpret_cast<const void*>(decode_maxima_kernel<E, D, RT>), dim3((unsigned)g.wgs),
                         dim3(SC_NT), params, 0, s);
}

template <typename E, int D, int NT>
hipError_t launch_solve(const DecodeArgs& a, hipStream_t s) {
  auto kernel = decode_solve_kernel<E, D, 0, NT>;
  if (a.gk == 1) kernel = decode_solve_kernel<E, D, 1, NT>;
  if (a.gk == 2) kernel = decode_solve_kernel<E, D, 2, NT>;
  if (a.gk == 4) kernel = decode_solve_kernel<E, D, 4, NT>;
  return launch_kernel(kernel, dim3((unsigned)(a.requests * a.heads)), dim3(NT), s, a);
}

template <typename E, int D>
hipError_t launch_decode_d(const DecodeArgs& a, hipStream_t s) {
  hipError_t e;
  if (row_tile(sizeof(E) == 4, a.requests * a.group) == 2)
    e = launch_maxima<E, D, sizeof(E) == 2 ? 2 : 1>(a, s);
  else
    e = launch_maxima<E, D, 1>(a, s);
  if (e != hipSuccess) return e;
  // Rows for two waves on every compute unit have one each, few or long ones
  // four.  A call in a graph, us, one wave against four, rows of 16 blocks (no
  // prefix), 136 and 480 (16/4 heads, d = 128): c = 1, 256 rows 18, 22, 28 against
  // 16, 17, 22; 512 20, 25, 34 against 19, 20, 28; 1024 24, 27, 43 against 25, 26,
  // 40; 2048 33, 32, 61 against 42, 41, 69.  c = 4, where fewer quads are left:
  // 256 17, 19, 23 against 19, 19, 22; 512 19, 19, 29 against 20, 21, 29; 1024 22,
  // 21, 36 against 26, 26, 39.  Longer: solve alone, 1024 rows of 2050 blocks 33
  // against 23.
  const bool one = a.requests * a.heads >= 512 && a.prefix_runs + a.own_runs <= SO_SHORT / DEC_RUN;
  return one ? launch_solve<E, D, 64>(a, s) : launch_solve<E, D, 256>(a, s);
}

}  // namespace

int64_t decode_maxima_wgs(const DecodeArgs& a, int dtype) { return maxima_grid(a, dtype != 0).wgs; }

hipError_t launch_decode(const DecodeArgs& a, int dtype, int head_dim, hipStream_t s) {
  if (dtype == 0) return head_dim == 64 ? launch_decode_d<__bf16, 64>(a, s) : launch_decode_d<__bf16, 128>(a, s);
  return head_dim == 64 ? launch_decode_d<float, 64>(a, s) : launch_decode_d<float, 128>(a, s);
}

}  // namespace ea
