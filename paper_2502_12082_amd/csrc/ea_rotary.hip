// ea_rotary.hip -- RMS norm of every query and key head and the rotation by
// the token's position, in one pass, and its backward.
//
// Forward, for one row x of D values (one head of one token):
//   r = (mean x^2 + eps)^(-1/2),  y = r x w
//   pair i of rot / 2:  phi = pos[axis of i] f_i
//   (a, b) -> (a cos phi - b sin phi, a sin phi + b cos phi)
// for (a, b) = (y_i, y_{i + rot/2}), or (y_2i, y_2i+1) interleaved; the other
// D - rot values stay y.  Backward, with dz the gradient of the result:
//   dy = the rotation by -phi of dz,  g = dy w,  xh = r x
//   dx = r (g - xh mean(g xh)),  dw = sum over tokens and heads of dy xh
//
// Both are bound by HBM: the forward reads and writes every value once, the
// backward reads two and writes one (32768 tokens, 16/8 heads, d = 128, bf16:
// 76 us, 5.3 TB/s, and 133 us, 4.6 TB/s; a copy of 1 GiB 5.2).  Layout: a lane holds two chunks of eight
// values that contain whole pairs, D / 16 lanes hold a row, a wave takes 64 /
// (D / 16) heads of one token at a time.  A token's angles are taken once, one
// pair per lane, and shared through LDS by all of its heads: positions reach
// 2^31 and angles 10^5 radians, where fp32 has no digits left after the
// point, so the angle is reduced to a fraction of a turn in fp64.  Statistics,
// rotation and sums are fp32; a value is rounded once, where it is stored.
//
// dw: a wave keeps sums of its own over its tokens (16 per lane for queries
// and for keys), a workgroup adds up its waves in a fixed order and writes one
// partial, and a second kernel adds those: no atomics, so that a call repeated
// gives the same bits.
#include "ea_common.h"
#include "ea_internal.h"

namespace ea {

namespace {

constexpr int ROT_NT = 256;
constexpr int ROT_WAVES = ROT_NT / 64;

// Eight consecutive values as fp32.
__device__ __forceinline__ void load8(const __bf16* p, float (&x)[8]) {
  const u32x4 v = *reinterpret_cast<const u32x4*>(p);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = __uint_as_float(v[i] << 16);
    x[2 * i + 1] = __uint_as_float(v[i] & 0xFFFF0000u);
  }
}
__device__ __forceinline__ void load8(const float* p, float (&x)[8]) {
  const f32x4 a = *reinterpret_cast<const f32x4*>(p), b = *reinterpret_cast<const f32x4*>(p + 4);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[i] = a[i];
    x[4 + i] = b[i];
  }
}
__device__ __forceinline__ void store8(__bf16* p, const float (&x)[8]) {
  bf16x8 v;
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = (__bf16)x[i];
  *reinterpret_cast<bf16x8*>(p) = v;
}
__device__ __forceinline__ void store8(float* p, const float (&x)[8]) {
  *reinterpret_cast<f32x4*>(p) = f32x4{x[0], x[1], x[2], x[3]};
  *reinterpret_cast<f32x4*>(p + 4) = f32x4{x[4], x[5], x[6], x[7]};
}

// The calling lane's part of every row it works on.
template <int D>
struct RowPart {
  static constexpr int LANES = D / 16;    // lanes per row
  static constexpr int HEADS = 64 / LANES;  // rows of a wave
  int c0, c1;     // its two chunks (of eight values)
  bool rotated;   // c0 holds pairs (and c1 too, or their other halves)
  bool rotated1;  // c1 holds pairs of its own (interleaved)
  int pair0, pair1;  // first pair of c0, and of c1

  __device__ __forceinline__ RowPart(int rot, bool interleaved) {
    const int l = lane_id() % LANES, half = rot / 16;
    if (interleaved) {
      c0 = 2 * l;
      c1 = 2 * l + 1;
      rotated = 8 * c0 < rot;
      rotated1 = 8 * c1 < rot;
      pair0 = 4 * c0;
      pair1 = 4 * c1;
    } else {
      rotated = l < half;
      rotated1 = false;
      c0 = rotated ? l : 2 * l;  // (2 half chunks rotate, then two a lane)
      c1 = rotated ? l + half : c0 + 1;
      pair0 = 8 * l;
      pair1 = 0;
    }
  }
  // Rotates the lane's values by its cosines and sines (cs[0..8) of pairs
  // pair0 .., in the interleaved form four of pair0 and four of pair1).
  __device__ __forceinline__ void rotate(bool interleaved, const float (&co)[8], const float (&si)[8],
                                         float (&a)[8], float (&b)[8]) const {
    if (interleaved) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float x = a[2 * i], y = a[2 * i + 1], u = b[2 * i], v = b[2 * i + 1];
        a[2 * i] = x * co[i] - y * si[i];
        a[2 * i + 1] = x * si[i] + y * co[i];
        b[2 * i] = u * co[4 + i] - v * si[4 + i];
        b[2 * i + 1] = u * si[4 + i] + v * co[4 + i];
      }
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float x = a[i], y = b[i];
        // (a lane whose values stay has cos 1 and sin 0, and its chunks are no pairs)
        a[i] = x * co[i] - y * si[i];
        b[i] = x * si[i] + y * co[i];
      }
    }
  }
};

// Sum over the lanes of a row, in all of them.
template <int LANES>
__device__ __forceinline__ float row_sum(float v) {
#pragma unroll
  for (int o = 1; o < LANES; o <<= 1) v += __shfl_xor(v, o);
  return v;
}

// The cosines and sines of a token, one pair per lane, into `table` (a wave's
// own part of LDS).
template <int D>
__device__ __forceinline__ void angles(const RotaryArgs& a, int token, float2* table) {
  const int p = lane_id();
  if (p < a.rot / 2) {
    int axis = 0;
#pragma unroll
    for (int x = 0; x + 1 < ROT_MAX_AXES; ++x) axis += x + 1 < a.axes && p >= a.axis_end[x] ? 1 : 0;
    const double turns = (double)a.positions[(size_t)axis * a.position_stride + token] *
                         ((double)a.freqs[p] * 0.15915494309189535);
    // the nearest quarter turn apart, so that fp32 holds the rest with an error
    // of 2^-28 turns at most
    const double quarters = rint(4.0 * turns);
    const int q = (int)(quarters - 4.0 * floor(0.25 * quarters));
    float s, c;
    sincospif(2.f * (float)(turns - 0.25 * quarters), &s, &c);
    table[p] = q == 0 ? make_float2(c, s) : q == 1 ? make_float2(-s, c) : q == 2 ? make_float2(-c, -s) : make_float2(s, -c);
  }
}

// The lane's eight cosines and sines (sines times `sign`); 1 and 0 where it
// holds no pairs.
template <int D>
__device__ __forceinline__ void lane_angles(const RowPart<D>& part, bool interleaved, const float2* table,
                                            float sign, float (&co)[8], float (&si)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const bool second = interleaved && i >= 4;
    const bool ok = second ? part.rotated1 : part.rotated;
    const float2 v = table[ok ? (second ? part.pair1 + i - 4 : part.pair0 + i) : 0];
    co[i] = ok ? v.x : 1.f;
    si[i] = ok ? sign * v.y : 0.f;
  }
}

template <typename E, int D>
__device__ __forceinline__ void load_weights(const void* w, bool f32, const RowPart<D>& part, float (&w0)[8],
                                             float (&w1)[8]) {
  if (w == nullptr) {
#pragma unroll
    for (int i = 0; i < 8; ++i) w0[i] = w1[i] = 1.f;
  } else if (f32) {
    load8(static_cast<const float*>(w) + 8 * part.c0, w0);
    load8(static_cast<const float*>(w) + 8 * part.c1, w1);
  } else {
    load8(static_cast<const E*>(w) + 8 * part.c0, w0);
    load8(static_cast<const E*>(w) + 8 * part.c1, w1);
  }
}

// Row of head h (queries first, then keys) of a token.
template <typename E>
__device__ __forceinline__ E* head_row(const RotaryRows& q, const RotaryRows& k, int hq, int h, int token) {
  const bool key = h >= hq;
  const RotaryRows& t = key ? k : q;
  return static_cast<E*>(t.p) + (int64_t)token * t.row + (int64_t)(key ? h - hq : h) * t.head;
}

// Wave `parts * token + part` takes groups part, part + parts, ... of the
// token's heads.
template <typename E, int D>
__global__ __launch_bounds__(ROT_NT) void rotary_fwd_kernel(RotaryArgs a) {
  using P = RowPart<D>;
  __shared__ float2 table[ROT_WAVES][D / 2];
  const int w = wave_id(), id = blockIdx.x * ROT_WAVES + w;
  const int token = id / a.parts, first = id % a.parts;
  if (token >= a.tokens) return;
  const bool inter = a.interleaved != 0;
  const P part(a.rot, inter);
  angles<D>(a, token, table[w]);
  __builtin_amdgcn_wave_barrier();
  float co[8], si[8];
  lane_angles<D>(part, inter, table[w], 1.f, co, si);
  float wq0[8], wq1[8], wk0[8], wk1[8];
  load_weights<E, D>(a.q_weight, a.weight_f32, part, wq0, wq1);
  load_weights<E, D>(a.k_weight, a.weight_f32, part, wk0, wk1);
  const int heads = a.hq + a.hk, mine = lane_id() / P::LANES;
  for (int h0 = first * P::HEADS; h0 < heads; h0 += a.parts * P::HEADS) {
    const int h = h0 + mine;
    const bool ok = h < heads, key = h >= a.hq;
    const E* x = head_row<E>(a.q, a.k, a.hq, ok ? h : heads - 1, token);
    float x0[8], x1[8];
    load8(x + 8 * part.c0, x0);
    load8(x + 8 * part.c1, x1);
    float ss = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) ss = fmaf(x0[i], x0[i], fmaf(x1[i], x1[i], ss));
    const float r = 1.f / sqrtf(row_sum<P::LANES>(ss) * (1.f / D) + a.eps);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      x0[i] *= r * (key ? wk0[i] : wq0[i]);
      x1[i] *= r * (key ? wk1[i] : wq1[i]);
    }
    part.rotate(inter, co, si, x0, x1);
    if (ok) {
      E* y = head_row<E>(a.q_out, a.k_out, a.hq, h, token);
      store8(y + 8 * part.c0, x0);
      store8(y + 8 * part.c1, x1);
    }
  }
}

// A wave takes the tokens wave, wave + waves, ... of the launch, every head of
// each, and keeps its sums of dw.
template <typename E, int D>
__global__ __launch_bounds__(ROT_NT) void rotary_bwd_kernel(RotaryArgs a) {
  using P = RowPart<D>;
  __shared__ float2 table[ROT_WAVES][D / 2];
  __shared__ float sums[2][D];
  const int w = wave_id(), waves = gridDim.x * ROT_WAVES;
  const bool inter = a.interleaved != 0;
  const P part(a.rot, inter);
  float wq0[8], wq1[8], wk0[8], wk1[8];
  load_weights<E, D>(a.q_weight, a.weight_f32, part, wq0, wq1);
  load_weights<E, D>(a.k_weight, a.weight_f32, part, wk0, wk1);
  float dw[2][16] = {};  // of queries, of keys
  const int heads = a.hq + a.hk, mine = lane_id() / P::LANES;
  for (int token = blockIdx.x * ROT_WAVES + w; token < a.tokens; token += waves) {
    __builtin_amdgcn_wave_barrier();
    angles<D>(a, token, table[w]);
    __builtin_amdgcn_wave_barrier();
    float co[8], si[8];
    lane_angles<D>(part, inter, table[w], -1.f, co, si);
    for (int h0 = 0; h0 < heads; h0 += P::HEADS) {
      const int h = h0 + mine;
      const bool ok = h < heads, key = h >= a.hq;
      const int hs = ok ? h : heads - 1;
      const E* x = head_row<E>(a.q, a.k, a.hq, hs, token);
      const E* dz = head_row<E>(a.dq, a.dk, a.hq, hs, token);
      float x0[8], x1[8], g0[8], g1[8];
      load8(x + 8 * part.c0, x0);
      load8(x + 8 * part.c1, x1);
      load8(dz + 8 * part.c0, g0);
      load8(dz + 8 * part.c1, g1);
      float ss = 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) ss = fmaf(x0[i], x0[i], fmaf(x1[i], x1[i], ss));
      const float r = 1.f / sqrtf(row_sum<P::LANES>(ss) * (1.f / D) + a.eps);
      part.rotate(inter, co, si, g0, g1);
      float dot = 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        x0[i] *= r;
        x1[i] *= r;
        const float t0 = g0[i] * x0[i], t1 = g1[i] * x1[i];
        // (branch-free: each lane's row is a query's or a key's)
        dw[0][i] += ok && !key ? t0 : 0.f;
        dw[0][8 + i] += ok && !key ? t1 : 0.f;
        dw[1][i] += ok && key ? t0 : 0.f;
        dw[1][8 + i] += ok && key ? t1 : 0.f;
        g0[i] *= key ? wk0[i] : wq0[i];
        g1[i] *= key ? wk1[i] : wq1[i];
        dot = fmaf(g0[i], x0[i], fmaf(g1[i], x1[i], dot));
      }
      dot = row_sum<P::LANES>(dot) * (1.f / D);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        x0[i] = r * (g0[i] - x0[i] * dot);
        x1[i] = r * (g1[i] - x1[i] * dot);
      }
      if (ok) {
        E* y = head_row<E>(a.q_out, a.k_out, a.hq, h, token);
        store8(y + 8 * part.c0, x0);
        store8(y + 8 * part.c1, x1);
      }
    }
  }
  // the heads of a wave, then the waves one after another
#pragma unroll
  for (int s = 0; s < 2; ++s)
#pragma unroll
    for (int i = 0; i < 16; ++i)
#pragma unroll
      for (int o = P::LANES; o < 64; o <<= 1) dw[s][i] += __shfl_xor(dw[s][i], o);
  for (int turn = 0; turn < ROT_WAVES; ++turn) {
    if (w == turn && mine == 0) {
#pragma unroll
      for (int s = 0; s < 2; ++s)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int at = 8 * (i < 8 ? part.c0 : part.c1) + (i & 7);
          sums[s][at] = turn == 0 ? dw[s][i] : sums[s][at] + dw[s][i];
        }
    }
    __syncthreads();
  }
  for (int x = threadIdx.x; x < 2 * D; x += ROT_NT) a.partials[(size_t)blockIdx.x * 2 * D + x] = sums[x / D][x % D];
}

// dw from the workgroups' partials: 16 values per workgroup, each the sum of
// 64 threads' sums over every 64th partial (at most 16 loads each, all in
// flight at once: 1024 partials of 2 x 128 values in 5 us, with a quarter of
// the threads 20).
constexpr int DW_NT = 1024;
constexpr int DW_ROWS = DW_NT / 16;
__global__ __launch_bounds__(DW_NT) void rotary_dw_kernel(RotaryArgs a) {
  __shared__ float part[DW_ROWS][17];
  const int c = threadIdx.x & 15, r = threadIdx.x >> 4, width = 2 * a.d, col = blockIdx.x * 16 + c;
  static_assert(ROT_MAX_PARTIALS <= 16 * DW_ROWS, "sixteen loads a thread");
  float s = 0.f, v[16];
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const int x = r + i * DW_ROWS;
    v[i] = x < a.partial_count ? a.partials[(size_t)x * width + col] : 0.f;
  }
#pragma unroll
  for (int i = 0; i < 16; ++i) s += v[i];
  part[r][c] = s;
  __syncthreads();
#pragma unroll
  for (int half = DW_ROWS / 2; half >= 1; half /= 2) {
    if (r < half) part[r][c] += part[r + half][c];
    __syncthreads();
  }
  if (r == 0) {
    float* out = col < a.d ? a.dq_weight : a.dk_weight;
    if (out) out[col < a.d ? col : col - a.d] = part[0][c];
  }
}

template <typename E, int D>
hipError_t launch_fwd_d(RotaryArgs a, hipStream_t s) {
  // A wave per token takes all of its heads where there are enough tokens to
  // fill the device (8 waves on each SIMD of 256 compute units); a few tokens
  // have their heads spread over several waves.
  const int groups = (a.hq + a.hk + RowPart<D>::HEADS - 1) / RowPart<D>::HEADS;
  const int64_t enough = 8192;
  a.parts = (int)(a.tokens >= enough ? 1 : enough / a.tokens < groups ? enough / a.tokens : groups);
  const int64_t waves = (int64_t)a.tokens * a.parts;
  return launch_kernel(rotary_fwd_kernel<E, D>, dim3((unsigned)((waves + ROT_WAVES - 1) / ROT_WAVES)),
                       dim3(ROT_NT), s, a);
}

template <typename E, int D>
hipError_t launch_bwd_d(const RotaryArgs& a, hipStream_t s) {
  if (a.partial_count > 0) {
    const hipError_t e = launch_kernel(rotary_bwd_kernel<E, D>, dim3((unsigned)a.partial_count), dim3(ROT_NT), s, a);
    if (e != hipSuccess) return e;
  }
  if (!(a.dq_weight || a.dk_weight)) return hipSuccess;
  return launch_kernel(rotary_dw_kernel, dim3(2 * D / 16), dim3(DW_NT), s, a);
}

}  // namespace

int rotary_partials(int tokens) {
  const int blocks = (tokens + ROT_WAVES - 1) / ROT_WAVES;
  return blocks < ROT_MAX_PARTIALS ? blocks : ROT_MAX_PARTIALS;
}

hipError_t launch_rotary_fwd(const RotaryArgs& a, int dtype, hipStream_t s) {
  if (dtype == 0) return a.d == 64 ? launch_fwd_d<__bf16, 64>(a, s) : launch_fwd_d<__bf16, 128>(a, s);
  return a.d == 64 ? launch_fwd_d<float, 64>(a, s) : launch_fwd_d<float, 128>(a, s);
}

hipError_t launch_rotary_bwd(const RotaryArgs& a, int dtype, hipStream_t s) {
  if (dtype == 0) return a.d == 64 ? launch_bwd_d<__bf16, 64>(a, s) : launch_bwd_d<__bf16, 128>(a, s);
  return a.d == 64 ? launch_bwd_d<float, 64>(a, s) : launch_bwd_d<float, 128>(a, s);
}

}  // namespace ea
