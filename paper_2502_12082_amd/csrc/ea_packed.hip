// ea_packed.hip -- the tiles of packed sequences, listed on the GPU.
//
// Sequence s of a batch packed into one row of tokens is the rows [cu[s],
// cu[s + 1]).  Every kernel of the packed forms gives a workgroup one tile of
// 64 or 128 rows of one sequence, so it needs to know which tile of which
// sequence workgroup x has, those with the most keys first (a grid lasts as
// long as the workgroup that ends last).  That is a function of cu alone, and
// cu is known on the device: one launch lists the tiles for every layer's
// forward and backward of a step, without the host having to wait for it.
//
// One wave takes 64 tiles of one sequence.  It finds its sequence by walking
// over cu (at most one wave more than necessary per sequence is launched), and
// the place of each of its tiles in the order by a second walk that counts the
// tiles before it: no sort, no atomics, and the same order every time.  A
// walk's step is 64 sequences, one to a lane, the next ones on their way
// meanwhile; the work still grows with the square of the sequences, so their
// number is bounded (MAX_SEQS).  A call on 700, 4096, 16384 and 65536 sequences
// of one row takes 15, 83, 840 and 11900 us (one sequence at a step, by scalar
// loads: 204, 3030, 42800 and 661000).
#include "ea_common.h"
#include "ea_internal.h"

namespace ea {

namespace {

constexpr int PLAN_NT = 256;

// Sum over the wave, in all lanes.
__device__ __forceinline__ int wave_sum(int v) {
#if defined(__HIP_DEVICE_COMPILE__)
  // (inside quads, mirrored inside 8 and 16 lanes, then over the four rows)
  v += __builtin_amdgcn_update_dpp(0, v, 0xB1, 0xf, 0xf, true);
  v += __builtin_amdgcn_update_dpp(0, v, 0x4E, 0xf, 0xf, true);
  v += __builtin_amdgcn_update_dpp(0, v, 0x141, 0xf, 0xf, true);
  v += __builtin_amdgcn_update_dpp(0, v, 0x140, 0xf, 0xf, true);
  return __builtin_amdgcn_readlane(v, 0) + __builtin_amdgcn_readlane(v, 16) + __builtin_amdgcn_readlane(v, 32) +
         __builtin_amdgcn_readlane(v, 48);
#else
  return v;
#endif
}

// The sequences in turn, 64 at a time, each with its rows: none where cu does
// not describe 1 .. max_seqlen rows inside the tensors and behind the sequences
// before, so that whatever cu holds, the rows listed are those of `tokens` rows
// at most and every list has room for its tiles.  use(s0, begin, n, prev) takes
// the lane's sequence s0 + lane (n: its rows, 0 past the last) and the end of
// the last one that counts before s0; it returns whether to go on.
template <typename F>
__device__ __forceinline__ void walk(const PlanArgs& a, F&& use) {
  const int lane = lane_id();
  int last = 0, prev = -1;  // last: the end of the sequences that count so far
  int begin = a.cu[min(lane, a.seq_count)], end = a.cu[min(lane + 1, a.seq_count)];
  for (int s0 = 0; s0 < a.seq_count; s0 += 64) {
    const int next = min(s0 + 64 + lane, a.seq_count);
    const int begin2 = a.cu[next], end2 = a.cu[min(next + 1, a.seq_count)];
    // (where begin >= 0, so that the difference does not overflow)
    bool ok = begin >= 0 && end > begin && end <= a.tokens && end - begin <= a.max_seqlen;
    if (__ballot(begin < last || end < begin) != 0ull) {
      // some sequence begins before an earlier one ends: one after another
      bool mine = false;
      int at = last;
      for (int i = 0; i < 64; ++i) {
        const bool counts = __builtin_amdgcn_readlane((int)ok, i) && __builtin_amdgcn_readlane(begin, i) >= at;
        if (counts) at = __builtin_amdgcn_readlane(end, i);
        if (lane == i) mine = counts;
      }
      ok = mine;
    }
    if (!use(s0, begin, ok ? end - begin : 0, prev)) return;
    const unsigned long long m = __ballot(ok);
    if (m != 0ull) prev = last = __builtin_amdgcn_readlane(end, 63 - __builtin_clzll(m));
    begin = begin2;
    end = end2;
  }
}

__device__ __forceinline__ int tiles_of(int rows, int size) { return (rows + (64 << size) - 1) / (64 << size); }

__global__ __launch_bounds__(PLAN_NT) void plan_kernel(PlanArgs a) {
  const int lane = lane_id();
  const int wave = __builtin_amdgcn_readfirstlane(blockIdx.x * (PLAN_NT / 64) + wave_id());
  // the wave's sequence, which 64 of its tiles, the blocks before it, and the
  // rows between it and the sequence before (or cu[0])
  int seq = -1, start = 0, len = 0, chunk = 0, waves = 0, block = 0, gap = 0, total[2] = {};
  const int cu0 = min(max(a.cu[0], 0), a.tokens);
  int first = cu0, last = cu0;
  walk(a, [&](int s0, int begin, int n, int prev) {
    const int need = s0 + lane < a.seq_count ? max(tiles_of(n, 6), 1) : 0;  // (an empty sequence has a record too)
    int incl = need;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int v = __shfl_up(incl, o);
      if (lane >= o) incl += v;
    }
    const unsigned long long some = __ballot(n > 0);
    const unsigned long long mine = __ballot(wave >= waves + incl - need && wave < waves + incl);
    if (mine != 0ull) {
      const int i = __builtin_ctzll(mine);
      seq = s0 + i;
      len = __builtin_amdgcn_readlane(n, i);
      start = len ? __builtin_amdgcn_readlane(begin, i) : 0;
      chunk = wave - waves - __builtin_amdgcn_readlane(incl - need, i);
      block = total[0] + wave_sum(lane < i ? tiles_of(n, 0) : 0);
      const unsigned long long before = some & ((1ull << i) - 1);
      const int from = before ? __builtin_amdgcn_readlane(begin + n, 63 - __builtin_clzll(before)) : prev < 0 ? cu0 : prev;
      gap = len ? max(start - from, 0) : 0;
      if (wave != 0) return false;  // (the totals are the first wave's)
    }
    waves += __builtin_amdgcn_readlane(incl, 63);
    if (some != 0ull) {
      first = min(first, __builtin_amdgcn_readlane(begin, __builtin_ctzll(some)));
      last = __builtin_amdgcn_readlane(begin + n, 63 - __builtin_clzll(some));
    }
#pragma unroll
    for (int z = 0; z < 2; ++z) total[z] += wave_sum(tiles_of(n, z));
    return true;
  });
  if (wave == 0 && lane == 0) {
    const int end = max(last, min(a.cu[a.seq_count], a.tokens));
    *a.header = PackedHeader{{total[0], total[1]}, first, end, last};
  }
  if (seq < 0) return;
  if (chunk == 0 && lane == 0) a.seqs[seq] = PackedSeq{start, len, block, gap};
  const int t0 = 64 * chunk, t = t0 + lane;
  const int mine = min(tiles_of(len, 0) - t0, 64);  // the wave's tiles of 64 rows
  if (mine <= 0) return;
  // tiles before tile t of each size: longer ones of any sequence, and as long
  // ones of an earlier one.  Causal tiles are as long as their number, others
  // as long as their sequence.
  int before[2] = {};
  constexpr int FEW = 8;
  if (!a.causal) {
    walk(a, [&](int s0, int, int n, int) {
      const bool ahead = n > len || (n == len && s0 + lane < seq);
#pragma unroll
      for (int z = 0; z < 2; ++z) before[z] += ahead ? tiles_of(n, z) : 0;
      return true;
    });
#pragma unroll
    for (int z = 0; z < 2; ++z) before[z] = wave_sum(before[z]) + t;
  } else if (mine <= FEW) {
    // a lane counts for its sequences, every tile in turn
    int count[2][FEW] = {};
    walk(a, [&](int s0, int, int n, int) {
      const int less = s0 + lane >= seq ? 1 : 0;
#pragma unroll
      for (int z = 0; z < 2; ++z)
#pragma unroll
        for (int k = 0; k < FEW; ++k) count[z][k] += max(tiles_of(n, z) - t0 - k - less, 0);
      return true;
    });
#pragma unroll
    for (int z = 0; z < 2; ++z)
#pragma unroll
      for (int k = 0; k < FEW; ++k) {
        const int sum = wave_sum(count[z][k]);
        if (lane == k) before[z] = sum;
      }
  } else {
    // a lane counts for its tile, every sequence in turn that is long enough
    walk(a, [&](int s0, int, int n, int) {
      for (unsigned long long m = __ballot(tiles_of(n, 0) > t0); m != 0ull; m &= m - 1) {
        const int i = __builtin_ctzll(m), rows = __builtin_amdgcn_readlane(n, i), less = s0 + i >= seq ? 1 : 0;
#pragma unroll
        for (int z = 0; z < 2; ++z) before[z] += max(tiles_of(rows, z) - t - less, 0);
      }
      return true;
    });
  }
#pragma unroll
  for (int z = 0; z < 2; ++z)
    if (t < tiles_of(len, z)) a.tiles[z][before[z]] = PackedTile{seq, t};
}

}  // namespace

hipError_t launch_plan(const PlanArgs& a, hipStream_t s) {
  const int waves = packed_tiles(a.tokens, a.seq_count, 6);  // 64 << 6 rows: 64 blocks
  return launch_kernel(plan_kernel, dim3((unsigned)((waves + PLAN_NT / 64 - 1) / (PLAN_NT / 64))), dim3(PLAN_NT), s, a);
}

}  // namespace ea
