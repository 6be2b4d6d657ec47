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
// walk's step is a scalar load and a few instructions for the whole wave.
#include "ea_common.h"
#include "ea_internal.h"

namespace ea {

namespace {

constexpr int PLAN_NT = 256;

// The sequences in turn, each with its rows: none where cu does not describe
// 1 .. max_seqlen rows inside the tensors and behind the sequences before, so
// that whatever cu holds, the rows listed are those of `tokens` rows at most
// and every list has room for its tiles.
template <typename F>
__device__ __forceinline__ void walk(const PlanArgs& a, F&& use) {
  const ci32* cu = (const ci32*)a.cu;
  int last = 0, begin = cu[0];
  for (int s = 0; s < a.seq_count; ++s) {
    const int end = cu[s + 1];
    // (begin >= 0 by then, so the difference does not overflow)
    const bool ok = begin >= last && end > begin && end <= a.tokens && end - begin <= a.max_seqlen;
    use(s, begin, ok ? end - begin : 0);
    if (ok) last = end;
    begin = end;
  }
}

__device__ __forceinline__ int tiles_of(int rows, int size) { return (rows + (64 << size) - 1) / (64 << size); }

__global__ __launch_bounds__(PLAN_NT) void plan_kernel(PlanArgs a) {
  const int lane = lane_id();
  const int wave = __builtin_amdgcn_readfirstlane(blockIdx.x * (PLAN_NT / 64) + wave_id());
  // the wave's sequence, which 64 of its tiles, the blocks before it, and the
  // rows between it and the sequence before (or cu[0])
  int seq = -1, start = 0, len = 0, chunk = 0, waves = 0, block = 0, gap = 0, total[2] = {};
  const int cu0 = min(max(((const ci32*)a.cu)[0], 0), a.tokens);
  int first = cu0, last = cu0;
  walk(a, [&](int s, int begin, int n) {
    const int need = max(tiles_of(n, 6), 1);  // (an empty sequence has a record too)
    if (wave >= waves && wave < waves + need) {
      seq = s;
      start = n ? begin : 0;
      len = n;
      chunk = wave - waves;
      block = total[0];
      gap = n ? max(begin - last, 0) : 0;
    }
    waves += need;
    if (n) {
      first = min(first, begin);
      last = begin + n;
    }
#pragma unroll
    for (int z = 0; z < 2; ++z) total[z] += tiles_of(n, z);
  });
  if (wave == 0 && lane == 0) {
    const int end = max(last, min(((const ci32*)a.cu)[a.seq_count], a.tokens));
    *a.header = PackedHeader{{total[0], total[1]}, first, end, last};
  }
  if (seq < 0) return;
  if (chunk == 0 && lane == 0) a.seqs[seq] = PackedSeq{start, len, block, gap};
  const int t = 64 * chunk + lane;
  // tiles before tile t of each size: longer ones of any sequence, and as long
  // ones of an earlier one.  Causal tiles are as long as their number, others
  // as long as their sequence.
  int before[2] = {};
  walk(a, [&](int s, int, int n) {
#pragma unroll
    for (int z = 0; z < 2; ++z) {
      const int N = tiles_of(n, z);
      if (a.causal)
        before[z] += max(N - t - 1, 0) + (s < seq && N > t ? 1 : 0);
      else
        before[z] += n > len || (n == len && s < seq) ? N : 0;
    }
  });
#pragma unroll
  for (int z = 0; z < 2; ++z)
    if (t < tiles_of(len, z)) a.tiles[z][before[z] + (a.causal ? 0 : t)] = PackedTile{seq, t};
}

}  // namespace

hipError_t launch_plan(const PlanArgs& a, hipStream_t s) {
  const int waves = packed_tiles(a.tokens, a.seq_count, 6);  // 64 << 6 rows: 64 blocks
  return launch_kernel(plan_kernel, dim3((unsigned)((waves + PLAN_NT / 64 - 1) / (PLAN_NT / 64))), dim3(PLAN_NT), s, a);
}

}  // namespace ea
