// ea_packed.h -- where a workgroup of a kernel's packed form works.
#pragma once

#include <type_traits>

#include "ea_common.h"
#include "ea_internal.h"

namespace ea {

template <typename A>
struct is_packed : std::false_type {};
template <typename A>
struct is_packed<Packed<A>> : std::true_type {};

// Tile `tile` (64 << size rows) of a sequence of n rows and T blocks, for
// query head `head` (dK/dV: key head `head`, part `part` of its query heads).
struct Place {
  int head, part, item, tile, seq, start, n, T;
  int block;             // the sequence's first block among all
  int gap;               // rows before it of a sequence that is left out
  size_t row0, blk0;  // of the query head: its first row in tau, and first block in the tables
};

// The place of workgroup b of a grid of `heads` workgroups per tile, heads
// fastest.  Query heads of one key head are `kv_heads` apart in that order, so
// that with kv_heads a multiple of 8 they meet on the XCD that holds their
// keys (workgroups are handed to the eight XCDs in turn).  False: no such tile.
__device__ __forceinline__ bool packed_place(const PackedArgs& pk, int b, int heads, bool key_heads, Place& at) {
  const int x = b % heads, kv = x % pk.kv_heads, rest = x / pk.kv_heads;
  at.item = b / heads;
  at.head = key_heads ? kv : kv * pk.group + rest;
  at.part = key_heads ? rest : 0;
  if (at.item >= ((const ci32*)pk.header->count)[pk.size]) return false;
  const ci32* const tile = (const ci32*)(pk.tiles + at.item);
  const ci32* const seq = (const ci32*)(pk.seqs + tile[0]);
  at.seq = tile[0];
  at.tile = tile[1];
  at.start = seq[0];
  at.n = seq[1];
  at.T = (at.n + BLK - 1) / BLK;
  at.row0 = (size_t)at.head * pk.tokens + at.start;
  at.block = seq[2];
  at.gap = seq[3];
  at.blk0 = (size_t)at.head * pk.blocks + at.block;
  return at.n > 0;
}

// Sets rows [r0, r1) of `head` to the 32-bit word `word` (every thread of a
// workgroup of NT).  D values of type E, 16-byte aligned rows.
template <typename E, int D, int NT>
__device__ __forceinline__ void fill_rows(E* base, const Strides& st, int head, int r0, int r1, uint32_t word) {
  constexpr int VEC = 16 / (int)sizeof(E), CPR = D / VEC;
  for (int64_t x = threadIdx.x; x < (int64_t)(r1 - r0) * CPR; x += NT)
    *reinterpret_cast<u32x4*>(base + (r0 + x / CPR) * st.row + head * st.head + (x % CPR) * VEC) =
        u32x4{word, word, word, word};
}
// Sets the rows of `head` that belong to no sequence to 0.
template <typename E, int D, int NT>
__device__ void zero_rest(const PackedArgs& pk, E* base, const Strides& st, int head) {
  fill_rows<E, D, NT>(base, st, head, 0, pk.header->begin, 0u);
  fill_rows<E, D, NT>(base, st, head, pk.header->end, pk.tokens, 0u);
}
// The rows of `head` that belong to sequences which are left out: NaN, since
// whoever gave such a sequence should see it.  By the workgroups of item 0 (the
// rows behind the last sequence that is computed; `work`: whether it has one)
// and of every sequence's tile 0 (those before it).
template <typename E, int D, int NT>
__device__ void left_out(const PackedArgs& pk, const Place& at, bool work, E* base, const Strides& st, int head) {
  constexpr uint32_t NAN_WORD = sizeof(E) == 2 ? 0x7FC07FC0u : 0x7FC00000u;
  if (at.item == 0) fill_rows<E, D, NT>(base, st, head, pk.header->last, pk.header->end, NAN_WORD);
  if (work && at.tile == 0) fill_rows<E, D, NT>(base, st, head, at.start - at.gap, at.start, NAN_WORD);
}

}  // namespace ea
