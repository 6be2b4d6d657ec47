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
  at.blk0 = (size_t)at.head * pk.blocks + at.block;
  return at.n > 0;
}

// Sets the rows of `head` that belong to no sequence to 0 (every thread of a
// workgroup of NT).  D values of type E, 16-byte aligned rows.
template <typename E, int D, int NT>
__device__ void zero_rest(const PackedArgs& pk, E* base, const Strides& st, int head) {
  constexpr int VEC = 16 / (int)sizeof(E), CPR = D / VEC;
  const int begin = pk.header->begin, rest = begin + pk.tokens - pk.header->end;
  for (int64_t x = threadIdx.x; x < (int64_t)rest * CPR; x += NT) {
    const int r = (int)(x / CPR), row = r < begin ? r : r - begin + pk.header->end;
    *reinterpret_cast<u32x4*>(base + (int64_t)row * st.row + head * st.head + (x % CPR) * VEC) = u32x4{0, 0, 0, 0};
  }
}

}  // namespace ea
