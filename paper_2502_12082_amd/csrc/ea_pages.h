// ea_pages.h -- where a token of a paged 4-bit cache lies, and what one row of a
// page table keeps and needs in an update.  Plain integer arithmetic, the same on
// the device and in a host build (the tests compile it with the host's compiler):
// everything that a table, a position or a length on the device can say is
// checked here, so that no value of theirs leads outside the buffers.
#pragma once

#include <stdint.h>

#if defined(__HIPCC__)
#define EA_HD __host__ __device__ __forceinline__
#else
#define EA_HD inline
#endif

namespace ea {

// Tokens of a tile; a tile of one key head holds 16 rows of D / 2 bytes of codes
// (e2m1, two to a byte), then 16 rows of D / 32 bytes of scales (e8m0).
constexpr int PAGE_TILE = 16;
EA_HD constexpr int tile_bytes(int D) { return PAGE_TILE * (D / 2 + D / 32); }

// A cache: pages of kv_heads heads, of each the tiles of its keys and then those
// of its values.
struct PageDims {
  int32_t pages, shift, kv_heads, head_dim;  // a page holds 1 << shift tokens
};
EA_HD int64_t part_bytes(const PageDims& c) {  // the keys, or the values, of one head in one page
  return (int64_t)tile_bytes(c.head_dim) << (c.shift - 4);
}
EA_HD int64_t page_bytes(const PageDims& c) { return 2 * part_bytes(c) * c.kv_heads; }

struct PageTable {
  const int32_t* ids;
  int32_t rows, width;
  int64_t stride;  // from row to row
};
// Page of token `at` of row `row`, -1 where there is none: no such row, no such
// place in it, or an entry that names no page.
EA_HD int32_t page_of(const PageDims& c, const PageTable& t, int32_t row, int32_t at) {
  if (row < 0 || row >= t.rows || at < 0 || (at >> c.shift) >= t.width) return -1;
  const int32_t id = t.ids[row * t.stride + (at >> c.shift)];
  return id >= 0 && id < c.pages ? id : -1;
}
// Bytes from the cache's start to the tile of token `at` of a page, for key head
// `head`: of its keys, or (values) of its values.
EA_HD int64_t tile_at(const PageDims& c, int32_t page, int32_t head, bool values, int32_t at) {
  const int32_t tile = (at & ((1 << c.shift) - 1)) >> 4;
  return page * page_bytes(c) + (2 * (int64_t)head + (values ? 1 : 0)) * part_bytes(c) +
         (int64_t)tile * tile_bytes(c.head_dim);
}

// One row of an update: it goes on from a row of `old` tokens and gains `count`
// (loses, where negative).
struct RowPlan {
  int32_t old, wanted;  // tokens before and after
  int32_t kept;         // pages that stay: entries [0, kept) of the row that it goes on from
  int32_t grown;        // pages behind those
  bool fits;            // the table is wide enough; else the row stays as it is
  bool writes;          // it gains tokens and its last page has room: the first of them go there
};
EA_HD int32_t pages_of(int64_t tokens, int shift) { return (int32_t)((tokens + (1 << shift) - 1) >> shift); }
EA_HD RowPlan plan_row(int32_t length, int32_t count, int32_t width, int shift) {
  RowPlan r;
  const int64_t most = (int64_t)width << shift;
  const int64_t old = length < 0 ? 0 : length > most ? most : length;
  int64_t wanted = old + count;
  if (wanted < 0) wanted = 0;
  r.fits = wanted <= most;
  if (!r.fits) wanted = old;
  r.old = (int32_t)old;
  r.wanted = (int32_t)wanted;
  r.kept = pages_of(wanted < old ? wanted : old, shift);
  r.grown = pages_of(wanted, shift) - r.kept;
  r.writes = wanted > old && (old & ((1 << shift) - 1)) != 0;
  return r;
}
// A page that rows are about to write to, and that no other row holds, is kept by one of
// them: row `keeper`; the others get copies, which are made before anything is written.
// With pages enough for all copies the keeper is the lowest of them.  Otherwise rows that get no
// copy go on holding the page, and the keeper must not write where they have tokens: it
// is the row whose tokens end furthest into the page, of several the lowest.  (Either way there
// are as many copies.)
EA_HD bool copies(int32_t holders, int32_t writers, int32_t keeper, int32_t row) {
  return holders > 1 && (holders > writers || keeper != row);
}
// A number of a row of `old` tokens that writes to its last page, the smallest of that
// row's; pages hold at most 2^10 tokens, and rows are fewer than 2^20 (their numbers).
constexpr int KEEPER_ROW_BITS = 20;
EA_HD int32_t keeper_key(int32_t old, int shift, int32_t row) {
  const int32_t end = (1 << shift) - 1;
  return (end - (old & end)) << KEEPER_ROW_BITS | row;
}
EA_HD int32_t keeper_row(int32_t key) { return key & ((1 << KEEPER_ROW_BITS) - 1); }

}  // namespace ea
