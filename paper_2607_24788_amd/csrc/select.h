// Launch descriptors of the attention over selected pages (kernels in
// select.hip, host side in select_api.hip).
#pragma once

#include "paged.h"

namespace glide {

// Rows of one workgroup of page_scores.
constexpr int kScoreRows = 8;
// Its workgroups take more pages each where there would be more than these.
constexpr int64_t kScoreWorkgroups = 4096;
// As many units (row, KV head) have a wave each (picked_rows), eight to a CU;
// fewer share workgroups (attend_rows).  bf16, d = 128: 2048 units of 2048 keys
// 168 us by waves, 207 by workgroups; 1024 of them 131, 111.
constexpr int64_t kPickedUnits = 2048;
// Rows of a sequence share a wave (picked_tiles; bf16, pages of 32 tokens or more)
// where that leaves so many waves, of 1.6 rows or more on average.  d = 128, 32 /
// 8 heads: 1880 rows of 16 of 23 pages of 128 tokens 409 us, 928 by picked_rows;
// 2048 of 32 of 250 pages of 64 837, 1221; 256 of them (512 waves) 277, 168.
// 64 / 8 heads, two rows to a wave: 1881 rows of 12 of 39 pages of 128 493, 722,
// of 40 of 559 of 32 945, 1043; 60 sequences of 5 rows (1.67 to a wave) 223, 289
// and 292, 324; 200 of one or two (1.5) 318, 322 and 358, 327.
// Pages of 16 tokens fill half a tile: there only if a page is selected by enough
// of a wave's rows, the root of them.  2000 rows of 250 pages, by waves / alone: four
// rows to a wave, 60 pages each (1.4 rows to a page) 766 / 721 us, 120 (2.1) 1043 /
// 1143, 180 1206 / 1568; 16 rows (d = 64), 30 (2.2) 475 / 387, 60 (3.9) 563 / 567,
// 120 604 / 928.
constexpr int64_t kSharedUnits = 1024;
// A launch's scores take at most so many bytes (one row's at least).
constexpr int64_t kMaxScoreBytes = int64_t(1) << 28;

// Who attends to a launch's rows: the four waves of a workgroup to a unit in
// pieces (attend_rows), a wave to a unit (picked_rows), a wave to several rows
// (picked_tiles).
enum class SparseForm : int32_t { workgroups, waves, tiles };
// Which, of the first launch of a valid call of one row or more; not a part of
// the library's interface (for its tests).
extern "C" int32_t glide_internal_sparse_form(const glide_paged_config* cfg, const int32_t* cu_seqlens_host,
                                              int32_t n_select, int64_t max_len);

struct SelectArgs {
  const char* q;         // [T][Hq][d]
  const char* bounds;    // [n_pages][Hkv][2][d]
  const int32_t *table, *lens;
  int32_t Hq, Hkv, G;
  int32_t n_pages, max_pages, shift, cap;
  int32_t n_select, n_first, n_recent;
  int32_t negative;      // the score's scale is below 0
  int32_t single;        // every sequence of the launch has one row
  int32_t chunk;         // pages of one workgroup of page_scores, at a time: a multiple of 32
  int32_t row0, row1;    // packed rows of this launch
  uint64_t* keys;        // [row1 - row0][Hkv][max_pages]
  int32_t* selected;     // [T][Hkv][n_select]
  int32_t *pages, *held; // of this launch's rows: [..][Hkv][n_select] pages, [..][Hkv] tokens
};

// seqs: start and len of whole sequences; tile0 counts workgroups of kScoreRows
// rows among row0 .. row1 - 1.  pages: of a sequence, at most (it sizes a grid
// only)
hipError_t launch_select(const SelectArgs& a, const PagedSeqs& s, int64_t pages, int d, int dtype, hipStream_t stream);

// Tiles of picked_tiles: first positions, kNoTile behind the last.
constexpr int32_t kTileSlots = 32, kNoTile = 0x7fffffff;
// The tile behind the one at j0 in the same page, among positions up to tmax;
// kNoTile where there is none.
constexpr int32_t next_in_page(int32_t j0, int32_t shift, int32_t tmax) {
  if (j0 == kNoTile) return kNoTile;  // (before j0 is added to)
  const int32_t j = j0 + kTileSlots;
  return (j & ((1 << shift) - 1)) != 0 && j <= tmax ? j : kNoTile;
}

// The attention of a launch's units (row, KV head), a wave each; a as for
// launch_paged_decode with per_head, in one piece.
hipError_t launch_picked(const PagedArgs& a, int32_t units, int d, int dtype, hipStream_t stream);

// The same (bf16) with `rows` neighbouring rows of a sequence (16 / G, 2 or more) to
// a wave, over pages of 16 tokens or more; a: the sequences' own table and lens;
// seqs.tile0 counts waves per KV head.
hipError_t launch_picked_tiles(const PagedArgs& a, const PagedSeqs& s, const SelectArgs& e, int rows, int d,
                               hipStream_t stream);

}  // namespace glide
