// How the trees' attention is shared out: which kernel, columns of a workgroup, items of a launch, what its workspace has room for.  Plain C++, so that a program without HIP can include it.
#pragma once
#include <algorithm>

#include "la.h"
#include "la_attend_plan.h"

namespace la {

constexpr int TA_WAVES = 4, TA_WHOLE_WAVES = 8;  // of a workgroup; where requests are not cut and workgroups are few
constexpr size_t TA_NOTE = 8;                    // bytes of what the join is told of a request

// Whether the wide kernel is for this shape.
inline bool tree_wide(int dtype, int head_dim, int page_size) {
  return dtype != LA_F32 && page_size % 8 == 0 && (head_dim == 64 || head_dim == 96 || head_dim == 128 || head_dim == 256);
}

// Which kernel, and what is cut; each rule with both sides as measured, in microseconds, 32 query heads of 128 channels unless said.
// TA_FEW: where no request is cut and workgroups of 16 columns are no more than the CUs, eight waves share a workgroup's keys (1 tree of 8 rows at 500 keys: 11.7, with four waves 14.7; 1 of 16:
//   13.5 and 16.4).  More than 32 columns, or more workgroups, go through LDS.
// Wide from 17 columns: 1 x 8 rows at 1000, 11.7 and with the other kernel 14.4; at 2000, 13.7 and 16.2; 8 x 8 at 4000, 35.8 both; 2 x 57 at 19000 with pages of 8, 50 and 134.  At 16 columns and
// fewer three quarters of its waves would idle.
constexpr int TA_FEW = 256;
// Requests are left whole up to AT_WHOLE keys (16 x 16 rows at 400: 16.4, cut 21.4; 16 x 64 at 500: 35 and 46), float ones up to half as many, their products being 1/16 as fast (3 x 8 at 500: cut
//   11.0, 13.5 whole).  Where wide workgroups of whole requests are fewer than TA_MANY, only up to TA_WHOLE_WIDE keys (1 x 64 at 500: cut 23, 34 whole; 4 x 16 at 500, 64 workgroups: 18.6 whole and
//   cut 16.5, but 4 x 32 at 600, as many, 22.6 and 26.5: the rule takes the smaller loss of the two), and so always for heads of 256 channels (22 of 1 to 12 rows at up to 747: cut 21, whole 34; one row at 500 14.3 and 18.3).
constexpr int TA_WHOLE_WIDE = 256, TA_MANY = 64;
// 128 columns a workgroup rather than 64 (K and V pass through LDS half as often) where one of 512 then has this many keys, if all requests are as long as the table: 4 x 64 rows at 500, 128
//   columns 26.4 and 64 20.0, 1 x 40 at 3000, 28.9 and 23.5, 4 x 64 at 4000, 512 keys, 49.9 and 48.3, 4 x 40 of three heads of 96 channels at 16000, 930 keys, 57.4 and 64.5, 16 x 64 at 4000,
//   2000 keys, 129 and 134, 4 x 64 at 16000, 119 and 134, 2 x 64 at 65000, 230 and 284.  Heads of 256 channels (one of 16 query heads), one workgroup a CU: 1 x 10 at 15800,
//   38 keys, 28.5 and 26.9, 8 x 33 at 2000, 129 keys, 38.2 and 44.1, 4 x 30 at 5000, 146 keys, 39.6 and 42.2.
constexpr int TA_LONG = 768, TA_LONG_256 = 128;
// Workgroups that items are cut for: one of 64 columns a CU (16 of 1 to 16 rows at up to 4096, 25.5; 384 of them 27.4, 512 26.1; 32 x 16 rows at 2000 62, 75 and 69), or two where a request has
//   several and each keeps TA_SHARE keys (1 x 64 rows of 64 heads at 8000: 48.1, one 54.9; 1 x 40 at 3000, 117 keys: 23.5 and 21.9); two of 128; at_workgroups' for the kernel above.
constexpr int TA_SHARE = 256;
// Bytes of the items' records at most; fewer items keep to it.  A record is written and read again: 4 us and 10 us at 34 KB an item and kv head of two requests of 64 rows.
constexpr size_t TA_RECORDS = (size_t)64 << 20;
// The join's waves share a row's and head's records where a request may have that many items and rows and heads are fewer than waves that fill the chip: one row of 8 heads at 30000 keys 37.6, shared
//   21.0, 1 x 10 of 16 heads of 256 channels at 15800, 37.7 and 28.3, 1 x 8 of 32 at 4000, 17.8 and 16.1; from 8 or 4 items a request on: no difference; 2 x 64 of 32 heads: 231 both.
constexpr int TA_MANY_RECORDS = 16, TA_PAIRS = 2048;
struct TreePlan {
  int wide, waves, tiles, uncut, target, items;
  bool split;  // the join's waves share a row's records
  unsigned grid;
  size_t notes, list, bytes;
};
// Kernel, columns of a workgroup and workgroups of an item and kv head; how many items are resident at once.  cap: positions that the table has room for.
inline TreePlan ta_shape(const la_pages_desc &p, int Hq, int max_rows, int R, long long cap) {
  TreePlan r{};
  const int columns = Hq / p.n_kv_heads * max_rows;
  const bool few = cap <= AT_WHOLE && p.head_dim <= 128 && columns <= 32 && (long long)R * p.n_kv_heads * ((columns + 15) / 16) <= TA_FEW;
  const double share = (double)R * p.n_kv_heads * columns * (double)cap / 512;  // columns times keys of one of 512 workgroups
  if (columns > 16 && !few && tree_wide(p.dtype, p.head_dim, p.page_size)) r.wide = columns > 64 && share >= 128. * (p.head_dim <= 128 ? TA_LONG : TA_LONG_256) ? 128 : 64;
  r.waves = few ? TA_WHOLE_WAVES : TA_WAVES;
  r.tiles = (columns + (r.wide ? r.wide : 16) - 1) / (r.wide ? r.wide : 16);
  const int groups = !r.wide ? at_workgroups(p.head_dim) : p.head_dim <= 128 && (r.wide == 128 || (r.tiles > 1 && share >= 64. * TA_SHARE)) ? 512 : 256;
  r.target = std::max(1, groups / (p.n_kv_heads * r.tiles));
  return r;
}
inline TreePlan ta_plan(const la_pages_desc &p, int Hq, int max_blocks, int R, int max_rows) {
  const long long cap = (long long)max_blocks * p.page_size;
  TreePlan r = ta_shape(p, Hq, max_rows, R, cap);
  const int target = r.target;
  r.target = 0;
  const bool sparse = (long long)R * p.n_kv_heads * r.tiles < TA_MANY;
  r.uncut = p.head_dim > 128 || (r.wide && sparse) ? TA_WHOLE_WIDE : p.dtype == LA_F32 ? AT_WHOLE / 2 : AT_WHOLE;
  const bool whole = cap <= r.uncut;
  if (!whole) r.waves = TA_WAVES;
  if (!whole && sparse && p.dtype == LA_F32) r.uncut = std::min(r.uncut, TA_WHOLE_WIDE);  // (the join is launched anyway, and four waves have the keys: 1 x 8 rows at 402, 16.4 and 11.8)
  r.items = R;
  if (!whole) {
    const size_t record = (size_t)Hq * max_rows * (p.head_dim + 4) * 4;
    const long long pieces = R * ((cap + AT_PIECE - 1) / AT_PIECE);
    for (r.target = target;; r.target = r.target * 3 / 4) {
      const int cut = (2 * R > r.target ? AT_FINE : 1) * r.target;
      r.items = (int)std::min((long long)cut + R, pieces);
      r.bytes = std::min(r.items, 2 * cut) * record;  // (of requests that are cut: fewer than `cut`, with one item more than their share of `cut` each)
      if (r.bytes <= TA_RECORDS || r.target == 1) break;
    }
    r.split = std::min((long long)r.target, (cap + AT_PIECE - 1) / AT_PIECE) >= TA_MANY_RECORDS * (long long)R && (long long)R * max_rows * Hq < TA_PAIRS;
    r.notes = r.bytes;
    r.bytes += ((size_t)R * TA_NOTE + 15) / 16 * 16;
    if (R > 64) {
      r.list = r.bytes;
      r.bytes += r.items * sizeof(AtItem) + (size_t)R * 4;
    }
  }
  const long long groups = (long long)r.items * p.n_kv_heads, grid = r.tiles > 1 ? (groups + 7) / 8 * 8 * r.tiles : groups;
  r.grid = grid < 1ll << 24 ? (unsigned)grid : 1u << 24;
  return r;
}

// Workspace of trees of up to LA_MAX_ROWS rows of as many requests together, at any of their sizes.
inline size_t tree_attend_bytes(const la_pages_desc &p, int Hq) {
  size_t most = 0;
  la_pages_desc d = p;
  for (int page : {16, 17})  // (a page size that the wide kernel takes, one that it does not; the longest table, for which the most items are resident)
    for (int rows = 1; rows <= LA_MAX_ROWS; ++rows) {
      d.page_size = page;
      const size_t record = (size_t)Hq * rows * (p.head_dim + 4) * 4;
      most = std::max(most, std::min(2 * AT_FINE * (size_t)ta_shape(d, Hq, rows, 1, 1ll << 62).target, std::max(TA_RECORDS / record, (size_t)2 * AT_FINE)) * record);
    }
  return most + LA_MAX_ROWS * TA_NOTE;
}

}  // namespace la
