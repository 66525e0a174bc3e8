// How the paged attention's keys are dealt to workgroups: the items of a row, how many of them a launch and its workspace have room for.  Plain C++, so that a program without HIP can
// include it; the kernels form the items from the rows' positions with the same functions.
#pragma once
#include <stddef.h>

#ifdef __HIPCC__
#define LA_HD __host__ __device__
#else
#define LA_HD
#endif

namespace la {

struct AtItem {
  int b, r, n, C, index, first, count;  // row, its request and keys; keys per item; which of the row's items; the row's first item; how many it has
  int record;  // of a row that is cut: the item among all such rows' items
};

constexpr int AT_ROWS = 16;        // query heads of a tile
constexpr int AT_PIECE = 128;      // an item's keys are a multiple of this (but for a row's last)
constexpr int AT_UNCUT = 0x7fffffff;  // keys per item that no row is cut at: a row has fewer than 2^31

// The items: a row of n keys has max(1, ceil(n / C)) of them, as equal as multiples of AT_PIECE are; the last one ends with the row.
LA_HD inline int at_pieces(long long keys) {
  const long long n = (keys + AT_PIECE - 1) / AT_PIECE;
  return (int)(n < 1 ? 1 : n < 0xffffff ? n : 0xffffff) * AT_PIECE;
}
LA_HD inline int at_rows_items(int n, int C) { return n > C ? (int)(((unsigned)n + (unsigned)C - 1u) / (unsigned)C) : 1; }  // (n + C passes 31 bits)
LA_HD inline int at_item_keys(int n, int count) { return at_pieces(((unsigned)n + (unsigned)count - 1u) / (unsigned)count); }
LA_HD inline int at_item_end(const AtItem &it) { return it.index + 1 < it.count ? (it.index + 1) * it.C : it.n; }
// C.  `target` items of the same length are all resident at once.
//   Up to half as many rows: all keys over `target`, and longer while the rows' remainders make more items than are resident (AT_TURNS times at most).
//   More rows: where the longest row is longer than 5/4 of what a resident item would have of all keys, a third of the latter, so that what is left to the last items is little;
// otherwise rows are not cut.  us with items as for few rows / a half / a third / a quarter, 8 kv heads of 128 channels, rows from one position to n each: 48 rows, n = 4000 48 / 38 / 39 /
// 39, 64 rows, 4000 60 / 44 / 45 / 45, 64 rows, 30000 386 / 214 / 207 / 205, 256 rows, 4000 152 / 115 / 111 / 112; rows of 2000 each: 40 rows 79 / 65 / 65 / 71, 48 rows 84 / 82 / 76 / 82;
// 64 rows 89, cut 96 to 102; 96 rows 132, cut 142 to 183.
//   A row adds one item to its share of keys / C at most, so that there are B more than the keys over C: what at_plan makes room for.
constexpr int AT_TURNS = 3, AT_FINE = 3;
template <typename Items>
LA_HD inline int at_cut(int B, int target, long long keys, int longest, Items items) {
  if (2 * B > target) return longest * 4ll * target <= 5 * keys ? AT_UNCUT : at_pieces((keys + AT_FINE * target - 1) / (AT_FINE * target));
  int C = at_pieces((keys + target - 1) / target);
  for (int turn = 0; turn < AT_TURNS; ++turn) {
    const int n = items(C);
    if (n <= target) break;
    C = at_pieces((long long)C * n / target + 1);
  }
  return C;
}

// Workgroups for all keys together: as many as are resident at once, which goes by the registers that a head_dim takes.  512 or 1024 of them at 8 kv heads: 64 channels,
// 16 rows of 8000 56 / 48 us, 128 channels, 8 rows of 2048 19.3 / 21.9, 64 rows of 1000 47.8 / 52.5; 256: 22.5, 47.3, two rows of 131072 262 (512: 189, both without ONCE).
// A row of a cache of up to AT_WHOLE positions is not cut: the second launch costs more than the blocks of keys that a wave has left.  Cut / not, 8 kv heads of 128 channels:
// one row of 300 10.3 / 7.5, of 500 10.4 / 9.1, of 640 10.4 / 10.2, of 768 10.4 / 11.2, of 1000 10.5 / 13.6; 8 rows of 768 13.2 / 12.0, of 1000 13.7 / 15.0; 16 rows of 600
// 16.1 / 11.0; 64 rows of 768 38.9 / 35.3.
constexpr int AT_WHOLE = 768;
inline int at_workgroups(int dh) { return dh <= 64 ? 1024 : dh <= 128 ? 512 : 256; }
struct AtPlan {
  int target, items, tiles;
  size_t list, bytes;  // where the list of items begins in the workspace, 0: there is none
};
inline AtPlan at_plan(int head_dim, int n_kv_heads, int page_size, int Hq, int max_blocks, int B) {
  AtPlan r{};
  r.tiles = (Hq / n_kv_heads + AT_ROWS - 1) / AT_ROWS;
  const long long cap = (long long)max_blocks * page_size;
  r.items = B;
  if (cap > AT_WHOLE) {
    const int target = at_workgroups(head_dim) / (n_kv_heads * r.tiles);
    r.target = target > 1 ? target : 1;
    const long long cut = (2 * B > r.target ? (long long)AT_FINE : 1) * r.target + B, pieces = B * ((cap + AT_PIECE - 1) / AT_PIECE);
    r.items = (int)(cut < pieces ? cut : pieces);
    r.bytes = (size_t)r.items * Hq * (head_dim + 4) * 4;
    if (B > 64) {
      r.list = r.bytes;
      r.bytes += r.items * sizeof(AtItem) + (size_t)B * 4;
    }
  }
  return r;
}

}  // namespace la
