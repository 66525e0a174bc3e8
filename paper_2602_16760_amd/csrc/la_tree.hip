// Trees of drafted tokens, one behind the committed positions of each request: where their rows stand and what they see (la_tree_layout), and which path a step commits
// (la_tree_accept).  The attention of their rows is in la_tree_attend.hip.
#include "la_device.h"
#include "la_internal.h"
#include "la_lanes.h"

namespace la {

constexpr int TREE_WAVES = 4;  // requests of a workgroup

// A request's rows: the first one's number and how many a mask has bits for.  What is outside [0, B) is no row.
struct TreeRows {
  long long first;
  int n;
};
__device__ __forceinline__ TreeRows tree_rows(const int32_t *first, int r, int B) {
  const long long f = first[r], e = first[r + 1], n = (e < B ? e : B) - f;
  return {f, f < 0 || n < 0 ? 0 : n < LA_MAX_ROWS ? (int)n : LA_MAX_ROWS};
}

// Masks.  vis_j = 2^j | vis_parent(j): a lane a row, and with every turn each row takes over what the row that it has come up to has gathered, so that six turns gather all 64; a
// row's depth is the number of bits but its own.  Rows without a way to row 0 lack bit 0.  A wave a request, no words that waves pass to each other: bound by the launch, 1.7 us for one tree of
// eight rows, 2.8 for 512 of 1 to 64 (6.5 and 6.6 with the call).  Four waves a workgroup: at 512 requests that is 128 workgroups, a wave on every other SIMD.
__global__ __launch_bounds__(64 * TREE_WAVES) void tree_layout_kernel(const int32_t *parent, const int32_t *first, const int32_t *len, int R, int B, int32_t *pos, uint64_t *vis) {
  const int lane = threadIdx.x & 63, r = uniform((int)(blockIdx.x * TREE_WAVES + (threadIdx.x >> 6)));
  if (r < R) {
    const TreeRows rows = tree_rows(first, r, B);
    const int L = len[r];
    const int p = lane < rows.n ? parent[rows.first + lane] : -1;
    int up = p >= 0 && p < lane ? p : lane;
    unsigned long long mask = 1ull << lane;
#pragma unroll
    for (int turn = 0; turn < 6; ++turn) {
      mask |= __shfl(mask, up, 64);
      up = __shfl(up, up, 64);
    }
    if (lane < rows.n) {
      const bool rooted = mask & 1;
      pos[rows.first + lane] = rooted ? L + (int)__popcll(mask) - 1 : -1;
      vis[rows.first + lane] = rooted ? mask : 0;
    }
    const long long end = first[r + 1] < B ? first[r + 1] : B;
    for (long long i = rows.first + LA_MAX_ROWS + lane; rows.first >= 0 && i < end; i += 64) {  // (rows that no mask has a bit for)
      pos[i] = -1;
      vis[i] = 0;
    }
  }
  // rows of no request
  const long long t = (long long)blockIdx.x * 64 * TREE_WAVES + threadIdx.x, threads = (long long)gridDim.x * 64 * TREE_WAVES;
  const long long front = first[0] < B ? first[0] : B, back = first[R] > 0 ? first[R] : 0;
  for (long long i = t; i < front; i += threads) {
    pos[i] = -1;
    vis[i] = 0;
  }
  for (long long i = back + t; i < B; i += threads) {
    pos[i] = -1;
    vis[i] = 0;
  }
}

// The path: from row 0 on to the first row that hangs on the present one and holds the token that the present one chose.  A wave a request, a lane a row: a step is one
// ballot and three scalar reads of what the lanes hold, so a path of 63 drafts costs no more memory than one.  Bound by the launch and by the chain of a request's reads (first, then its rows): 1.9 us
// for one tree of eight rows, 4.1 for 512 of 1 to 64 (9.0 and 9.2 with the call).
struct TreeAccept {
  const int32_t *parent, *tok, *ids, *slot, *first, *len, *limit;
  int R, B, max_path;
  int32_t *n_new, *new_len, *last, *out, *from, *to;
};
__global__ __launch_bounds__(64 * TREE_WAVES) void tree_accept_kernel(TreeAccept a) {
  const int lane = threadIdx.x & 63, r = uniform((int)(blockIdx.x * TREE_WAVES + (threadIdx.x >> 6)));
  if (r >= a.R) return;
  const TreeRows rows = tree_rows(a.first, r, a.B);
  const int L = a.len[r], limit = a.limit ? a.limit[r] : LA_MAX_ROWS, most = uniform(limit < a.max_path ? limit : a.max_path);
  const bool there = lane < rows.n;
  const long long i = rows.first + (there ? lane : 0);
  const int parent = there ? a.parent[i] : -1, tok = there ? a.tok[i] : -1, id = there ? a.ids[i] : -1, slot = there ? a.slot[i] : -1;
  int row = 0, moved = 0, n_new = 0, at = 0;  // of lane k: the path's k-th row
  if (rows.n > 0 && most > 0) {
    for (;;) {
      const int chosen = lane_value(id, at);
      if (lane == moved) row = at;
      ++moved;
      if (chosen < 0) break;
      if (++n_new == most) break;
      const unsigned long long next = __ballot(lane > at && parent == at && tok == chosen);  // (a lane without a row has no parent)
      if (!next) break;
      at = __builtin_ctzll(next);
    }
  }
  const int from_id = __shfl(id, row, 64), from_slot = __shfl(slot, row, 64);
  if (lane < a.max_path) {
    const size_t to = (size_t)r * a.max_path + lane;
    const bool moves = lane < moved && row != lane && from_slot >= 0 && slot >= 0;
    a.out[to] = lane < n_new ? from_id : -1;
    a.from[to] = moves ? from_slot : -1;
    a.to[to] = moves ? slot : -1;
  }
  if (lane == 0) {
    a.n_new[r] = n_new;
    a.new_len[r] = L + moved;
    a.last[r] = moved ? (int)(rows.first + at) : -1;
  }
}

}  // namespace la

using namespace la;

extern "C" int la_tree_layout(const int32_t *parent, const int32_t *first, const int32_t *len, int R, int B, int32_t *pos, uint64_t *vis, void *stream) {
  LA_REQUIRE(R >= 0 && R <= LA_MAX_ATTEND_ROWS && B >= 0 && B <= LA_MAX_ATTEND_ROWS, LA_EINVAL, "R=%d requests of B=%d rows, each 0 to %d", R, B, LA_MAX_ATTEND_ROWS);
  if (B == 0) return LA_OK;
  LA_REQUIRE(parent && first && len && pos && vis, LA_EINVAL, "NULL argument");
  LA_REQUIRE(R >= 1, LA_EINVAL, "%d rows of no request", B);
  LA_REQUIRE((uintptr_t)vis % 8 == 0, LA_EINVAL, "vis must be 8-byte aligned");
  hipStream_t s = (hipStream_t)stream;
  ProfScope ps("tree_layout", s);
  tree_layout_kernel<<<ceil_div(R, TREE_WAVES), 64 * TREE_WAVES, 0, s>>>(parent, first, len, R, B, pos, vis);
  LA_HIP(hipGetLastError());
  return LA_OK;
}

extern "C" int la_tree_accept(const int32_t *parent, const int32_t *tok, const int32_t *ids, const int32_t *slot, const int32_t *first, const int32_t *len, const int32_t *limit, int R,
                              int B, int max_path, int32_t *n_new, int32_t *new_len, int32_t *last, int32_t *out, int32_t *from, int32_t *to, void *stream) {
  LA_REQUIRE(R >= 0 && R <= LA_MAX_ATTEND_ROWS && B >= 0 && B <= LA_MAX_ATTEND_ROWS, LA_EINVAL, "R=%d requests of B=%d rows, each 0 to %d", R, B, LA_MAX_ATTEND_ROWS);
  LA_REQUIRE(max_path >= 1 && max_path <= LA_MAX_ROWS, LA_EINVAL, "max_path=%d outside [1, %d]", max_path, LA_MAX_ROWS);
  if (R == 0) return LA_OK;
  LA_REQUIRE(first && len && n_new && new_len && last && out && from && to, LA_EINVAL, "NULL argument");
  LA_REQUIRE(B == 0 || (parent && tok && ids && slot), LA_EINVAL, "NULL argument");
  hipStream_t s = (hipStream_t)stream;
  ProfScope ps("tree_accept", s);
  tree_accept_kernel<<<ceil_div(R, TREE_WAVES), 64 * TREE_WAVES, 0, s>>>(TreeAccept{parent, tok, ids, slot, first, len, limit, R, B, max_path, n_new, new_len, last, out, from, to});
  LA_HIP(hipGetLastError());
  return LA_OK;
}
