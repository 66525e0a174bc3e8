// A cache that several requests share: pages of page_size positions each, handed out per request.  Block tables and slot maps from the requests'
// lengths (la_page_map) and the rows' way into the pages (la_paged_write); the attention that reads them is in la_attend.hip.
#include <algorithm>

#include "la_lanes.h"
#include "la_paged.h"

namespace la {

// ---- block tables and slot maps ---------------------------------------------------------------------------
// Requests in order; request r grows from old[r] to new[r] positions (or shrinks).  With up(x) = ceil(x / page):
//   pages taken   take_r = max(0, up(new) - up(old)), from the ring's head on;  pages given back  give_r = max(0, up(old) - up(new)), behind its last free one
//   new tokens    add_r = max(0, new - old), rows first_r .. of the packed order, first = exclusive sum of add
// Everything else follows from the three exclusive sums over the requests in front.  Every workgroup forms them for its own few requests by reading all
// lengths (8 bytes a request, from L2): one launch and no words that workgroups pass to each other.  A row's page comes from the ring where the request took
// it in this call, not from the table, which another workgroup may be writing.
// Bytes do not bound it (48 requests in a step 1.3 KB, 512 requests in a turn with 400000 rows 4.9 MB = 0.9 us at a copy's rate): it is one chain of dependent steps, the
// lengths, the sums over a wave and over the waves, the row's request by bisection, its page.  4.4 us for the step, 7.2 for the turn.
constexpr int MAP_THREADS = 256;
struct PageMap {
  const int32_t *old_len, *new_len;
  int R, per_group, page;
  int32_t *table;
  int64_t ldt;
  int max_blocks;
  int32_t *ring;
  int n_pages;
  const int32_t *heads_in;
  int32_t *heads_out, *slot, *pos, *req;
  int max_rows;
  int32_t *first;
};

__global__ __launch_bounds__(MAP_THREADS) void page_map_kernel(PageMap a) {
  constexpr int WAVES = MAP_THREADS / 64;
  __shared__ long long red[WAVES][9], ends[3][MAP_THREADS];  // sums over waves; inclusive sums over the group's requests: rows, taken, given
  __shared__ int old_s[MAP_THREADS], had_s[MAP_THREADS], bad_s[WAVES];
  const int t = threadIdx.x, wave = t >> 6, lane = t & 63;
  const int r0 = (int)blockIdx.x * a.per_group, nr = a.R - r0 < a.per_group ? a.R - r0 : a.per_group;
  const int head = a.heads_in[0], n_free = a.heads_in[1];
  const long long cap = (long long)a.max_blocks * a.page;
  auto up = [&](int x) { return (int)(((unsigned)x + (unsigned)a.page - 1u) / (unsigned)a.page); };  // (x < 2^31, page < 2^31)
  // rows, taken and given pages of a request of which both lengths are in range
  auto steps = [&](int x, int y, long long (&v)[3]) {
    const int d = up(y) - up(x);
    v[0] = y > x ? y - x : 0;
    v[1] = d > 0 ? d : 0;
    v[2] = d < 0 ? -d : 0;
  };
  int x = 0, y = 0;
  if (t < nr) {
    x = a.old_len[r0 + t];
    y = a.new_len[r0 + t];
  }
  long long in_front[3] = {0, 0, 0}, total[3] = {0, 0, 0}, own[3];
  bool bad = false;
  for (int r = t; r < a.R; r += MAP_THREADS) {
    const int p = a.old_len[r], q = a.new_len[r];
    if (p < 0 || q < 0 || p > cap || q > cap) {
      bad = true;
      continue;
    }
    long long v[3];
    steps(p, q, v);
#pragma unroll
    for (int i = 0; i < 3; ++i) {
      total[i] += v[i];
      if (r < r0) in_front[i] += v[i];
    }
  }
  steps(x < 0 ? 0 : x, y < 0 ? 0 : y, own);  // (nothing is done with what is out of range)
  old_s[t] = x;
  had_s[t] = up(x < 0 ? 0 : x);
  const unsigned long long bads = __ballot(bad);
#pragma unroll
  for (int i = 0; i < 3; ++i) {
    own[i] = lane_through(own[i]);
    const long long f = lane_through(in_front[i]), s = lane_through(total[i]);
    if (lane == 63) {
      red[wave][i] = f;
      red[wave][3 + i] = s;
      red[wave][6 + i] = own[i];
    }
  }
  if (lane == 0) bad_s[wave] = bads != 0;
  __syncthreads();
  bool any_bad = false;
#pragma unroll
  for (int i = 0; i < 3; ++i) {
    in_front[i] = total[i] = 0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
      in_front[i] += red[w][i];
      total[i] += red[w][3 + i];
      if (w < wave) own[i] += red[w][6 + i];
    }
    ends[i][t] = own[i];
  }
#pragma unroll
  for (int w = 0; w < WAVES; ++w) any_bad = any_bad || bad_s[w];
  __syncthreads();
  int error = 0;
  if (head < 0 || head >= a.n_pages || n_free < 0 || n_free > a.n_pages) error = 4;
  else if (any_bad) error = 3;
  else if (total[2] > a.n_pages - n_free) error = 4;  // (pages given back that the ring has already)
  else if (total[0] > a.max_rows) error = 2;
  else if (total[1] > n_free) error = 1;
  const int part = blockIdx.y, parts = gridDim.y, stride = parts * MAP_THREADS, k0 = part * MAP_THREADS + t;
  if (part == 0) {
    if (t < nr) a.first[r0 + t] = error ? 0 : (int)(in_front[0] + (t > 0 ? ends[0][t - 1] : 0));
    if (blockIdx.x == 0 && t == 0) {
      a.first[a.R] = error ? 0 : (int)total[0];
      a.heads_out[0] = error ? head : (int)((head + total[1]) % a.n_pages);
      a.heads_out[1] = error ? n_free : (int)(n_free - total[1] + total[2]);
      a.heads_out[2] = error ? 0 : (int)total[0];
      a.heads_out[3] = error;
    }
  }
  // rows that no token has
  const long long grid_t = ((long long)blockIdx.y * gridDim.x + blockIdx.x) * MAP_THREADS + t, grid_n = (long long)gridDim.x * parts * MAP_THREADS;
  for (long long i = (error ? 0 : total[0]) + grid_t; i < a.max_rows; i += grid_n) a.slot[i] = a.pos[i] = a.req[i] = -1;
  if (error) return;
  auto find = [&](const long long *e, long long k) {  // first request of the group whose sum is above k
    int lo = 0, hi = nr - 1;
    while (lo < hi) {
      const int m = (lo + hi) / 2;
      if (e[m] > k) hi = m; else lo = m + 1;
    }
    return lo;
  };
  auto taken = [&](int q, int block) {  // the page that request r0 + q takes for a block behind those it had
    const long long k = in_front[1] + (q > 0 ? ends[1][q - 1] : 0) + (block - had_s[q]);
    return a.ring[(head + k) % a.n_pages];
  };
  const long long n_take = ends[1][nr - 1], n_give = ends[2][nr - 1], n_rows = ends[0][nr - 1];
  for (long long k = k0; k < n_take; k += stride) {
    const int q = find(ends[1], k), block = had_s[q] + (int)(k - (q > 0 ? ends[1][q - 1] : 0));
    a.table[(r0 + q) * a.ldt + block] = taken(q, block);
  }
  for (long long k = k0; k < n_give; k += stride) {
    const int q = find(ends[2], k), block = had_s[q] - (int)(ends[2][q] - k);  // (blocks up(new) .. up(old) - 1, in order)
    a.ring[(head + n_free + in_front[2] + k) % a.n_pages] = a.table[(r0 + q) * a.ldt + block];
  }
  for (long long k = k0; k < n_rows; k += stride) {
    const int q = find(ends[0], k), p = old_s[q] + (int)(k - (q > 0 ? ends[0][q - 1] : 0)), block = p / a.page;
    const int page = block < had_s[q] ? a.table[(r0 + q) * a.ldt + block] : taken(q, block);
    const long long i = in_front[0] + k;
    a.slot[i] = (unsigned)page < (unsigned)a.n_pages ? page * a.page + (p - block * a.page) : -1;
    a.pos[i] = p;
    a.req[i] = r0 + q;
  }
}

// ---- rows into pages ------------------------------------------------------------------------------------------
// Pages are [page][kv head][place][channel]: what one head has in a page is contiguous, so that the attention reads whole lines.  Thread per 16 bytes of K and of V.
// Bound by the copy's bytes: 16000 rows of 8 heads of 128 f16 channels, 131 MB read and written, 26 us with new rows every time (5.0 TB/s; a large copy reaches 5.2), 20 with the same ones, part of
// which the last-level cache holds; 64 rows 2.6 us.
__global__ __launch_bounds__(256) void paged_write_kernel(uint4 *kp, uint4 *vp, const uint4 *k, const uint4 *v, int64_t ldk, int64_t ldv, const int32_t *slot, int n, int Hkv,
                                                          int per_head, int page, int n_pages) {
  const int per_row = Hkv * per_head;
  const long long i = (long long)blockIdx.x * 256 + threadIdx.x;
  if (i >= (long long)n * per_row) return;
  const int row = (int)(i / per_row), c = (int)(i - (long long)row * per_row), h = c / per_head;
  const int s = slot[row], pg = s / page;
  if (s < 0 || pg >= n_pages) return;
  const size_t to = (((size_t)pg * Hkv + h) * page + (s - pg * page)) * per_head + (c - h * per_head);
  kp[to] = k[row * ldk + c];
  vp[to] = v[row * ldv + c];
}

// ---- slots to other slots, in every layer ---------------------------------------------------------------------
// A thread takes 16 bytes of a kv head of the rows of one run, of K or V of one layer after the other: it has read all of a run's sources before it writes one of its destinations, and
// nobody else has to do with those bytes, so a run may move rows onto each other's places.  RUN sources wait in registers: the next larger of 1, 4, 8, 16 and 64 (of 64 with their places they are
// all 512 that a lane can have and 20 bytes of scratch memory: a path of 16 rows of one request in 32 layers 6.3 us, of 17 14.9, of 63 19.9).  Places that a run does
// not have are read from row 0 and thrown away, since a condition on each load sent the array to scratch memory (64 paths of 12: 154 us against 27).
// Bound by bandwidth: one fork of 1000 positions in 32 layers, 262 MB, 50.2 us = 5.2 TB/s, as a large copy; paths of up to 6 rows of 32 requests in 32 layers, 21 MB, 6.4 (the kernel; 8.0 a launch of a graph), are one chain of index and row.  Up to
// 32 workgroups share the layers' K and V (a launch with 8, 16, 32, 64 of them: paths 11.2, 8.8, 8.1, 8.4; fork 53.9, 52.1, 51.5, 51.8), each with one layer's row in flight: unrolled over its layers
// the fork took 83.
struct PagedCopy {
  uint4 *k, *v;  // of the first layer
  size_t layer;  // 16-byte pieces of one
  int layers, Hkv, per_head, page, n_pages, shift;  // shift: page_size is 2^shift, -1: no power of two
  const int32_t *from, *to;
  int n, run;
};
template <int RUN>
__global__ __launch_bounds__(256) void paged_copy_kernel(PagedCopy a) {
  const int h = blockIdx.y;
  const long long i = (long long)blockIdx.x * 256 + threadIdx.x;
  const int r = (int)(i / a.per_head), c = (int)(i - (long long)r * a.per_head);
  if ((long long)r * a.run >= a.n) return;
  const int n_slots = a.n_pages * a.page;
  long long src[RUN], dst[RUN];
#pragma unroll
  for (int j = 0; j < RUN; ++j) {
    const long long m = (long long)r * a.run + j;
    const bool in = j < a.run && m < a.n;
    const int s = in ? a.from[m] : -1, d = in ? a.to[m] : -1;
    const bool moves = (unsigned)s < (unsigned)n_slots && (unsigned)d < (unsigned)n_slots;
    auto at = [&](int slot) {
      const int pg = a.shift >= 0 ? slot >> a.shift : slot / a.page;
      return (((long long)pg * a.Hkv + h) * a.page + (slot - pg * a.page)) * a.per_head + c;
    };
    src[j] = moves ? at(s) : -1;
    dst[j] = moves ? at(d) : -1;
  }
  for (int l = blockIdx.z; l < 2 * a.layers; l += gridDim.z) {
    typedef unsigned __attribute__((ext_vector_type(4))) piece;
    piece *p = (piece *)((l & 1 ? a.v : a.k) + (l >> 1) * a.layer), x[RUN];
#pragma unroll
    for (int j = 0; j < RUN; ++j) x[j] = p[src[j] >= 0 ? src[j] : 0];  // (no condition around the loads: all are on their way at once)
#pragma unroll
    for (int j = 0; j < RUN; ++j)
      if (src[j] >= 0) p[dst[j]] = x[j];
  }
}

int check_pages(const la_pages_desc *p, int layer) {
  LA_REQUIRE(p && p->k && p->v, LA_EINVAL, "NULL pages");
  LA_REQUIRE(p->n_layers > 0 && p->n_pages > 0 && p->page_size > 0 && p->n_kv_heads > 0, LA_EINVAL, "page dimensions must be positive");
  LA_REQUIRE(p->head_dim > 0 && p->head_dim % 8 == 0 && p->head_dim <= 256, LA_EINVAL, "head_dim %d must be a multiple of 8, at most 256", p->head_dim);
  LA_REQUIRE(p->dtype == LA_F32 || p->dtype == LA_BF16 || p->dtype == LA_F16, LA_EINVAL, "unknown dtype %d", p->dtype);
  LA_REQUIRE((long long)p->n_pages * p->page_size < (1ll << 31), LA_EINVAL, "%d pages of %d positions: slots are 32-bit numbers", p->n_pages, p->page_size);
  LA_REQUIRE(aligned16({p->k, p->v}), LA_EINVAL, "pages must be 16-byte aligned");
  LA_REQUIRE(layer >= 0 && layer < p->n_layers, LA_ERANGE, "layer %d outside the pages' %d layers", layer, p->n_layers);
  return LA_OK;
}

}  // namespace la

using namespace la;

extern "C" int la_page_map(const int32_t *old_len, const int32_t *new_len, int R, int page_size, int32_t *table, int64_t table_stride, int max_blocks,
                           int32_t *ring, int n_pages, const int32_t *heads_in, int32_t *heads_out, int32_t *slot, int32_t *pos, int32_t *req, int max_rows,
                           int32_t *first, void *stream) {
  LA_REQUIRE(old_len && new_len && table && ring && heads_in && heads_out && slot && pos && req && first, LA_EINVAL, "NULL argument");
  LA_REQUIRE(heads_in != heads_out, LA_EINVAL, "heads_out must not be heads_in: every workgroup reads the one while one writes the other");
  LA_REQUIRE(R >= 1 && page_size >= 1 && max_blocks >= 1 && n_pages >= 1 && max_rows >= 1, LA_EINVAL, "dimensions must be positive");
  LA_REQUIRE(R <= 1 << 30, LA_EINVAL, "R=%d requests, at most 2^30", R);  // (a thread's next request is a 32-bit number too)
  LA_REQUIRE(table_stride >= max_blocks || R == 1, LA_EINVAL, "table rows overlap");
  LA_REQUIRE((long long)n_pages * page_size < (1ll << 31), LA_EINVAL, "%d pages of %d positions: slots are 32-bit numbers", n_pages, page_size);
  hipStream_t s = (hipStream_t)stream;
  // 16 requests a workgroup (more where there are very many, each of which reads all lengths), in as many parts as give a thread two rows.  Rows a thread, us of the turn
  // above: 1 9.1, 2 7.2, 4 7.3, 8 9.0.
  int per_group = 16;
  while (per_group < MAP_THREADS && R / per_group > 64) per_group *= 2;
  const int groups = ceil_div(R, per_group), parts = (int)std::min(64ll, std::max(1ll, max_rows / (groups * MAP_THREADS * 2ll)));
  const PageMap a{old_len, new_len, R, per_group, page_size, table, table_stride, max_blocks, ring, n_pages, heads_in, heads_out, slot, pos, req, max_rows, first};
  ProfScope ps("page_map", s);
  page_map_kernel<<<dim3(groups, parts), MAP_THREADS, 0, s>>>(a);
  LA_HIP(hipGetLastError());
  return LA_OK;
}

extern "C" int la_paged_write(const la_pages_desc *pages, int layer, const void *k, const void *v, int64_t k_stride, int64_t v_stride, const int32_t *slot, int n,
                              void *stream) {
  if (const int rc = check_pages(pages, layer)) return rc;
  const la_pages_desc &p = *pages;
  const size_t e = esize(&p);
  LA_REQUIRE(n >= 0, LA_EINVAL, "n=%d is negative", n);
  if (n == 0) return LA_OK;
  LA_REQUIRE(k && v && slot, LA_EINVAL, "NULL argument");
  LA_REQUIRE(aligned16({k, v}) && k_stride * e % 16 == 0 && v_stride * e % 16 == 0, LA_EINVAL, "K and V rows must be 16-byte aligned");
  hipStream_t s = (hipStream_t)stream;
  const int per_head = (int)(p.head_dim * e / 16);
  const long long wgs = ((long long)n * p.n_kv_heads * per_head + 255) / 256;
  LA_REQUIRE(wgs < (1ll << 24), LA_EINVAL, "%d rows are more than one launch takes", n);  // (2^32 threads)
  ProfScope ps("paged_write", s);
  paged_write_kernel<<<(unsigned)wgs, 256, 0, s>>>((uint4 *)((char *)p.k + layer * layer_bytes(&p)), (uint4 *)((char *)p.v + layer * layer_bytes(&p)), (const uint4 *)k,
                                                   (const uint4 *)v, k_stride * (int64_t)e / 16, v_stride * (int64_t)e / 16, slot, n, p.n_kv_heads, per_head, p.page_size,
                                                   p.n_pages);
  LA_HIP(hipGetLastError());
  return LA_OK;
}

extern "C" int la_paged_copy(const la_pages_desc *pages, int layer_begin, int layer_end, const int32_t *from, const int32_t *to, int n, int run, void *stream) {
  if (const int rc = check_pages(pages, 0)) return rc;
  const la_pages_desc &p = *pages;
  LA_REQUIRE(layer_begin >= 0 && layer_begin <= layer_end && layer_end <= p.n_layers, LA_ERANGE, "layers [%d, %d) outside the pages' %d layers", layer_begin, layer_end, p.n_layers);
  LA_REQUIRE(n >= 0, LA_EINVAL, "n=%d is negative", n);
  LA_REQUIRE(run >= 1 && run <= LA_MAX_ROWS, LA_EINVAL, "run=%d outside [1, %d]", run, LA_MAX_ROWS);
  if (n == 0 || layer_begin == layer_end) return LA_OK;
  LA_REQUIRE(from && to, LA_EINVAL, "NULL argument");
  LA_REQUIRE(p.n_kv_heads <= 65535, LA_EINVAL, "%d kv heads are more than one launch takes", p.n_kv_heads);
  const size_t e = esize(&p);
  const int per_head = (int)(p.head_dim * e / 16);
  const long long runs = ((long long)n + run - 1) / run, wgs = (runs * per_head + 255) / 256;
  const int layers = layer_end - layer_begin, z = std::min(2 * layers, 32);
  LA_REQUIRE(wgs * p.n_kv_heads < 1ll << 24, LA_EINVAL, "%d rows of %d kv heads are more than one launch takes", n, p.n_kv_heads);
  const size_t layer = layer_bytes(&p);
  const PagedCopy a{(uint4 *)((char *)p.k + layer_begin * layer), (uint4 *)((char *)p.v + layer_begin * layer), layer / 16, layers, p.n_kv_heads, per_head, p.page_size, p.n_pages,
                    (p.page_size & (p.page_size - 1)) == 0 ? __builtin_ctz(p.page_size) : -1, from, to, n, run};
  hipStream_t s = (hipStream_t)stream;
  ProfScope ps("paged_copy", s);
  const dim3 grid((unsigned)wgs, p.n_kv_heads, z);
  if (run == 1) paged_copy_kernel<1><<<grid, 256, 0, s>>>(a);
  else if (run <= 4) paged_copy_kernel<4><<<grid, 256, 0, s>>>(a);
  else if (run <= 8) paged_copy_kernel<8><<<grid, 256, 0, s>>>(a);
  else if (run <= 16) paged_copy_kernel<16><<<grid, 256, 0, s>>>(a);
  else paged_copy_kernel<64><<<grid, 256, 0, s>>>(a);
  LA_HIP(hipGetLastError());
  return LA_OK;
}
