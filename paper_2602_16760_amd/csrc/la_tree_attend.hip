// Attention of trees of drafted tokens over the pages of their requests (la_paged_tree_attend).
#include "la_lanes.h"
#include "la_paged.h"

namespace la {

struct TreeAttend {
  const void *K, *V;  // of the layer
  int n_pages, page, Hkv, dh;
  const void *q;
  int64_t ldq;
  int Hq;
  float scale;
  const int32_t *table;
  int64_t ldt;
  int n_req, max_blocks;
  const int32_t *first, *len;
  const uint64_t *vis;
  int max_rows, B;
  void *out;
  int64_t ldo;
};

// A wave per row and query head; a lane a key for the scores, a lane four channels for the sums.
template <typename T>
__global__ __launch_bounds__(64) void tree_attend_simple_kernel(TreeAttend a) {
  const int i = blockIdx.x, head = blockIdx.y, lane = threadIdx.x, h = head / (a.Hq / a.Hkv);
  int lo = 0, hi = a.n_req;  // the last request that begins at or in front of the row
  while (hi - lo > 1) {
    const int m = (lo + hi) / 2;
    if (a.first[m] <= i) lo = m; else hi = m;
  }
  while (lo > 0 && a.first[lo] > i) --lo;
  const int r = lo, j = i - a.first[r];
  const bool in = j >= 0 && i < a.first[r + 1] && j < a.max_rows;
  const unsigned long long vis = in ? a.vis[i] : 0;
  const long long L = a.len[r], cap = (long long)a.max_blocks * a.page;
  const T *q = (const T *)a.q + i * a.ldq + (int64_t)head * a.dh;
  float o[4] = {0.f, 0.f, 0.f, 0.f}, m_run = -INFINITY, l = 0.f;
  const long long rows = a.first[r + 1] - a.first[r] < a.max_rows ? a.first[r + 1] - a.first[r] : a.max_rows;
  const long long n = vis && L >= 0 ? (L + rows < cap ? L + rows : cap) : 0;
  for (long long k0 = 0; k0 < n; k0 += 64) {
    const long long k = k0 + lane;
    bool seen = k < n && (k < L || (vis >> (k - L) & 1));
    long long at = 0;
    if (seen) {
      const int pg = a.table[r * a.ldt + k / a.page];
      seen = (unsigned)pg < (unsigned)a.n_pages;
      at = (((long long)pg * a.Hkv + h) * a.page + k % a.page) * a.dh;
    }
    float s = -INFINITY;
    if (seen) {
      s = 0.f;
      for (int c = 0; c < a.dh; ++c) s += load_as_float<T>(q + c) * load_as_float<T>((const T *)a.K + at + c);
      s *= a.scale;
    }
    float m = s;
    for (int x = 32; x > 0; x >>= 1) m = fmaxf(m, __shfl_xor(m, x, 64));
    m = fmaxf(m, m_run);
    const float base = m > -INFINITY ? m : 0.f, f = expf(m_run - base), p = seen ? expf(s - base) : 0.f;
    m_run = m;
    float sum = p;
    for (int x = 32; x > 0; x >>= 1) sum += __shfl_xor(sum, x, 64);
    l = l * f + sum;
    for (int x = 0; x < 4; ++x) o[x] *= f;
    for (int t = 0; t < 64; ++t) {
      const int s_t = __shfl((int)seen, t, 64);
      const float p_t = __shfl(p, t, 64);
      const long long at_t = __shfl(at, t, 64);
      if (!s_t) continue;
      for (int x = 0; x < 4; ++x)
        if (lane + 64 * x < a.dh) o[x] += p_t * load_as_float<T>((const T *)a.V + at_t + lane + 64 * x);
    }
  }
  for (int x = 0; x < 4; ++x)
    if (lane + 64 * x < a.dh) store_from_float<T>((T *)a.out + i * a.ldo + (int64_t)head * a.dh + lane + 64 * x, l > 0.f || l != l ? o[x] / l : 0.f);
}

}  // namespace la

using namespace la;

extern "C" size_t la_paged_tree_attend_workspace(const la_pages_desc *pages, int n_q_heads, int max_blocks, int n_requests, int max_rows) {
  if (check_pages(pages, 0) || n_q_heads < 1 || n_q_heads % pages->n_kv_heads || max_blocks < 1 || n_requests < 1 || max_rows < 1 || max_rows > LA_MAX_ROWS) return 0;
  return 0;
}

extern "C" int la_paged_tree_attend(const la_pages_desc *pages, int layer, const void *q, int64_t q_stride, int n_q_heads, float scale, const int32_t *table, int64_t table_stride,
                                    int n_requests, int max_blocks, const int32_t *first, const int32_t *len, const uint64_t *vis, int max_rows, int B, void *out,
                                    int64_t out_stride, void *workspace, size_t workspace_bytes, void *stream) {
  if (const int rc = check_pages(pages, layer)) return rc;
  const la_pages_desc &p = *pages;
  const size_t e = esize(&p);
  LA_REQUIRE(B >= 0, LA_EINVAL, "B=%d is negative", B);
  if (B == 0) return LA_OK;
  LA_REQUIRE(q && table && first && len && vis && out, LA_EINVAL, "NULL argument");
  LA_REQUIRE(n_q_heads > 0 && n_q_heads % p.n_kv_heads == 0, LA_EINVAL, "n_q_heads %d is not a multiple of n_kv_heads %d", n_q_heads, p.n_kv_heads);
  LA_REQUIRE(n_requests >= 1 && max_blocks >= 1 && (table_stride >= max_blocks || n_requests == 1), LA_EINVAL, "bad table dimensions");
  LA_REQUIRE((long long)max_blocks * p.page_size < (1ll << 31), LA_EINVAL, "%d blocks of %d positions: positions are 32-bit numbers", max_blocks, p.page_size);
  LA_REQUIRE(max_rows >= 1 && max_rows <= LA_MAX_ROWS, LA_EINVAL, "max_rows=%d outside [1, %d]", max_rows, LA_MAX_ROWS);
  LA_REQUIRE(B <= LA_MAX_ATTEND_ROWS && n_requests <= LA_MAX_ATTEND_ROWS && n_q_heads <= 65535, LA_EINVAL, "%d rows of %d requests and %d heads, at most %d of %d and 65535", B, n_requests,
             n_q_heads, LA_MAX_ATTEND_ROWS, LA_MAX_ATTEND_ROWS);
  LA_REQUIRE(aligned16({q, out}) && q_stride * e % 16 == 0 && out_stride * e % 16 == 0, LA_EINVAL, "q and out rows must be 16-byte aligned");
  LA_REQUIRE((uintptr_t)vis % 8 == 0, LA_EINVAL, "vis must be 8-byte aligned");
  LA_REQUIRE(scale - scale == 0.f, LA_EINVAL, "scale is not finite");
  (void)workspace, (void)workspace_bytes;
  hipStream_t s = (hipStream_t)stream;
  const size_t at = layer * layer_bytes(&p);
  const TreeAttend a{(const char *)p.k + at, (const char *)p.v + at, p.n_pages, p.page_size, p.n_kv_heads, p.head_dim, q, q_stride, n_q_heads, scale, table, table_stride,
                     n_requests, max_blocks, first, len, vis, max_rows, B, out, out_stride};
  ProfScope ps("tree_attend", s);
  const dim3 grid(B, n_q_heads);
  if (p.dtype == LA_F32) tree_attend_simple_kernel<float><<<grid, 64, 0, s>>>(a);
  else if (p.dtype == LA_F16) tree_attend_simple_kernel<_Float16><<<grid, 64, 0, s>>>(a);
  else tree_attend_simple_kernel<uint16_t><<<grid, 64, 0, s>>>(a);
  LA_HIP(hipGetLastError());
  return LA_OK;
}
