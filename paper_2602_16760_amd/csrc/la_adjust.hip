// What stands between stored logits and the choice of a token: penalties for tokens that occurred, biases, a grammar's mask (la_logits_adjust).
#include "la_device.h"
#include "la_internal.h"
#include "la_lanes.h"

namespace la {

// A workgroup per chunk of a row.  How often each of the chunk's tokens occurred is counted in LDS, from the request's committed tokens and those drafted on the row's path; then the
// logits pass once.  Counts are whole numbers and a token's biases are added in the list's order: results do not depend on the order of the atomics.
constexpr int ADJ_THREADS = 512, ADJ_PER = 16, ADJ_CHUNK = ADJ_THREADS * ADJ_PER;
constexpr unsigned ADJ_SEEN = 1u << 31, ADJ_BIASED = 1u << 30, ADJ_COUNT = ADJ_BIASED - 1;  // a token's word: occurred in the prompt; has a bias; times it was emitted

struct Adjust {
  const void *x;
  void *y;
  int64_t ldx, ldy;
  int B, V;
  la_adjust p;
};

template <typename T>
__device__ __forceinline__ T adjust_round(float f) {  // (float_to_bf16 takes finite numbers)
  if constexpr (sizeof(T) == 2 && !__is_same(T, _Float16)) return __builtin_bit_cast(uint16_t, (__bf16)f);
  else return (T)f;
}

template <typename T>
__global__ __launch_bounds__(ADJ_THREADS) void logits_adjust_kernel(Adjust a) {
  __shared__ unsigned word[ADJ_CHUNK];
  const int b = blockIdx.y, t = threadIdx.x, v0 = blockIdx.x * ADJ_CHUNK, n = a.V - v0 < ADJ_CHUNK ? a.V - v0 : ADJ_CHUNK;
  const la_adjust &p = a.p;
  const int r = p.req ? p.req[b] : b;
  const bool known = (unsigned)r < (unsigned)p.n_requests;
  auto setting = [&](const float *f, float off, bool positive) {  // (what is no number, or no factor, is off)
    const float v = f && known ? f[r] : off;
    return v - v == 0.f && (!positive || v > 0.f) ? v : off;
  };
  const float rho = setting(p.repetition, 1.f, true), beta = setting(p.presence, 0.f, false), alpha = setting(p.frequency, 0.f, false);
  const bool counts = rho != 1.f || beta != 0.f || alpha != 0.f, biases = known && p.n_bias > 0;
  if (counts || biases) {
    for (int i = t; i < ADJ_CHUNK; i += ADJ_THREADS) word[i] = 0;
    __syncthreads();
    if (counts && p.tokens) {
      const int32_t *tokens = p.tokens + r * p.tokens_stride;
      const int all = p.n_tokens[r] < p.max_tokens ? p.n_tokens[r] : p.max_tokens, prompt = p.n_prompt ? p.n_prompt[r] : 0;
      for (int i = t; i < all; i += ADJ_THREADS) {
        const int d = tokens[i], v = d - v0;
        if (d >= v0 && v < n) {
          if (i < prompt) atomicOr(&word[v], ADJ_SEEN);
          else atomicAdd(&word[v], 1u);
        }
      }
    }
    if (counts && p.draft && t > 0 && t < LA_MAX_ROWS && p.vis[b] >> t & 1) {  // (row 0 is the last of the committed tokens)
      const long long row = (long long)p.first[r] + t;
      const int d = row >= 0 && row < a.B ? p.draft[row] : -1, v = d - v0;
      if (d >= v0 && v < n) atomicAdd(&word[v], 1u);
    }
    if (biases)
      for (int i = t; i < p.n_bias; i += ADJ_THREADS) {
        const int d = p.bias_token[r * p.bias_stride + i], v = d - v0;
        if (d >= v0 && v < n) atomicOr(&word[v], ADJ_BIASED);
      }
    __syncthreads();
  }
  const uint32_t *allowed = nullptr;
  if (p.allowed) {
    const int m = p.allowed_index ? p.allowed_index[b] : b;
    if ((unsigned)m < (unsigned)p.n_allowed) allowed = p.allowed + m * p.allowed_stride;
  }
  const T *x = (const T *)a.x + b * a.ldx + v0;
  T *y = (T *)a.y + b * a.ldy + v0;
  for (int i = t; i < n; i += ADJ_THREADS) {
    float f = load_as_float<T>(x + i);
    const unsigned w = counts || biases ? word[i] : 0;
    const unsigned c = w & ADJ_COUNT;
    if (counts && w & (ADJ_SEEN | ADJ_COUNT)) f = f > 0.f ? f / rho : f * rho;
    if (counts && c) f = f - alpha * (float)c - beta;
    if (w & ADJ_BIASED)
      for (int k = 0; k < p.n_bias; ++k)
        if (p.bias_token[r * p.bias_stride + k] == v0 + i) f += p.bias[r * p.bias_stride + k];
    if (allowed && !(allowed[(v0 + i) >> 5] >> ((v0 + i) & 31) & 1)) f = -INFINITY;
    y[i] = adjust_round<T>(f);
  }
}

}  // namespace la

using namespace la;

extern "C" int la_logits_adjust(const void *logits, int dtype, int64_t row_stride, int B, int V, const la_adjust *how, void *out, int64_t out_stride, void *stream) {
  LA_REQUIRE(how != nullptr, LA_EINVAL, "NULL argument");
  LA_REQUIRE(B >= 0 && B <= 65535, LA_EINVAL, "B=%d outside [0, 65535]", B);
  if (B == 0) return LA_OK;
  const la_adjust &p = *how;
  LA_REQUIRE(logits && out, LA_EINVAL, "NULL argument");
  LA_REQUIRE(dtype == LA_F32 || dtype == LA_BF16 || dtype == LA_F16, LA_EINVAL, "unknown dtype %d", dtype);
  LA_REQUIRE(V >= 1 && V <= LA_MAX_SAMPLE_VOCAB, LA_EINVAL, "vocab %d outside [1, %d]", V, LA_MAX_SAMPLE_VOCAB);
  LA_REQUIRE((row_stride >= V && out_stride >= V) || B == 1, LA_EINVAL, "rows overlap");
  LA_REQUIRE(logits != out || row_stride == out_stride || B == 1, LA_EINVAL, "rows in place need one stride");
  LA_REQUIRE(p.n_requests >= 0 && p.max_tokens >= 0 && p.n_bias >= 0 && p.n_allowed >= 0, LA_EINVAL, "a size is negative");
  LA_REQUIRE(p.req || B <= p.n_requests || !(p.repetition || p.presence || p.frequency || p.tokens || p.draft || p.n_bias), LA_EINVAL, "%d rows for %d requests and no row map", B, p.n_requests);
  LA_REQUIRE(!p.tokens || (p.n_tokens && (p.tokens_stride >= p.max_tokens || p.n_requests <= 1)), LA_EINVAL, "tokens without their number, or rows of them that overlap");
  LA_REQUIRE(p.max_tokens <= LA_MAX_HISTORY, LA_EINVAL, "%d tokens of a request, at most %d", p.max_tokens, LA_MAX_HISTORY);
  LA_REQUIRE(!p.draft || (p.first && p.vis), LA_EINVAL, "drafted tokens without the rows' masks");
  LA_REQUIRE(!p.n_bias || (p.bias && p.bias_token && (p.bias_stride >= p.n_bias || p.n_requests <= 1)), LA_EINVAL, "biases without tokens, or rows of them that overlap");
  LA_REQUIRE(p.n_bias <= LA_MAX_BIAS, LA_EINVAL, "%d biases of a request, at most %d", p.n_bias, LA_MAX_BIAS);
  LA_REQUIRE(!p.allowed || ((p.allowed_stride >= (V + 31) / 32 || p.n_allowed <= 1) && (p.allowed_index || B <= p.n_allowed)), LA_EINVAL, "masks that overlap, or fewer than rows and no map");
  hipStream_t s = (hipStream_t)stream;
  const Adjust a{logits, out, row_stride, out_stride, B, V, p};
  ProfScope ps("logits_adjust", s);
  const dim3 grid(ceil_div(V, ADJ_CHUNK), B);
  if (dtype == LA_F32) logits_adjust_kernel<float><<<grid, ADJ_THREADS, 0, s>>>(a);
  else if (dtype == LA_F16) logits_adjust_kernel<_Float16><<<grid, ADJ_THREADS, 0, s>>>(a);
  else logits_adjust_kernel<uint16_t><<<grid, ADJ_THREADS, 0, s>>>(a);
  LA_HIP(hipGetLastError());
  return LA_OK;
}
