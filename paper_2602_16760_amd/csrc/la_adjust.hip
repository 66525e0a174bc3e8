// What stands between stored logits and the choice of a token: penalties for tokens that occurred, biases, a grammar's mask (la_logits_adjust).
#include <type_traits>

#include "la_device.h"
#include "la_internal.h"
#include "la_lanes.h"

namespace la {

// A workgroup per chunk of a row.  How often each of the chunk's tokens occurred is counted in LDS, from the request's committed tokens and those drafted on the row's path; then the
// logits, requested before, pass once.  Counts are whole numbers and a token's biases are added in the list's order: results do not depend on the order of the atomics, nor on the chunks.
// Bound by a chain (settings, history, LDS, division) at few rows, 4.8 us for one of 32768; by the bytes and that chain at many: 64 rows of 131072, 67.6 MB, 8192 tokens of history each, 19.2 us =
// 3.5 TB/s, all workgroups resident and in step (64 registers; with 67 a fourth workgroup did not fit a CU: 22.4).  16 bytes at a time wherever a row begins: 64 rows of 100001 in bfloat16, rows
// at every second byte, 15 us, as rows of 100000; element by element 23, and without asking for all of them first 50.
// 300 biases for nine rows of 1731: 6.2 us; as a search through the list by each token that has one 80.
constexpr int ADJ_THREADS = 512;
constexpr int ADJ_PER = 16, ADJ_PER_SHORT = 4;  // tokens of a thread: chunks of 8192 and of 2048
constexpr int ADJ_FEW = 1024;                   // short chunks of a launch at most
constexpr unsigned ADJ_SEEN = 1u << 31, ADJ_COUNT = ADJ_SEEN - 1;  // a token's word: occurred in the prompt; times it was emitted

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

template <typename T, int PER>
__global__ __launch_bounds__(ADJ_THREADS, 8) void logits_adjust_kernel(Adjust a) {
  constexpr int CHUNK = ADJ_THREADS * PER, G = 16 / (int)sizeof(T) < PER ? 16 / (int)sizeof(T) : PER, GROUPS = PER / G;  // tokens of a group; groups of a thread
  typedef T __attribute__((ext_vector_type(G), aligned(sizeof(T)))) group;  // (rows begin at any number)
  __shared__ __attribute__((aligned(16))) unsigned word[CHUNK];
  __shared__ __attribute__((aligned(16))) unsigned seen[3 * CHUNK / 32];  // a bit a token: has a bias; has more than one, or one of an earlier turn; its word is its logit with biases
  __shared__ int entry[ADJ_THREADS];
  __shared__ float entry_bias[ADJ_THREADS];
  unsigned *twice = seen + CHUNK / 32, *done = twice + CHUNK / 32;
  const int b = blockIdx.y, t = threadIdx.x, v0 = blockIdx.x * CHUNK, n = a.V - v0 < CHUNK ? a.V - v0 : CHUNK;
  const la_adjust &p = a.p;
  const T *x = (const T *)a.x + b * a.ldx + v0;
  T *y = (T *)a.y + b * a.ldy + v0;
  // token i of group j is j * ADJ_THREADS * G + t * G + i of the chunk
  T in[GROUPS][G];
#pragma unroll
  for (int j = 0; j < GROUPS; ++j) {
    const int at = (j * ADJ_THREADS + t) * G;
    if (at + G <= n) {
      const group v = *(const group *)(x + at);
#pragma unroll
      for (int i = 0; i < G; ++i) in[j][i] = v[i];
    } else {
#pragma unroll
      for (int i = 0; i < G; ++i) in[j][i] = x[at + i < n ? at + i : 0];
    }
  }
  const int r = uniform(p.req ? p.req[b] : b);
  const bool known = (unsigned)r < (unsigned)p.n_requests;
  unsigned mask = ~0u;  // a group's bits are those from bit j G on
  if (p.allowed) {
    const int m = uniform(p.allowed_index ? p.allowed_index[b] : b);
    if ((unsigned)m < (unsigned)p.n_allowed) {
      const uint32_t *allowed = p.allowed + m * p.allowed_stride;
      mask = 0;
#pragma unroll
      for (int j = 0; j < GROUPS; ++j) {
        const int at = v0 + (j * ADJ_THREADS + t) * G;
        mask |= (allowed[(at < a.V ? at : 0) >> 5] >> (at & 31) & ((1u << G) - 1)) << (j * G);  // (a group lies in one word)
      }
    }
  }
  auto setting = [&](const float *f, float off, bool positive) {  // (what is no number, or no factor, is off)
    const float v = f && known ? f[r] : off;
    return __uint_as_float(uniform((int)__float_as_uint(v - v == 0.f && (!positive || v > 0.f) ? v : off)));
  };
  const float rho = setting(p.repetition, 1.f, true), beta = setting(p.presence, 0.f, false), alpha = setting(p.frequency, 0.f, false);
  const bool counts = rho != 1.f || beta != 0.f || alpha != 0.f, biases = known && p.n_bias > 0;
  if (uniform(counts || biases)) {
    for (int i = 4 * t; i < CHUNK; i += 4 * ADJ_THREADS) *(uint4 *)(word + i) = uint4{0, 0, 0, 0};
    if (biases)
      for (int i = t; i < 3 * CHUNK / 32; i += ADJ_THREADS) seen[i] = 0;
    __syncthreads();
    if (counts && p.tokens) {
      const int32_t *tokens = p.tokens + r * p.tokens_stride;
      const int all = p.n_tokens[r] < p.max_tokens ? p.n_tokens[r] : p.max_tokens, prompt = p.n_prompt ? p.n_prompt[r] : 0;
      constexpr int N = 8;
      for (int i0 = t; i0 < all; i0 += N * ADJ_THREADS) {
        int d[N];
#pragma unroll
        for (int k = 0; k < N; ++k) d[k] = tokens[i0 + k * ADJ_THREADS < all ? i0 + k * ADJ_THREADS : i0];
#pragma unroll
        for (int k = 0; k < N; ++k) {
          const int i = i0 + k * ADJ_THREADS, v = d[k] - v0;
          if (i >= all || d[k] < v0 || v >= n) continue;
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
    __syncthreads();
  }
  auto penalized = [&](float f, unsigned w) {
    const unsigned c = w & ADJ_COUNT;
    if (counts && w & (ADJ_SEEN | ADJ_COUNT)) f = f > 0.f ? f / rho : f * rho;
    return counts && c ? f - alpha * (float)c - beta : f;
  };
  // Biases, a turn of the threads with an entry of the list each: the first entry's thread of a token adds them all to its logit, in the list's order, and leaves the sum in the token's word.
  // Only where a token's bit was set before can there be more of them to look for.
#pragma unroll 1
  for (int i0 = 0; biases && i0 < p.n_bias; i0 += ADJ_THREADS) {
    const int i = i0 + t, left = p.n_bias - i0 < ADJ_THREADS ? p.n_bias - i0 : ADJ_THREADS;
    const int d = t < left ? p.bias_token[r * p.bias_stride + i] : -1, v = d >= v0 && d - v0 < n ? d - v0 : -1;
    const unsigned bit = 1u << (v & 31);
    float logit = 0.f, bias = 0.f;
    if (v >= 0) {
      bias = p.bias[r * p.bias_stride + i];
      logit = load_as_float<T>(x + v);  // (nobody writes before the last turn)
      if (atomicOr(&seen[v >> 5], bit) & bit) atomicOr(&twice[v >> 5], bit);
    }
    entry[t] = v;
    entry_bias[t] = bias;
    __syncthreads();
    if (v >= 0) {
      const bool more = twice[v >> 5] & bit;
      bool own = true;
#pragma unroll 4
      for (int k = 0; more && k < t; ++k) own = own && entry[k] != v;
      if (own) {
        float f = (done[v >> 5] & bit ? __uint_as_float(word[v]) : penalized(logit, word[v])) + bias;
#pragma unroll 4
        for (int k = t + 1; more && k < left; ++k)
          if (entry[k] == v) f += entry_bias[k];
        word[v] = __float_as_uint(f);
        atomicOr(&done[v >> 5], bit);
      }
    }
    __syncthreads();
  }
#pragma unroll
  for (int j = 0; j < GROUPS; ++j) {
    const int at = (j * ADJ_THREADS + t) * G;
    if (at >= n) continue;
    T out[G];
    const unsigned biased = biases ? done[at >> 5] >> (at & 31) : 0u;  // (a group lies in one word)
#pragma unroll
    for (int i = 0; i < G; ++i) {
      float f = load_as_float<T>(&in[j][i]);
      const unsigned w = counts || biases ? word[at + i] : 0u;
      if (biased >> i & 1) f = __uint_as_float(w);
      else if (w) f = penalized(f, w);
      if (!(mask >> (j * G + i) & 1)) f = -INFINITY;
      out[i] = adjust_round<T>(f);
    }
    if (at + G <= n) {
      group v;
#pragma unroll
      for (int i = 0; i < G; ++i) v[i] = out[i];
      *(group *)(y + at) = v;
    } else {
#pragma unroll
      for (int i = 0; i < G; ++i)
        if (at + i < n) y[at + i] = out[i];
    }
  }
}

template <typename T>
static void adjust_launch(const Adjust &a, hipStream_t s) {
  auto launch = [&](auto per) {
    constexpr int PER = decltype(per)::value;
    logits_adjust_kernel<T, PER><<<dim3(ceil_div(a.V, ADJ_THREADS * PER), a.B), ADJ_THREADS, 0, s>>>(a);
  };
  // Short chunks while they are no more than the chip takes at once: more workgroups, each of which looks through the whole history.  us, short / long: one row of 32768 5.6 / 8.2, one of 100001
  // 7.1 / 11.5, 64 of 32768 10.1 / 11.3, 16 of 131072 in bfloat16 8.5 / 9.1, 64 of 131072 27.3 / 20.8.
  (long long)a.B * ceil_div(a.V, ADJ_THREADS * ADJ_PER_SHORT) <= ADJ_FEW ? launch(std::integral_constant<int, ADJ_PER_SHORT>{}) : launch(std::integral_constant<int, ADJ_PER>{});
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
  if (dtype == LA_F32) adjust_launch<float>(a, s);
  else if (dtype == LA_F16) adjust_launch<_Float16>(a, s);
  else adjust_launch<uint16_t>(a, s);
  LA_HIP(hipGetLastError());
  return LA_OK;
}
