// What stands between stored logits and the choice of a token: penalties for tokens that occurred, biases, a grammar's mask (la_logits_adjust).
#include <limits.h>

#include <type_traits>

#include "la_device.h"
#include "la_internal.h"
#include "la_lanes.h"

namespace la {

// A workgroup per chunk of a row.  How often each of the chunk's tokens occurred is counted in LDS, from the request's committed tokens and those drafted on the row's path; then the
// logits, requested before, pass once.  Counts are whole numbers and a token's biases are added in the list's order: results do not depend on the order of the atomics, nor on the chunks.
// Bound by a chain (settings, history, LDS, division) at few rows, 5.0 us for one of 32768; by the bytes and that chain at many: 64 rows of 131072, 67.6 MB, 8192 tokens of history each, 19.4 us =
// 3.5 TB/s, all workgroups resident and in step (64 registers; with 67 a fourth workgroup did not fit a CU: 22.4).  Loads and stores of four bytes, requested as they were needed, took 50; a
// search through all biases by each token that has one 116 instead of 11.6 us where 300 fall on one row.
constexpr int ADJ_THREADS = 512;
constexpr int ADJ_PER = 16, ADJ_PER_SHORT = 4;  // tokens of a thread: chunks of 8192 and of 2048
constexpr int ADJ_LIST = 256;                   // biases of a chunk that are kept in LDS
constexpr int ADJ_FEW = 1024;                   // short chunks of a launch at most
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

// VEC: rows are 16-byte aligned, a thread has 16 bytes at a time.
template <typename T, int PER, bool VEC>
__global__ __launch_bounds__(ADJ_THREADS, 8) void logits_adjust_kernel(Adjust a) {
  constexpr int CHUNK = ADJ_THREADS * PER, G = 16 / (int)sizeof(T) < PER ? 16 / (int)sizeof(T) : PER, GROUPS = PER / G;  // tokens of a group; groups of a thread
  typedef T __attribute__((ext_vector_type(G))) group;
  __shared__ __attribute__((aligned(16))) unsigned word[CHUNK];
  __shared__ int list_token[ADJ_LIST], list_at[ADJ_LIST], n_list;
  __shared__ float list_bias[ADJ_LIST], list_x[ADJ_LIST];
  const int b = blockIdx.y, t = threadIdx.x, v0 = blockIdx.x * CHUNK, n = a.V - v0 < CHUNK ? a.V - v0 : CHUNK;
  const la_adjust &p = a.p;
  const T *x = (const T *)a.x + b * a.ldx + v0;
  T *y = (T *)a.y + b * a.ldy + v0;
  // token i of group j is j * ADJ_THREADS * G + t * G + i of the chunk
  T in[GROUPS][G];
#pragma unroll
  for (int j = 0; j < GROUPS; ++j) {
    const int at = (j * ADJ_THREADS + t) * G;
    if (VEC && at + G <= n) {
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
  unsigned mask[GROUPS];  // a group's bits, from bit 0 on
#pragma unroll
  for (int j = 0; j < GROUPS; ++j) mask[j] = ~0u;
  const uint32_t *allowed = nullptr;
  if (p.allowed) {
    const int m = uniform(p.allowed_index ? p.allowed_index[b] : b);
    if ((unsigned)m < (unsigned)p.n_allowed) {
      allowed = p.allowed + m * p.allowed_stride;
#pragma unroll
      for (int j = 0; j < GROUPS; ++j) {
        const int at = v0 + (j * ADJ_THREADS + t) * G;
        mask[j] = allowed[(at < a.V ? at : 0) >> 5] >> (at & 31);  // (a group lies in one word)
      }
    }
  }
  auto setting = [&](const float *f, float off, bool positive) {  // (what is no number, or no factor, is off)
    const float v = f && known ? f[r] : off;
    return v - v == 0.f && (!positive || v > 0.f) ? v : off;
  };
  const float rho = setting(p.repetition, 1.f, true), beta = setting(p.presence, 0.f, false), alpha = setting(p.frequency, 0.f, false);
  const bool counts = rho != 1.f || beta != 0.f || alpha != 0.f, biases = known && p.n_bias > 0;
  if (uniform(counts || biases)) {
    for (int i = 4 * t; i < CHUNK; i += 4 * ADJ_THREADS) *(uint4 *)(word + i) = uint4{0, 0, 0, 0};
    if (t == 0) n_list = 0;
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
    if (biases)
      for (int i = t; i < p.n_bias; i += ADJ_THREADS) {
        const int d = p.bias_token[r * p.bias_stride + i], v = d - v0;
        if (d < v0 || v >= n) continue;
        atomicOr(&word[v], ADJ_BIASED);
        const int at = atomicAdd(&n_list, 1);
        if (at < ADJ_LIST) {
          list_token[at] = v;
          list_at[at] = i;
          list_bias[at] = p.bias[r * p.bias_stride + i];
          list_x[at] = load_as_float<T>(x + v);  // (nobody writes before the barrier)
        }
      }
    __syncthreads();
  }
  auto penalized = [&](float f, unsigned w) {
    const unsigned c = w & ADJ_COUNT;
    if (counts && w & (ADJ_SEEN | ADJ_COUNT)) f = f > 0.f ? f / rho : f * rho;
    return counts && c ? f - alpha * (float)c - beta : f;
  };
  // Tokens with biases: the thread of the first of a token's entries adds them all up, in the list's order, and stores the token; everybody else leaves it out.  More entries than LDS has room
  // for: the tokens' own threads go through the whole list.
  const bool listed = uniform(biases) && n_list <= ADJ_LIST;
  if (listed && t < n_list) {
    const int v = list_token[t], at = list_at[t];
    bool own = true, more = false;
    for (int k = 0; k < n_list; ++k)
      if (list_token[k] == v && k != t) {
        more = true;
        own = own && list_at[k] > at;
      }
    if (own) {
      float f = penalized(list_x[t], word[v]) + list_bias[t];
      for (int last = at; more;) {
        int next = INT_MAX;
        float add = 0.f;
        for (int k = 0; k < n_list; ++k)
          if (list_token[k] == v && list_at[k] > last && list_at[k] < next) {
            next = list_at[k];
            add = list_bias[k];
          }
        if (next == INT_MAX) break;
        f += add;
        last = next;
      }
      if (allowed && !(allowed[(v0 + v) >> 5] >> ((v0 + v) & 31) & 1)) f = -INFINITY;
      y[v] = adjust_round<T>(f);
    }
  }
#pragma unroll
  for (int j = 0; j < GROUPS; ++j) {
    const int at = (j * ADJ_THREADS + t) * G;
    if (at >= n) continue;
    T out[G];
    unsigned whose = 0;  // bit i: token i is stored by another thread
#pragma unroll
    for (int i = 0; i < G; ++i) {
      float f = load_as_float<T>(&in[j][i]);
      const unsigned w = counts || biases ? word[at + i] : 0;
      if (w) {
        f = penalized(f, w);
        if (w & ADJ_BIASED) {
          if (listed) whose |= 1u << i;
          else
            for (int k = 0; k < p.n_bias; ++k)
              if (p.bias_token[r * p.bias_stride + k] == v0 + at + i) f += p.bias[r * p.bias_stride + k];
        }
      }
      if (!(mask[j] >> i & 1)) f = -INFINITY;
      out[i] = adjust_round<T>(f);
    }
    if (VEC && at + G <= n && !whose) {
      group v;
#pragma unroll
      for (int i = 0; i < G; ++i) v[i] = out[i];
      *(group *)(y + at) = v;
    } else {
#pragma unroll
      for (int i = 0; i < G; ++i)
        if (at + i < n && !(whose >> i & 1)) y[at + i] = out[i];
    }
  }
}

template <typename T>
static void adjust_launch(const Adjust &a, hipStream_t s) {
  const bool vec = ((uintptr_t)a.x | (uintptr_t)a.y) % 16 == 0 && (a.B == 1 || (a.ldx * sizeof(T) % 16 == 0 && a.ldy * sizeof(T) % 16 == 0));
  auto launch = [&](auto per, auto v) {
    constexpr int PER = decltype(per)::value;
    logits_adjust_kernel<T, PER, decltype(v)::value><<<dim3(ceil_div(a.V, ADJ_THREADS * PER), a.B), ADJ_THREADS, 0, s>>>(a);
  };
  auto sized = [&](auto per) { vec ? launch(per, std::true_type{}) : launch(per, std::false_type{}); };
  // Short chunks while they are no more than the chip takes at once: more workgroups, each of which looks through the whole history.  us, short / long: one row of 32768 5.6 / 8.2, one of 100001
  // 7.1 / 11.5, 64 of 32768 10.1 / 11.3, 16 of 131072 in bfloat16 8.5 / 9.1, 64 of 131072 27.3 / 20.8.
  (long long)a.B * ceil_div(a.V, ADJ_THREADS * ADJ_PER_SHORT) <= ADJ_FEW ? sized(std::integral_constant<int, ADJ_PER_SHORT>{}) : sized(std::integral_constant<int, ADJ_PER>{});
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
