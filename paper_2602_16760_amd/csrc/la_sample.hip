// Sampling of a token per row from stored logits: temperature, top-k, top-p, min-p, a given random number per row (la_sample).
#include "la_device.h"
#include "la_internal.h"

namespace la {

struct Sample {
  const void *x;
  int64_t ld;
  int V;
  la_sampling p;
  int32_t *ids;
  float *prob;
};

constexpr double LEAST_WEIGHT = 0x1p-64;

// A logit as it counts: NaN like -inf (no token), +inf like the largest finite value, -0 like 0.
template <typename T>
__device__ __forceinline__ float sample_logit(const T *p) {
  const float x = load_as_float<T>(p);
  return x != x ? -INFINITY : fminf(x, 3.402823466e38f) + 0.f;
}
__device__ __forceinline__ uint32_t sample_key(float x) {  // keys are ordered as the values are
  const uint32_t u = __float_as_uint(x);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

constexpr int SMP_THREADS = 1024;

template <typename T>
__global__ __launch_bounds__(SMP_THREADS) void sample_kernel(Sample a) {
  __shared__ double red[SMP_THREADS / 64], scan[SMP_THREADS / 64];
  __shared__ unsigned long long redu[SMP_THREADS / 64];
  __shared__ int found;
  const int b = blockIdx.x, t = threadIdx.x, V = a.V;
  const T *x = (const T *)a.x + b * a.ld;
  auto sum = [&](double v) {
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
    __syncthreads();
    if ((t & 63) == 0) red[t >> 6] = v;
    __syncthreads();
    double s = 0;
    for (int w = 0; w < SMP_THREADS / 64; ++w) s += red[w];
    return s;
  };
  // the row's first token in order: (value descending, index ascending), as one number
  auto place = [&](int i) { return (unsigned long long)sample_key(sample_logit<T>(x + i)) << 32 | (0xffffffffu - (unsigned)i); };
  unsigned long long best = 0;
  for (int i = t; i < V; i += SMP_THREADS) {
    const unsigned long long c = place(i);
    best = c > best ? c : best;
  }
  for (int o = 32; o > 0; o >>= 1) {
    const unsigned long long c = __shfl_xor(best, o, 64);
    best = c > best ? c : best;
  }
  if ((t & 63) == 0) redu[t >> 6] = best;
  __syncthreads();
  for (int w = 0; w < SMP_THREADS / 64; ++w) best = redu[w] > best ? redu[w] : best;
  const int i_top = (int)(0xffffffffu - (unsigned)best);
  const float top = sample_logit<T>(x + i_top);
  const float temp = a.p.temperature ? a.p.temperature[b] : 1.f;
  if (!(top > -INFINITY) || !(temp > 0.f)) {
    if (t == 0) {
      a.ids[b] = top > -INFINITY ? i_top : -1;
      if (a.prob) a.prob[b] = top > -INFINITY ? 1.f : 0.f;
    }
    return;
  }
  auto weight = [&](int i) {
    const float v = sample_logit<T>(x + i);
    const double w = v > -INFINITY ? exp(((double)v - (double)top) / (double)temp) : 0.0;
    return w < LEAST_WEIGHT ? 0.0 : w;
  };
  // the last token that is kept, by bisection over the order
  const int k = a.p.top_k && a.p.top_k[b] > 0 && a.p.top_k[b] < V ? a.p.top_k[b] : V;
  const float p = a.p.top_p ? a.p.top_p[b] : 1.f, low = a.p.min_p ? a.p.min_p[b] : 0.f;
  auto last_with = [&](auto enough) {  // the largest c whose tokens at c or in front of it are enough
    unsigned long long c = 0;
    for (int bit = 63; bit >= 0; --bit)
      if (enough(c | 1ull << bit)) c |= 1ull << bit;
    return c;
  };
  unsigned long long cut = k < V ? last_with([&](unsigned long long c) {
    double n = 0;
    for (int i = t; i < V; i += SMP_THREADS) n += place(i) >= c;
    return sum(n) >= (double)k;
  }) : 0;
  auto mass = [&](unsigned long long c) {
    double n = 0;
    for (int i = t; i < V; i += SMP_THREADS)
      if (place(i) >= c) n += weight(i);
    return sum(n);
  };
  if (p < 1.f) {
    const double want = (double)p * mass(cut);
    const unsigned long long c = p > 0.f ? last_with([&](unsigned long long c) { return mass(c) >= want; }) : best;
    cut = c > cut ? c : cut;
  }
  const double least = low > 0.f ? (low < 1.f ? (double)low : 1.0) : 0.0;
  auto kept = [&](int i) {
    const double w = i < V && place(i) >= cut ? weight(i) : 0.0;
    return w >= least ? w : 0.0;
  };
  // sums in index order, tiles of a token per thread; the second time until the sum passes u of the whole
  double want = -1.0, total = 0.0;
  for (int turn = 0; turn < 2; ++turn) {
    double before = 0.0;
    for (int i0 = 0; i0 < V; i0 += SMP_THREADS) {
      const double w = kept(i0 + t);
      double s = w;
      for (int o = 1; o < 64; o <<= 1) {
        const double y = __shfl_up(s, o, 64);
        if ((t & 63) >= o) s += y;
      }
      __syncthreads();
      if ((t & 63) == 63) scan[t >> 6] = s;
      if (t == 0) found = 0x7fffffff;
      __syncthreads();
      double front = before, all = before;
      for (int q = 0; q < SMP_THREADS / 64; ++q) {
        if (q < (t >> 6)) front += scan[q];
        all += scan[q];
      }
      if (turn == 1) {
        if (w > 0.0 && front + s > want) atomicMin(&found, i0 + t);
        __syncthreads();
        if (found != 0x7fffffff) {
          if (t == 0) a.ids[b] = found;
          if (i0 + t == found && a.prob) a.prob[b] = (float)(w / total);
          return;
        }
      }
      before = all;
    }
    total = before;
    float u = a.p.u_index ? a.p.u[min(max(a.p.u_index[b], 0), a.p.n_u - 1)] : a.p.u[b];
    u = u > 0.f ? u : 0.f;
    want = fmin((double)u, 1.0 - 0x1p-30) * total;
  }
}

}  // namespace la

using namespace la;

extern "C" size_t la_sample_workspace(int B, int V) {
  (void)B; (void)V;
  return 0;
}

extern "C" int la_sample(const void *logits, int dtype, int64_t row_stride, int B, int V, const la_sampling *how, int32_t *ids, float *prob, void *workspace,
                         size_t workspace_bytes, void *stream) {
  LA_REQUIRE(how != nullptr, LA_EINVAL, "NULL argument");
  LA_REQUIRE(B >= 0, LA_EINVAL, "B=%d is negative", B);
  if (B == 0) return LA_OK;
  LA_REQUIRE(logits && ids && how->u, LA_EINVAL, "NULL argument");
  LA_REQUIRE(dtype == LA_F32 || dtype == LA_BF16 || dtype == LA_F16, LA_EINVAL, "unknown dtype %d", dtype);
  LA_REQUIRE(V >= 1 && V <= LA_MAX_SAMPLE_VOCAB, LA_EINVAL, "vocab %d outside [1, %d]", V, LA_MAX_SAMPLE_VOCAB);
  LA_REQUIRE(row_stride >= V || B == 1, LA_EINVAL, "rows overlap");
  LA_REQUIRE(how->n_u >= (how->u_index ? 1 : B), LA_EINVAL, "%d random numbers for %d rows", how->n_u, B);
  (void)workspace; (void)workspace_bytes;
  hipStream_t s = (hipStream_t)stream;
  const Sample a{logits, row_stride, V, *how, ids, prob};
  ProfScope ps("sample", s);
  if (dtype == LA_F32) sample_kernel<float><<<B, SMP_THREADS, 0, s>>>(a);
  else if (dtype == LA_F16) sample_kernel<_Float16><<<B, SMP_THREADS, 0, s>>>(a);
  else sample_kernel<uint16_t><<<B, SMP_THREADS, 0, s>>>(a);
  LA_HIP(hipGetLastError());
  return LA_OK;
}
