// Sampling of a token per row from stored logits: temperature, top-k, top-p, min-p, a given random number per row (la_sample).
#include "la_device.h"
#include "la_internal.h"
#include "la_lanes.h"

namespace la {

// Weights.  With y = logit * 8 log2(e) / temperature (64 bits) and a = floor(y), a token's weight is 2^(a / 8) 2^((y - a) / 8): its bin is the number of eighths of
// an octave between its a and the row's largest, the second factor lies in [1, 1.091) and is rounded to 36 bits behind the point, wherever it is used.  Sums over a
// bin are then sums of whole numbers: they do not depend on the order in which LDS atomics take them, and equal logits have equal shares.  Everything behind them
// is added in a fixed order.  A sum of n weights is off by about 2^-38 / sqrt(n) of itself.  Bins reach 64 octaves down, below which a weight counts as none.
// Logits are read once, and then, of a row that is cut, the tokens of the cut's bin, of one that is not, a chunk.  The bytes bound neither launch: 64 rows of 131072, 34 MB, 6.5 us at a
// copy's rate, take 20 + 30 us.  The first is bound by its instructions: 59 a token, which is 94 % of what the CUs issue in the cycles that they are busy (their LDS is active in 40 %, half of
// that for lanes that meet in a bank).  The second is a chain in one workgroup a row: the chunks' first tokens, their sums, and for every filter that cuts a search by bins, the listed tokens' places
// and then their logits (two trips to memory) and a search among them, each with a few barriers; then the draw.  Both launches in a replayed graph, us, all 64 rows alike / one row: greedy 11 / 7,
// no filter 34 / 20, min-p 34 / 16, top-k of 50 31 / 18, of 1000 41 / 25, top-p of 0.9 39 / 26, top-k of 5000 and top-p of 0.95 43 / 30.  One row of 32768 5 + 11 us.
constexpr int SMP_BINS = 514, SMP_HIST = 520;  // (64 octaves below the largest token end in the 514th bin at the latest); row length of a chunk's sums
constexpr int SMP_SUM_THREADS = 512;          // of a workgroup of the first launch
constexpr int SMP_PER = 16, SMP_PER_SHORT = 4;  // ... tokens of each: chunks of 8192 and of 2048
constexpr int SMP_LIST = 4608;                // tokens of a cut that fit into LDS
constexpr int SMP_SHORT = 1024, SMP_FEW = 128;  // tokens down to a cut that are listed with it, a thread each; of them kept that are drawn from without looking at a chunk (two a lane)
constexpr int SMP_SUB = 1024;                 // parts that a range of tokens is cut into at a time
constexpr int SMP_COUNT_SHIFT = 50;           // a chunk's word of a bin: the number of its tokens above that bit, the sum of their factors below, in units of 2^-36
constexpr unsigned long long SMP_SUM_MASK = (1ull << SMP_COUNT_SHIFT) - 1;
constexpr double SMP_UNIT = 0x1p36, LEAST_WEIGHT = 0x1p-64;
constexpr int SMP_MOST = SMP_SUM_THREADS * SMP_PER;
static_assert(SMP_MOST * 1.1 * SMP_UNIT < (double)SMP_SUM_MASK && SMP_MOST <= 1 << 13, "a chunk in one bin");
static_assert(LA_MAX_SAMPLE_VOCAB * 1.1 * SMP_UNIT < 0x1p64 && LA_MAX_SAMPLE_VOCAB / SMP_MOST <= 64, "a row in one bin; a lane per chunk");
// Short chunks while that leaves a row at most 16 of them: the first launch has four times the workgroups, the second reads as many sums.  us, short / long chunks: 8192 tokens, 1, 8
// and 64 rows 17.5 / 19.4, 18.2 / 20.6, 18.9 / 21.1; 32768 17.0 / 19.2, 18.9 / 21.3, 24.4 / 22.6; 65536, 1 and 64 rows 20.0 / 19.9, 32.1 / 26.8; 131072, 1 row 24.8 / 20.7.  (Not by the
// number of rows: a row's sums are added by chunks, and do not depend on the rows beside it.)
static int sample_per(int V) { return V <= 16 * SMP_SUM_THREADS * SMP_PER_SHORT ? SMP_PER_SHORT : SMP_PER; }

struct Sample {
  const void *x;
  int64_t ld;
  int V, chunks;
  la_sampling p;
  int32_t *ids;
  float *prob;
  // per row and chunk: its first token in order; sums of weights and numbers of tokens of the bins down to each [SMP_HIST], from that token's bin on, up to the last bin that
  // has a token; its tokens by bin, as places in the chunk
  unsigned long long *best;
  double *sums;
  int32_t *counts, *used;
  uint16_t *sorted;
};

// A logit as it counts: NaN like -inf (no token), +inf like the largest finite value, -0 like 0.
template <typename T>
__device__ __forceinline__ float sample_logit(T raw) {
  const float x = load_as_float<T>(&raw);
  return x != x ? -INFINITY : fminf(x, 3.402823466e38f) + 0.f;
}
// A token as a number: larger is in front, (value descending, index ascending).
__device__ __forceinline__ unsigned long long sample_place(float x, int i) {
  const uint32_t u = __float_as_uint(x);
  return (unsigned long long)(u & 0x80000000u ? ~u : u | 0x80000000u) << 32 | (0xffffffffu - (unsigned)i);
}
__device__ __forceinline__ float sample_value(unsigned long long c) {
  const uint32_t k = (uint32_t)(c >> 32);
  return __uint_as_float(k & 0x80000000u ? k & 0x7fffffffu : ~k);
}
__device__ __forceinline__ int sample_index(unsigned long long c) { return (int)(0xffffffffu - (uint32_t)c); }

// 2^(f / 8), 0 <= f <= 1, in units of 2^-36: a polynomial that meets it in the six Chebyshev nodes (off by 3e-13 at most, a unit is 1.5e-11); 2^52 added to a number
// below it leaves the nearest whole number in the low bits.
__device__ __forceinline__ double sample_factor_52(double f) {
  const double z = f - 0.5;
  double s = 4.2495173672986880985e-8;
  s = __builtin_fma(s, z, 2.4523688009211048058e-6);
  s = __builtin_fma(s, z, 0.00011320602609171660186);
  s = __builtin_fma(s, z, 0.0039197225262626394621);
  s = __builtin_fma(s, z, 0.09047942850278266672);
  s = __builtin_fma(s, z, 1.0442737824277134712);
  return __builtin_fma(s, SMP_UNIT, 0x1p52);
}
__device__ __forceinline__ unsigned long long sample_factor(double f) { return __builtin_bit_cast(unsigned long long, sample_factor_52(f)) & ((1ull << 52) - 1); }
__device__ __forceinline__ double sample_factor_of(double f) { return sample_factor_52(f) - 0x1p52; }  // the same number
__device__ __forceinline__ double sample_eighths(int t) {  // 2^(-t / 8) units
  constexpr double e[8] = {1.0, 0.91700404320467123, 0.84089641525371454, 0.77110541270397041, 0.70710678118654752, 0.64841977732550483, 0.59460355750136053, 0.54525386633262883};
  double v = e[0];
#pragma unroll
  for (int i = 1; i < 8; ++i) v = (t & 7) == i ? e[i] : v;
  return ldexp(v * (1 / SMP_UNIT), -(t >> 3));
}

// y, rounded: what floor(y) and y - floor(y) are taken of.  (Left to the compiler, it may form the difference from the product as it is before its rounding; beyond 2^53 that is any
// number, not one of [0, 1), and the weights of equal logits are no longer the same bits wherever they are formed.)
__device__ __forceinline__ double sample_y(float x, double rate) {
#pragma clang fp contract(off)
  return (double)x * rate;
}

// How row b is sampled; the filters that are off are out of reach.
struct SampleRow {
  bool greedy;
  double rate;  // y = logit * rate
  int k;        // V: off
  float p, low;
};
__device__ __forceinline__ SampleRow sample_row(const Sample &a, int b) {
  SampleRow r;
  const float t = a.p.temperature ? a.p.temperature[b] : 1.f;
  r.greedy = uniform(!(t > 0.f)) != 0;
  r.rate = uniform(8 * 1.44269504088896340736 / (double)t);
  const int k = a.p.top_k ? a.p.top_k[b] : 0;
  r.k = k > 0 && k < a.V ? k : a.V;
  r.p = a.p.top_p ? a.p.top_p[b] : 1.f;
  if (!(r.p < 1.f)) r.p = 1.f;
  if (!(r.p > 0.f)) {  // the first token alone
    r.p = 1.f;
    r.k = 1;
  }
  r.low = a.p.min_p ? a.p.min_p[b] : 0.f;
  r.low = r.low > 0.f ? fminf(r.low, 1.f) : 0.f;
  r.k = uniform(r.k);
  r.p = __uint_as_float((unsigned)uniform((int)__float_as_uint(r.p)));
  r.low = __uint_as_float((unsigned)uniform((int)__float_as_uint(r.low)));
  return r;
}

// First launch, a workgroup per chunk of a row: its first token in order, and its bins' sums, relative to that token's.
template <typename T, int PER>
__global__ __launch_bounds__(SMP_SUM_THREADS) void sample_sum_kernel(Sample a) {
  constexpr int WAVES = SMP_SUM_THREADS / 64, CHUNK = SMP_SUM_THREADS * PER;
  __shared__ __attribute__((aligned(16))) unsigned long long hist[SMP_HIST];
  __shared__ unsigned long long red[WAVES];
  __shared__ double red_w[WAVES];
  __shared__ int red_n[WAVES], red_last[WAVES], before[SMP_HIST];
  __shared__ __attribute__((aligned(16))) uint16_t sorted[CHUNK];
  const int c = blockIdx.x, b = blockIdx.y, t = threadIdx.x, wave = t >> 6, lane = t & 63, i0 = c * CHUNK + t;
  const T *x = (const T *)a.x + b * a.ld;
  // (loads without a condition, and nothing done with one before all are requested)
  T raw[PER];
#pragma unroll
  for (int j = 0; j < PER; ++j) raw[j] = x[min(i0 + SMP_SUM_THREADS * j, a.V - 1)];
  float v[PER];
#pragma unroll
  for (int j = 0; j < PER; ++j) v[j] = i0 + SMP_SUM_THREADS * j < a.V ? sample_logit<T>(raw[j]) : -INFINITY;
  const SampleRow r = sample_row(a, b);
  for (int i = t; i < SMP_HIST; i += SMP_SUM_THREADS) hist[i] = 0;
  float top_v = -INFINITY;
#pragma unroll
  for (int j = 0; j < PER; ++j) top_v = fmaxf(top_v, v[j]);
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) top_v = fmaxf(top_v, __shfl_xor(top_v, o, 64));
  int top_i = 0;
  if (r.greedy) {  // (nobody else asks for it)
    top_i = 0x7fffffff;
#pragma unroll
    for (int j = PER - 1; j >= 0; --j) top_i = v[j] == top_v ? i0 + SMP_SUM_THREADS * j : top_i;
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) top_i = min(top_i, __shfl_xor(top_i, o, 64));
  }
  unsigned long long best = sample_place(top_v, top_i);
  if (lane == 0) red[wave] = best;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < WAVES; ++w) best = red[w] > best ? red[w] : best;
  best = uniform(best);
  const size_t at = (size_t)b * a.chunks + c;
  if (t == 0) a.best[at] = best;
  const float top = sample_value(best);
  if (r.greedy || !(top > -INFINITY)) return;
  const double first = floor(sample_y(top, r.rate));
  int at_bin[PER];  // bin and, from bit 10 on, the number of its tokens that were counted before
#pragma unroll
  for (int j = 0; j < PER; ++j) {
    const double y = sample_y(v[j], r.rate), low = floor(y), d = first - low;
    at_bin[j] = -1;
    if (v[j] > -INFINITY && d < SMP_BINS) {
      const int bin = (int)d;
      at_bin[j] = bin | (int)(atomicAdd(&hist[bin], (1ull << SMP_COUNT_SHIFT) + sample_factor(y - low)) >> SMP_COUNT_SHIFT) << 10;
    }
  }
  __syncthreads();
  // sums from the front, two bins a thread
  const bool own = 2 * t < SMP_HIST;
  double w0 = 0, w1 = 0;
  int n0 = 0, n1 = 0, last = 0;
  if (own) {
    const unsigned long long h0 = hist[2 * t], h1 = hist[2 * t + 1];
    w0 = (double)(h0 & SMP_SUM_MASK) * sample_eighths(2 * t);
    w1 = (double)(h1 & SMP_SUM_MASK) * sample_eighths(2 * t + 1);
    n0 = (int)(h0 >> SMP_COUNT_SHIFT);
    n1 = (int)(h1 >> SMP_COUNT_SHIFT);
    last = n1 ? 2 * t + 2 : n0 ? 2 * t + 1 : 0;
  }
  const unsigned long long any = __ballot(last > 0);
  if (lane == 0) red_last[wave] = any ? 2 * (64 * wave + 64 - (int)__builtin_clzll(any)) : 0;  // (rounded up to a whole thread's)
  const double w = lane_through(w0 + w1);
  int n = lane_through(n0 + n1);
  if (lane == 63) {
    red_w[wave] = w;
    red_n[wave] = n;
  }
  __syncthreads();
  // (a place is written once: by the token that the atomics gave its number; which of a bin's tokens that is changes nothing)
  const double front_w = sum_of(red_w, wave);
  n += sum_of(red_n, wave);
  int used = 0;
#pragma unroll
  for (int q = 0; q < WAVES; ++q) used = max(used, red_last[q]);
  if (own) {
    before[2 * t] = n - n1 - n0;
    before[2 * t + 1] = n - n1;
  }
  if (2 * t < used) {
    *(double2 *)(a.sums + at * SMP_HIST + 2 * t) = double2{front_w + (w - w1), front_w + w};
    *(int2 *)(a.counts + at * SMP_HIST + 2 * t) = int2{n - n1, n};
  }
  if (t == 0) a.used[at] = used;
  __syncthreads();
#pragma unroll
  for (int j = 0; j < PER; ++j)
    if (at_bin[j] >= 0) sorted[before[at_bin[j] & 1023] + (at_bin[j] >> 10)] = (uint16_t)(t + SMP_SUM_THREADS * j);
  __syncthreads();
  const int all = before[SMP_HIST - 1];  // (the last bin is past any token)
  for (int q = t; 8 * q < all; q += SMP_SUM_THREADS) *(uint4 *)(a.sorted + at * CHUNK + 8 * q) = *(const uint4 *)(sorted + 8 * q);
}

// Second launch, a workgroup per row: where the filters cut, what is left of every chunk, and in the chunk where u falls the token.
constexpr int SMP_THREADS = 1024, SMP_WAVES = SMP_THREADS / 64;
struct SampleShared {
  unsigned long long list[SMP_LIST];
  unsigned long long sub_w[SMP_SUB];
  unsigned sub_n[SMP_SUB];
  double through_w[SMP_BINS];  // sums over the bins up to and with this one
  int through_n[SMP_BINS];
  unsigned long long chunk_in[64];
  double before[64];
  double red_d[SMP_WAVES];
  unsigned long long red_u[SMP_WAVES];
  unsigned red_n[SMP_WAVES];
  unsigned long long lo, hi, base_w, kept_w, found;
  unsigned base_n, part_n, n_few;
  int hit, last, where;
  unsigned long long few_c[SMP_FEW], few_w[SMP_FEW];
  int rank[SMP_FEW];
  int from[64], ends[64];  // of a bin: where its tokens begin in each chunk's, how many there are up to and with each
  double eighths[8];
};

template <typename T, int PER>
__global__ __launch_bounds__(SMP_THREADS) void sample_kernel(Sample a) {
  constexpr int CHUNK = SMP_SUM_THREADS * PER;
  __shared__ SampleShared m;
  const int b = blockIdx.x, t = threadIdx.x, wave = t >> 6, lane = t & 63, V = a.V, C = a.chunks;
  const T *x = (const T *)a.x + b * a.ld;
  const SampleRow r = sample_row(a, b);
  // lane c of every wave: chunk c's first token, and the bins up to its last (without a token: nothing of its own was written, and nothing is looked at)
  const bool chunk = lane < C;
  const unsigned long long c_best = chunk ? a.best[(size_t)b * C + lane] : 0;
  const int c_used = chunk ? a.used[(size_t)b * C + lane] : 0;
  if (t < 64) m.chunk_in[t] = 0;
  if (t < 8) m.eighths[t] = sample_eighths(t);
  const float c_top = chunk ? sample_value(c_best) : -INFINITY;
  float top = c_top;
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor(top, o, 64));
  top = __uint_as_float((unsigned)uniform((int)__float_as_uint(top)));
  if (r.greedy || !(top > -INFINITY)) {
    unsigned long long best = c_best;
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
      const unsigned long long y = __shfl_xor(best, o, 64);
      best = y > best ? y : best;
    }
    if (t == 0) {
      a.ids[b] = top > -INFINITY ? sample_index(best) : -1;
      if (a.prob) a.prob[b] = top > -INFINITY ? 1.f : 0.f;
    }
    return;
  }
  const double y_top = uniform(sample_y(top, r.rate)), first = uniform(floor(y_top)), w_top = (double)sample_factor(y_top - first) * (1 / SMP_UNIT);
  const double c_down = first - floor(sample_y(c_top, r.rate));
  const int c_shift = c_down < SMP_BINS ? (int)c_down : SMP_BINS;
  const double c_scale = c_down < SMP_BINS ? sample_eighths((int)c_down) * SMP_UNIT : 0.0;
  const double *sums = a.sums + (size_t)b * C * SMP_HIST;
  const int32_t *counts = a.counts + (size_t)b * C * SMP_HIST;
  // ---- the row's sums down to each bin
  if (64 * wave < SMP_BINS) {  // (whole waves: a lane that takes no part does not have to keep what lane_value reads of it)
    double w = 0;
    int n = 0;
    constexpr int N = 16;
    for (int c0 = 0; c0 < C; c0 += N) {  // (loads without a condition, all on their way at once)
      double sw[N];
      int sn[N], l[N];
#pragma unroll
      for (int k = 0; k < N; ++k) {
        const int c = min(c0 + k, C - 1);
        l[k] = c0 + k < C ? t - lane_value(c_shift, c) : -1;
        const int at = max(min(l[k], lane_value(c_used, c) - 1), 0);
        sw[k] = sums[c * SMP_HIST + at];
        sn[k] = counts[c * SMP_HIST + at];
      }
#pragma unroll
      for (int k = 0; k < N; ++k) {
        w += l[k] >= 0 ? sw[k] * lane_value(c_scale, min(c0 + k, C - 1)) : 0.0;
        n += l[k] >= 0 ? sn[k] : 0;
      }
    }
    if (t < SMP_BINS) {
      m.through_w[t] = w;
      m.through_n[t] = n;
    }
  }
  __syncthreads();
  auto in_bins = [&](double y, int t0, int t1) { return y >= first - t1 && (t0 == 0 || y < first - t0 + 1); };
  int listed0 = SMP_BINS, listed1 = -1, n_list = 0;  // bins whose tokens are in the list, how many they are
  // Where the tokens of bins t0 .. t1 lie; their number.
  auto slices = [&](int t0, int t1) {
    __syncthreads();
    if (wave == 0) {
      const int top = c_used - 1, l0 = t0 - 1 - c_shift, l1 = t1 - c_shift;
      const bool any = l1 >= 0 && c_shift < SMP_BINS;
      const int32_t *n = counts + (any ? lane * SMP_HIST : 0);
      const int from = any && l0 >= 0 ? n[min(l0, top)] : 0, end = any ? n[min(l1, top)] : 0;
      m.from[lane] = from;
      m.ends[lane] = lane_through(end - from);
    }
    __syncthreads();
    return uniform(m.ends[63]);
  };
  // The i-th of them: its index.
  auto nth = [&](int i) {
    int lo = 0, hi = C - 1;
    while (lo < hi) {
      const int c = (lo + hi) / 2;
      if (m.ends[c] > i) hi = c; else lo = c + 1;
    }
    return lo * CHUNK + a.sorted[((size_t)b * C + lo) * CHUNK + m.from[lo] + i - (lo > 0 ? m.ends[lo - 1] : 0)];
  };
  // Tokens of bins t0 .. t1 into the list, if they fit.
  auto gather = [&](int t0, int t1) {
    const int n = slices(t0, t1);
    listed0 = n <= SMP_LIST ? t0 : SMP_BINS;
    listed1 = n <= SMP_LIST ? t1 : -1;
    n_list = n;
    if (n > SMP_LIST) return;
    for (int i = t; i < n; i += SMP_THREADS) {
      const int at = nth(i);
      m.list[i] = sample_place(sample_logit<T>(x[at]), at);
    }
    __syncthreads();
  };
  // Every token of bin `bin` and of places lo .. hi: f(its place, its factor).
  auto each = [&](int bin, unsigned long long lo, unsigned long long hi, auto f) {
    auto take = [&](unsigned long long c, float v) {
      const double y = sample_y(v, r.rate);
      if (c >= lo && c <= hi && in_bins(y, bin, bin)) f(c, sample_factor(y - floor(y)));
    };
    if (bin >= listed0 && bin <= listed1) {
      for (int i = t; i < n_list; i += SMP_THREADS) take(m.list[i], sample_value(m.list[i]));
    } else {  // (more tokens than the list holds)
      const int n = slices(bin, bin);
      for (int i0 = t; i0 < n; i0 += 4 * SMP_THREADS) {
        int at[4];
        T raw[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) at[j] = nth(min(i0 + SMP_THREADS * j, n - 1));
#pragma unroll
        for (int j = 0; j < 4; ++j) raw[j] = x[at[j]];
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (i0 + SMP_THREADS * j < n) take(sample_place(sample_logit<T>(raw[j]), at[j]), sample_logit<T>(raw[j]));
      }
    }
  };
  // The last of the tokens that are kept of a bin: the rank-th in order, or the first with which their sum of factors reaches want;
  // the last one at `from` or in front of it if none does.  m.kept_w: their sum.  The range of places is cut into SMP_SUB parts until one token is left, which
  // takes seven turns at most (a place has 64 bits, a turn settles ten), or until 64 tokens are left, which a wave compares with each other; a range without any token ends it too.
  auto last_kept = [&](int bin, unsigned long long from, unsigned rank, double want) {
    __syncthreads();
    if (t == 0) {
      // no token of the bin lies outside of its ends, which a float's rounding moves by less than they are widened here (no temperature's: everywhere)
      const double low = (first - bin) / r.rate, high = (first - bin + 1) / r.rate;
      const float l = (float)(low - fabs(low) * 0x1p-20 - 0x1p-120), h = (float)(high + fabs(high) * 0x1p-20 + 0x1p-120);
      const unsigned long long lo = r.rate > 0 && l > -3e38f && l < 3e38f ? sample_place(l, -1) & ~0xffffffffull : 0;
      const unsigned long long hi = r.rate > 0 && h > -3e38f && h < 3e38f ? sample_place(h, 0) | 0xffffffffull : ~0ull;
      m.lo = lo > from ? lo : from;
      m.hi = hi;
      m.base_n = 0;
      m.base_w = m.kept_w = 0;
      m.found = ~0ull;
      m.n_few = 0;
      m.part_n = (unsigned)(m.through_n[bin] - (bin > 0 ? m.through_n[bin - 1] : 0));
    }
    __syncthreads();
    for (int turn = 0; turn < 8; ++turn) {
      if (uniform((int)m.part_n) <= 64) {
        each(bin, uniform(m.lo), uniform(m.hi), [&](unsigned long long c, unsigned long long f) {
          const unsigned at = atomicAdd(&m.n_few, 1u);
          m.few_c[at] = c;
          m.few_w[at] = f;
        });
        __syncthreads();
        if (wave == 0) {
          const int n = uniform((int)m.n_few);
          const unsigned long long c = lane < n ? m.few_c[lane] : 0, f = lane < n ? m.few_w[lane] : 0;
          unsigned in_front = m.base_n;
          unsigned long long w = m.base_w;
          for (int j = 0; j < n; ++j) {
            const bool ahead = m.few_c[j] >= c;
            in_front += ahead ? 1 : 0;
            w += ahead ? m.few_w[j] : 0;
          }
          const unsigned long long hit = __ballot(lane < n && (rank ? in_front == rank : (double)w >= want && (double)(w - f) < want));
          const unsigned long long last = __ballot(lane < n && in_front == m.base_n + (unsigned)n);
          if (n > 0 && lane == (int)__builtin_ctzll(hit ? hit : last)) {
            m.found = c;
            m.kept_w = w;
          }
        }
        break;
      }
      const unsigned long long lo = uniform(m.lo), hi = uniform(m.hi);
      const int bits = 64 - __builtin_clzll((hi - lo) | 1), sh = bits > 10 ? bits - 10 : 0;
      m.sub_n[t] = 0;
      m.sub_w[t] = 0;
      __syncthreads();
      each(bin, lo, hi, [&](unsigned long long c, unsigned long long f) {
        const unsigned s = (unsigned)((c - lo) >> sh);
        atomicAdd(&m.sub_n[s], 1u);
        atomicAdd(&m.sub_w[s], f);
      });
      if (t == 0) {
        m.hit = SMP_THREADS;
        m.last = -1;
      }
      __syncthreads();
      const int s = SMP_SUB - 1 - t;  // from the front of the order on
      const unsigned own_n = m.sub_n[s];
      const unsigned long long own_w = m.sub_w[s];
      unsigned n = lane_through(own_n);
      unsigned long long w = lane_through(own_w);
      if (lane == 63) {
        m.red_n[wave] = n;
        m.red_u[wave] = w;
      }
      __syncthreads();
      n += m.base_n + sum_of(m.red_n, wave);
      w += m.base_w + sum_of(m.red_u, wave);
      const unsigned long long filled = __ballot(own_n > 0), enough = __ballot(own_n > 0 && (rank ? n >= rank : (double)w >= want));
      if (lane == 0) {
        if (enough) atomicMin(&m.hit, t + (int)__builtin_ctzll(enough));
        if (filled) atomicMax(&m.last, t + 63 - (int)__builtin_clzll(filled));
      }
      __syncthreads();
      const int hit = uniform(m.hit), last = uniform(m.last);
      if (last < 0) break;
      if (t == (hit < SMP_THREADS ? hit : last)) {
        const unsigned long long at = lo + ((unsigned long long)s << sh), end = at + ((1ull << sh) - 1);
        m.lo = at;
        m.hi = end < at || end > hi ? hi : end;
        m.base_n = n - own_n;
        m.base_w = w - own_w;
        m.kept_w = w;
        m.part_n = own_n;
      }
      __syncthreads();
    }
    __syncthreads();
    return uniform(m.found);
  };
  // ---- what is kept: the bins in front of `cut_bin`, and of that one the tokens at `cut` or in front of it
  int cut_bin = SMP_BINS;
  unsigned long long cut = 0;
  double partial = 0;  // sum of the latter
  auto first_bin = [&](auto ok) {
    __syncthreads();
    if (t == 0) m.hit = SMP_BINS;
    __syncthreads();
    const unsigned long long yes = __ballot(t < SMP_BINS && ok(t < SMP_BINS ? t : 0));
    if (lane == 0 && yes) atomicMin(&m.hit, t + (int)__builtin_ctzll(yes));
    __syncthreads();
    return uniform(m.hit);
  };
  auto cut_at = [&](int bin, unsigned long long from, unsigned rank, double want) {
    cut = last_kept(bin, from, rank, want);
    cut_bin = bin;
    partial = (double)uniform(m.kept_w) * sample_eighths(bin);
  };
  if (r.k < V) {
    const int h = first_bin([&](int i) { return m.through_n[i] >= r.k; });
    if (h < SMP_BINS) {
      const int through = uniform(m.through_n[h]);
      if (through == r.k) {
        cut_bin = h + 1;
        cut = ~0ull;
      } else {
        gather(through <= SMP_SHORT ? 0 : h, h);
        cut_at(h, 0, (unsigned)(r.k - (h > 0 ? uniform(m.through_n[h - 1]) : 0)), 0);
      }
    }
  }
  if (r.p < 1.f) {
    const double want = (double)r.p * ((cut_bin > 0 ? m.through_w[cut_bin - 1] : 0) + partial);
    const int h = first_bin([&](int i) { return i < cut_bin && m.through_w[i] >= want; });
    const bool inside = h < SMP_BINS;
    if (inside || (cut_bin < SMP_BINS && cut != ~0ull)) {
      const int bin = inside ? h : cut_bin;
      if (bin < listed0 || bin > listed1) gather(uniform(m.through_n[bin]) <= SMP_SHORT ? 0 : bin, bin);
      cut_at(bin, inside ? 0 : cut, 0, (want - (bin > 0 ? m.through_w[bin - 1] : 0)) / sample_eighths(bin));
    }
  }
  double w_least = LEAST_WEIGHT * w_top;
  if (r.low > 0.f) {
    const double d = first - floor(y_top + 8 * log2((double)r.low));
    w_least = fmax(w_least, (double)r.low * w_top);
    const int bin = uniform(d < SMP_BINS ? (int)d : SMP_BINS);
    if (bin < cut_bin) {
      cut_bin = bin;
      cut = 0;
    }
  }
  auto kept = [&](double f, int bin, float v, int i) {  // the token's weight, 0: not kept
    const double w = ldexp(f * m.eighths[bin & 7], -(bin >> 3));
    return (bin < cut_bin || (bin == cut_bin && sample_place(v, i) >= cut)) && w >= w_least ? w : 0.0;
  };
  float u = a.p.u_index ? a.p.u[min(max(a.p.u_index[b], 0), a.p.n_u - 1)] : a.p.u[b];
  u = u > 0.f ? fminf(u, 1.f) : 0.f;
  // ---- few tokens: those that are kept, put into the order of their indexes, and the sums over them
  if (cut_bin < SMP_BINS && uniform(m.through_n[cut_bin]) <= SMP_SHORT) {
    if (listed0 > 0 || cut_bin > listed1) gather(0, cut_bin);
    __syncthreads();
    if (t < SMP_FEW) m.rank[t] = 0;
    if (t == 0) m.n_few = 0;
    __syncthreads();
    for (int i = t; i < n_list; i += SMP_THREADS) {
      const unsigned long long c = m.list[i];
      const float v = sample_value(c);
      const double y = sample_y(v, r.rate), low = floor(y);
      const double w = kept(sample_factor_of(y - low), (int)(first - low), v, sample_index(c));
      if (w > 0.0) {
        const unsigned at = atomicAdd(&m.n_few, 1u);
        if (at < SMP_FEW) {
          m.few_c[at] = (unsigned)sample_index(c);
          m.few_w[at] = __builtin_bit_cast(unsigned long long, w);
        }
      }
    }
    __syncthreads();
    const int n = uniform((int)m.n_few);
    if (n > 0 && n <= SMP_FEW) {
      constexpr int PARTS = SMP_THREADS / SMP_FEW;
      const int i = t % SMP_FEW, part = t / SMP_FEW;
      const unsigned long long mine = i < n ? m.few_c[i] : 0;
      int in_front = 0;
      for (int j = part; j < n; j += PARTS) in_front += m.few_c[j] < mine ? 1 : 0;
      if (i < n && in_front) atomicAdd(&m.rank[i], in_front);
      __syncthreads();
      if (t < n) m.list[m.rank[t]] = (unsigned long long)t;  // (the list is through)
      __syncthreads();
      if (wave == 0) {
        constexpr int PAIR = SMP_FEW / 64;
        double w[PAIR], sum = 0;
        int id[PAIR];
#pragma unroll
        for (int q = 0; q < PAIR; ++q) {
          const int at = PAIR * lane + q, from = at < n ? (int)m.list[at] : 0;
          w[q] = at < n ? __builtin_bit_cast(double, m.few_w[from]) : 0.0;
          id[q] = (int)m.few_c[from];
          sum += w[q];
        }
        double run = lane_through(sum);
        const double total = lane_value(run, 63), want = (double)u * total;
        run -= sum;
        int hit = PAIR;
#pragma unroll
        for (int q = 0; q < PAIR; ++q) {
          run += w[q];
          if (hit == PAIR && w[q] > 0.0 && run > want) hit = q;
        }
        const unsigned long long past = __ballot(hit < PAIR);
        const int who = past ? (int)__builtin_ctzll(past) : (n - 1) / PAIR;  // (u is 1: the last one)
        if (lane == who) {
          if (!past) hit = (n - 1) % PAIR;
#pragma unroll
          for (int q = 0; q < PAIR; ++q)
            if (q == hit) {
              a.ids[b] = id[q];
              if (a.prob) a.prob[b] = (float)(w[q] / total);
            }
        }
      }
      return;
    }
  }
  // ---- what is left of each chunk
  __syncthreads();
  double mine = 0.0;
  if (lane < C) {
    const int l = (cut_bin < SMP_BINS ? cut_bin : SMP_BINS) - 1 - c_shift;
    if (l >= 0) mine = sums[lane * SMP_HIST + min(l, c_used - 1)] * c_scale;
  }
  if (cut_bin < SMP_BINS && cut != ~0ull) {
    if (cut_bin < listed0 || cut_bin > listed1) gather(cut_bin, cut_bin);
    each(cut_bin, cut, ~0ull, [&](unsigned long long c, unsigned long long f) {
      if (kept((double)f, cut_bin, sample_value(c), sample_index(c)) > 0.0) atomicAdd(&m.chunk_in[sample_index(c) / CHUNK], f);
    });
  }
  __syncthreads();
  mine += (double)m.chunk_in[lane] * sample_eighths(cut_bin);
  const double ends = lane_through(mine), total = lane_value(ends, 63);
  const double want = (double)u * total;
  const unsigned long long past = __ballot(mine > 0.0 && ends > want), some = __ballot(mine > 0.0);  // (the same in every wave)
  if (wave == 0) m.before[lane] = ends - mine;
  // ---- the token in the chunk (in the last chunk that has any where u is 1; a chunk whose sum is all of weights that count as none is passed over)
  for (int c = past ? __builtin_ctzll(past) : 63 - __builtin_clzll(some | 1); c < C; ++c) {
    if (!((some >> c) & 1)) continue;
    constexpr int N = CHUNK / SMP_THREADS;
    const int i0 = c * CHUNK + t * N;
    const double y_least = first - (cut_bin < SMP_BINS ? cut_bin : SMP_BINS - 1);  // (of a token that can be kept)
    constexpr int VEC = N * (int)sizeof(T) < 16 ? N * (int)sizeof(T) : 16;  // bytes of a load, where rows and chunks begin on such
    __attribute__((aligned(16))) T raw[N];
    double w[N], sum = 0;
    if ((uintptr_t)x % 16 == 0 && (c + 1) * CHUNK <= V && (VEC == 16 || VEC == 8)) {
#pragma unroll
      for (int j = 0; j < N; j += VEC / (int)sizeof(T)) {
        if constexpr (VEC == 16) *(uint4 *)(raw + j) = *(const uint4 *)(x + i0 + j);
        else if constexpr (VEC == 8) *(uint2 *)(raw + j) = *(const uint2 *)(x + i0 + j);
      }
    } else {
#pragma unroll
      for (int j = 0; j < N; ++j) raw[j] = x[min(i0 + j, V - 1)];
    }
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const float v = i0 + j < V ? sample_logit<T>(raw[j]) : -INFINITY;
      const double y = sample_y(v, r.rate);
      w[j] = 0.0;
      if (v > -INFINITY && y >= y_least) {
        const double low = floor(y);
        w[j] = kept(sample_factor_of(y - low), (int)(first - low), v, i0 + j);
      }
      sum += w[j];
    }
    double run = lane_through(sum);
    __syncthreads();
    if (lane == 63) m.red_d[wave] = run;
    if (t == 0) {
      m.where = 0x7fffffff;
      m.last = -1;
    }
    __syncthreads();
    run = (run - sum) + (m.before[c] + sum_of(m.red_d, wave));
    int hit = 0x7fffffff, last = -1;
#pragma unroll
    for (int j = 0; j < N; ++j) {
      run += w[j];
      if (w[j] > 0.0) {
        last = i0 + j;
        if (run > want && hit == 0x7fffffff) hit = i0 + j;
      }
    }
    const unsigned long long hits = __ballot(hit != 0x7fffffff), keeps = __ballot(last >= 0);  // (lanes are in the order of their tokens)
    const int first_hit = lane_value(hit, hits ? (int)__builtin_ctzll(hits) : 0), last_keep = lane_value(last, keeps ? 63 - (int)__builtin_clzll(keeps) : 0);
    if (lane == 0) {
      if (hits) atomicMin(&m.where, first_hit);
      if (keeps) atomicMax(&m.last, last_keep);
    }
    __syncthreads();
    const int id = uniform(m.where != 0x7fffffff ? m.where : m.last);
    if (id < 0) continue;
#pragma unroll
    for (int j = 0; j < N; ++j)
      if (i0 + j == id) {
        a.ids[b] = id;
        if (a.prob) a.prob[b] = (float)(w[j] / total);
      }
    return;
  }
  if (t == 0) {  // (not reached: the largest token is always kept)
    a.ids[b] = -1;
    if (a.prob) a.prob[b] = 0.f;
  }
}

}  // namespace la

using namespace la;

struct SampleLayout {
  int per, chunks;
  size_t sums, counts, used, sorted, total;  // byte offsets behind the first tokens, size of all
};
static SampleLayout sample_layout(int B, int V) {
  SampleLayout l{};
  l.per = sample_per(V);
  l.chunks = ceil_div(V, SMP_SUM_THREADS * l.per);
  const size_t n = (size_t)B * l.chunks;
  l.sums = (n * 8 + 15) / 16 * 16;
  l.counts = l.sums + n * SMP_HIST * 8;
  l.used = l.counts + n * SMP_HIST * 4;
  l.sorted = (l.used + n * 4 + 15) / 16 * 16;
  l.total = l.sorted + n * SMP_SUM_THREADS * l.per * 2;
  return l;
}
static_assert(SMP_HIST % 4 == 0, "16-byte aligned parts");
extern "C" size_t la_sample_workspace(int B, int V) {
  if (B < 1 || V < 1 || V > LA_MAX_SAMPLE_VOCAB) return 0;  // (what the call itself refuses)
  return sample_layout(B, V).total;
}

template <typename T, int PER>
static int sample_launch(const Sample &a, int B, hipStream_t s) {
  {
    ProfScope ps("sample_sum", s);
    sample_sum_kernel<T, PER><<<dim3(a.chunks, B), SMP_SUM_THREADS, 0, s>>>(a);
  }
  {
    ProfScope ps("sample", s);
    sample_kernel<T, PER><<<B, SMP_THREADS, 0, s>>>(a);
  }
  LA_HIP(hipGetLastError());
  return LA_OK;
}
template <typename T>
static int sample_launch(const Sample &a, int per, int B, hipStream_t s) {
  return per == SMP_PER ? sample_launch<T, SMP_PER>(a, B, s) : sample_launch<T, SMP_PER_SHORT>(a, B, s);
}

extern "C" int la_sample(const void *logits, int dtype, int64_t row_stride, int B, int V, const la_sampling *how, int32_t *ids, float *prob, void *workspace,
                         size_t workspace_bytes, void *stream) {
  LA_REQUIRE(how != nullptr, LA_EINVAL, "NULL argument");
  LA_REQUIRE(B >= 0 && B <= 65535, LA_EINVAL, "B=%d outside [0, 65535]", B);
  if (B == 0) return LA_OK;
  LA_REQUIRE(logits && ids && how->u, LA_EINVAL, "NULL argument");
  LA_REQUIRE(dtype == LA_F32 || dtype == LA_BF16 || dtype == LA_F16, LA_EINVAL, "unknown dtype %d", dtype);
  LA_REQUIRE(V >= 1 && V <= LA_MAX_SAMPLE_VOCAB, LA_EINVAL, "vocab %d outside [1, %d]", V, LA_MAX_SAMPLE_VOCAB);
  LA_REQUIRE(row_stride >= V || B == 1, LA_EINVAL, "rows overlap");
  LA_REQUIRE(how->n_u >= (how->u_index ? 1 : B), LA_EINVAL, "%d random numbers for %d rows", how->n_u, B);
  const SampleLayout l = sample_layout(B, V);
  LA_REQUIRE(workspace && workspace_bytes >= l.total, LA_ENOMEM, "workspace of %zu bytes, %zu needed", workspace_bytes, l.total);
  LA_REQUIRE((uintptr_t)workspace % 16 == 0, LA_EINVAL, "workspace must be 16-byte aligned");
  hipStream_t s = (hipStream_t)stream;
  uint8_t *w = (uint8_t *)workspace;
  const Sample a{logits, row_stride, V, l.chunks, *how, ids, prob, (unsigned long long *)w, (double *)(w + l.sums), (int32_t *)(w + l.counts), (int32_t *)(w + l.used),
                 (uint16_t *)(w + l.sorted)};
  if (dtype == LA_F32) return sample_launch<float>(a, l.per, B, s);
  if (dtype == LA_F16) return sample_launch<_Float16>(a, l.per, B, s);
  return sample_launch<uint16_t>(a, l.per, B, s);
}
