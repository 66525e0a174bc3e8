// What the kernels of the trees' attention share: their arguments, the requests' rows, how weights are formed and split.
#pragma once
#include <atomic>

#include "la_attend.h"
#include "la_tree_plan.h"

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
  int B, max_blocks;  // requests
  const int32_t *first, *len;
  const uint64_t *vis;
  int max_rows, N;  // rows of a request at most, of all
  void *out;
  int64_t ldo;
  int target, tiles, items;  // as at_plan has them
  int uncut;          // keys up to which no request is cut
  int q_tiles, kind;  // as la_paged_attend's
  bool once;          // K and V are read by one workgroup each and are more than the last-level cache holds: they are not kept there
  int rec;            // floats of a row's and head's record of an item
  float *part;        // [record][Hq][max_rows][rec]
  AtItem *list;
  int32_t *firsts;
  int2 *notes;  // of each request, where any may be cut: its first record, how many items it has
};
static_assert(sizeof(int2) == TA_NOTE, "what the join is told");

// A request's rows: the first one's number, and how many take part.
__device__ __forceinline__ int tree_rows(const TreeAttend &a, int r, int &f) {
  f = a.first[r];
  const int e = a.first[r + 1], n = (e < a.N ? e : a.N) - f;
  return f < 0 || n < 0 ? 0 : n < a.max_rows ? n : a.max_rows;
}
__device__ __forceinline__ int at_keys(const TreeAttend &a, int b, int &r) {
  int f;
  r = b;
  const int rows = tree_rows(a, b, f);
  const long long L = a.len[b], n = L + rows, cap = (long long)a.max_blocks * a.page;
  return rows == 0 || L < 0 ? 0 : (int)(n < cap ? n : cap);
}

// A column's offset is moved when a score is this many octaves above it, so that most blocks need no maximum over lanes and no sums to be rescaled (two requests of 64 rows at 65000, bfloat16: 210 us,
// with an offset that follows each maximum 245; half precision 237 and 249).  Weights are up to 2^LAZY then, and half precision's carry 2^UP besides, as la_paged_attend's do, so that a step of its
// smallest numbers is 2^-39 of the largest weight; the factor goes out with the sum.  2^(UP + LAZY) may be 2^16 at most, which ta_split still splits, so its offsets lag by less than an octave.
// (With 11 and 4 in place of 15 and 7/8 it took 221, but 600 keys of 2^-31 of a first one's weight came out 3 % off.)  The other types have 8 bits of exponent and need no factor.
template <typename T> constexpr float TA_LAZY = std::is_same<T, _Float16>::value ? 0.875f : 8.f;
template <typename T> constexpr float TA_UP = std::is_same<T, _Float16>::value ? 15.f : 0.f;
// Weights are 2^(factor s - base + UP), formed in one instruction, with factor s not rounded and base rounded: where scores are large that is off by a part of a float's spacing there, and by
// octaves from 2^24 on, so that the largest weight itself is no number of the type any more, or nothing.  Columns that are TA_FAR octaves from zero, where the part is 2^-14, round factor s as base
// was: its difference from base is exact then, and nothing for the largest.  Whether a wave has such columns is found out where offsets move; the others' weights are formed as ever.
constexpr float TA_FAR = 1024.f;
__device__ __forceinline__ bool ta_far(float m) { return __any(fabsf(m) > TA_FAR && m > -INFINITY); }
__device__ __forceinline__ float ta_from(float s, float factor, float base) {
#pragma clang fp contract(off)
  const float x = s * factor;
  return x - base;
}
template <typename T>
__device__ __forceinline__ float ta_exponent(float s, float factor, float base) {
  return fabsf(base) > TA_FAR ? ta_from(s, factor, base) + TA_UP<T> : __builtin_fmaf(s, factor, TA_UP<T> - base);
}
__device__ __forceinline__ int at_uncut(const TreeAttend &a) { return a.uncut; }

// Two weights as the sum of two 16-bit numbers each, 1 + TA_REST times the weight together: the first is the weight cut to the type, so the second is above zero where the weight is (an
// infinite V stays one), in half precision down to 2^-40 of the largest, below which nothing is left of a weight.  The factor is the same for all weights and goes out with their sum.  What is
// lost of a weight is 2^-20 of it at most or half a step of half precision's smallest numbers, 2^-40 of the largest (bfloat16: 2^-15 of it), so that the outputs' own rounding is what an output is
// off by; one number of 11 or 8 bits would have been half the products, and as far off as that rounding again.
template <typename T> constexpr float TA_REST = std::is_same<T, _Float16>::value ? 0x1p-10f : sizeof(T) == 2 ? 0x1p-12f : 0.f;
template <typename T>
__device__ __forceinline__ at_u2 ta_split(float x, float y) {
  if constexpr (std::is_same<T, _Float16>::value) {
    const auto cut = __builtin_amdgcn_cvt_pkrtz(x, y);
    typedef _Float16 __attribute__((ext_vector_type(2))) pair;
    const pair rest = {(_Float16)__builtin_fmaf(x, 1.f + TA_REST<T>, -(float)cut[0]), (_Float16)__builtin_fmaf(y, 1.f + TA_REST<T>, -(float)cut[1])};  // (one instruction each)
    return at_u2{__builtin_bit_cast(unsigned, cut), __builtin_bit_cast(unsigned, rest)};
  } else {
    const unsigned u = __float_as_uint(x), v = __float_as_uint(y);
    return at_u2{__builtin_amdgcn_perm(v, u, 0x07060302u), at_pack<T>(__builtin_fmaf(x, 1.f + TA_REST<T>, -__uint_as_float(u & 0xffff0000u)),
                                                                      __builtin_fmaf(y, 1.f + TA_REST<T>, -__uint_as_float(v & 0xffff0000u)))};
  }
}
template <typename T>
__device__ __forceinline__ bool ta_odd(unsigned v) {  // an infinity or NaN among a word's numbers
  if constexpr (sizeof(T) == 4) return (v & 0x7f800000u) == 0x7f800000u;
  constexpr unsigned E = std::is_same<T, _Float16>::value ? 0x7c00u : 0x7f80u;
  return (v & E) == E || (v >> 16 & E) == E;
}

// Zeros for rows that see nothing: those of no request, and a request's behind the ones that take part.
template <typename T>
__device__ __forceinline__ void ta_zero(const TreeAttend &a, long long i, int col0, int cols, int t, int threads) {
  for (int c = t; c < cols; c += threads) {
    if (a.kind != AT_OUT_ROWS) at_store_row(a, (int)i, col0 + c, 0.f);
    else ((T *)a.out)[i * a.ldo + col0 + c] = T(0);
  }
}

// Rows of no request, over the whole launch; a request's rows behind the ones that take part.
template <typename T>
__device__ __forceinline__ void ta_zero_outside(const TreeAttend &a, int threads) {
  const long long front = a.first[0], back = a.first[a.B];
  for (long long i = (back > 0 ? back : 0) + blockIdx.x; i < a.N; i += gridDim.x) ta_zero<T>(a, i, 0, a.Hq * a.dh, threadIdx.x, threads);
  for (long long i = blockIdx.x; i < (front < a.N ? front : a.N); i += gridDim.x) ta_zero<T>(a, i, 0, a.Hq * a.dh, threadIdx.x, threads);
}
template <typename T>
__device__ __forceinline__ void ta_zero_behind(const TreeAttend &a, int b, int first, int n_rows, int col0, int cols, int threads) {
  const long long end = a.first[b + 1];
  for (long long i = (long long)first + n_rows; first >= 0 && i < (end < a.N ? end : a.N); ++i) ta_zero<T>(a, i, col0, cols, threadIdx.x, threads);
}
// The item, kv head and tile of columns of a workgroup (item -1: none).  The tiles of one item and head read the same keys: they go to one XCD, eight workgroups apart.
__device__ __forceinline__ void ta_share(const TreeAttend &a, int block, int &item, int &h, int &tile) {
  const int turn = block / 8, group = a.tiles > 1 ? turn / a.tiles * 8 + block % 8 : block;
  tile = uniform(a.tiles > 1 ? turn % a.tiles : 0);
  item = uniform(group / a.Hkv);
  h = uniform(group - item * a.Hkv);
  if (item >= a.items) item = -1;
}

// What the join asks for, so that it does not form the items anew.
__device__ __forceinline__ void ta_note(const TreeAttend &a, const AtItem &it, int h, int tile) {
  if (a.notes && it.index == 0 && h == 0 && tile == 0 && threadIdx.x == 0) a.notes[it.b] = int2{it.record, it.count};
}

// A kernel's right to more LDS than 64 KB, asked for once a device.
template <auto KERNEL>
int ta_allow_lds(int bytes) {
  static std::atomic<unsigned long long> done{0};
  int device = 0;
  LA_HIP(hipGetDevice(&device));
  const unsigned long long bit = 1ull << (device & 63);
  if (done.load(std::memory_order_relaxed) & bit) return LA_OK;
  LA_HIP(hipFuncSetAttribute((const void *)KERNEL, hipFuncAttributeMaxDynamicSharedMemorySize, bytes));
  done.fetch_or(bit, std::memory_order_relaxed);
  return LA_OK;
}

// The wide kernel's launch (la_tree_wide.hip), where tree_wide says that it is for the shape; 64 or 128 columns of a workgroup.
int tree_attend_wide(const TreeAttend &a, int dtype, int columns, unsigned grid, hipStream_t s);

}  // namespace la
