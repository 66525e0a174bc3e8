// What the paged attentions' kernels share: their items, the matrix instructions of their types, the forms of their output.  A, their arguments: B rows whose keys they share out
// (at_keys), target, list and firsts as at_plan has them.
#pragma once
#include <type_traits>

#include "la_attend_plan.h"
#include "la_lanes.h"
#include "la_paged.h"

namespace la {

typedef __attribute__((__vector_size__(8 * sizeof(__bf16)))) __bf16 at_b8;
typedef _Float16 __attribute__((ext_vector_type(8))) at_h8;
typedef float __attribute__((ext_vector_type(4))) at_f4;
typedef unsigned __attribute__((ext_vector_type(4))) at_u4;
typedef unsigned __attribute__((ext_vector_type(2))) at_u2;

constexpr float AT_LOG2E = 1.4426950408889634f;
constexpr size_t AT_CACHED = (size_t)256 << 20;  // a layer's K and V pages of more bytes are not kept in the last-level cache

template <typename A>
__device__ __forceinline__ int at_uncut(const A &) { return 0; }

// The wanted item, or item 0 of the wanted row; b = -1: there is none.  Rows that are not cut are items themselves.  Of up to 64 rows every wave finds it from the rows'
// positions, a lane each; of more it was written down by a launch of its own: formed by every workgroup from all rows' positions, 64 at a time, the time grew with the square of the
// rows (512 rows of 1000 379 us, with the list 344; 65 rows 57 and 59).
// RECORDS: its place among the records of rows that are cut is wanted too.  Where no row has more than at_uncut(a) keys, none is cut.
template <bool BY_ROW, bool RECORDS, typename A>
__device__ __forceinline__ AtItem at_find(const A &a, int wanted) {
  AtItem it{};
  if (a.target <= 0) {
    int r;
    const int n = at_keys(a, wanted, r);
    it.b = wanted;
    it.r = uniform(r);
    it.n = uniform(n);
    it.C = AT_UNCUT;
    it.first = wanted;
    it.count = 1;
    return it;
  }
  if (a.list) return a.list[BY_ROW ? a.firsts[wanted] : wanted];
  const int lane = threadIdx.x & 63;
  int r = 0;
  const int n = lane < a.B ? at_keys(a, lane, r) : 0;
  int c = 0, ends = 0;
  auto items = [&](int C) {
    c = lane < a.B ? at_rows_items(n, C) : 0;
    ends = lane_through(c);
    return lane_value(ends, 63);
  };
  const int longest = lane_most(n);
  (void)items(RECORDS && longest <= at_uncut(a) ? AT_UNCUT : at_cut(a.B, a.target, lane_value(lane_through((long long)n), 63), longest, items));
  const int l = BY_ROW ? wanted : __builtin_popcountll(__ballot(ends <= wanted));
  it.b = -1;
  if (l >= a.B) return it;
  it.b = l;
  it.r = lane_value(r, l);
  it.n = lane_value(n, l);
  it.count = lane_value(c, l);
  it.C = uniform(at_item_keys(it.n, it.count));
  it.first = lane_value(ends, l) - it.count;
  it.index = BY_ROW ? 0 : wanted - it.first;
  if constexpr (RECORDS) {
    const int own = c > 1 ? c : 0, through = lane_through(own);
    it.record = lane_value(through, l) - it.count + it.index;  // (of a row that is cut)
  }
  return it;
}

// The same items of more than 64 rows, by one workgroup that goes through the rows a thread each; `items`: places in the list.
constexpr int AT_PLAN_THREADS = 1024;
template <bool RECORDS, typename A>
__global__ __launch_bounds__(AT_PLAN_THREADS) void paged_plan_kernel(A a, int items) {
  constexpr int WAVES = AT_PLAN_THREADS / 64;
  __shared__ long long red[WAVES];
  const int t = threadIdx.x, wave = t >> 6, lane = t & 63;
  auto all_of = [&](long long v) {  // its sum over the threads
    v = lane_through(v);
    __syncthreads();
    if (lane == 63) red[wave] = v;
    __syncthreads();
    return uniform((unsigned long long)sum_of(red, WAVES));
  };
  long long keys = 0;
  int r, longest = 0;
  for (int b = t; b < a.B; b += AT_PLAN_THREADS) {
    const int n = at_keys(a, b, r);
    keys += n;
    longest = longest > n ? longest : n;
  }
  keys = (long long)all_of(keys);
  __syncthreads();
  longest = lane_most(longest);
  if (lane == 0) red[wave] = longest;
  __syncthreads();
  longest = lane_most(lane < WAVES ? (int)red[lane] : 0);
  const int C = RECORDS && longest <= at_uncut(a) ? AT_UNCUT : at_cut(a.B, a.target, keys, longest, [&](int C) {
    long long c = 0;
    for (int b = t; b < a.B; b += AT_PLAN_THREADS) c += at_rows_items(at_keys(a, b, r), C);
    return (int)all_of(c);
  });
  int before = 0, records = 0;
  for (int b0 = 0; b0 < a.B; b0 += AT_PLAN_THREADS) {
    const int b = b0 + t, n = b < a.B ? at_keys(a, b, r) : 0, c = b < a.B ? at_rows_items(n, C) : 0;
    const int through = lane_through(c);
    const int total = (int)all_of(c);  // (what it leaves in `red` are the waves' sums)
    const int first = before + (int)sum_of(red, wave) + through - c;
    int record = 0;
    if constexpr (RECORDS) {
      const int own = c > 1 ? c : 0, own_through = lane_through(own), all = (int)all_of(own);
      record = records + (int)sum_of(red, wave) + own_through - own;
      records += all;
    }
    if (b < a.B) a.firsts[b] = first;
    for (int i = 0; i < c && first + i < items; ++i) a.list[first + i] = AtItem{b, r, n, at_item_keys(n, c), i, first, c, record + i};
    before += total;
  }
  for (int i = before + t; i < items; i += AT_PLAN_THREADS) a.list[i].b = -1;
}

__device__ __forceinline__ float at_max4(float v) {  // over the four lanes 16 apart
  v = fmaxf(v, __shfl_xor(v, 16, 64));
  return fmaxf(v, __shfl_xor(v, 32, 64));
}
__device__ __forceinline__ float at_sum4(float v) {
  v += __shfl_xor(v, 16, 64);
  return v + __shfl_xor(v, 32, 64);
}

template <typename T>
__device__ __forceinline__ unsigned at_pack(float lo, float hi) {  // to nearest even
  typedef float f2 __attribute__((ext_vector_type(2)));
  if constexpr (std::is_same<T, _Float16>::value) {
    typedef _Float16 h2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(unsigned, __builtin_convertvector((f2{lo, hi}), h2));
  } else {
    typedef __bf16 b2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(unsigned, __builtin_convertvector((f2{lo, hi}), b2));
  }
}
// Two weights as the sum of two 16-bit numbers each, both above zero where the weight is, so that an infinite V stays one: the first is short of the weight by one to three half
// steps, the second is what that leaves.  Together they are off by 2^-20 of the weight at most (half precision), 2^-14 (bfloat16).
template <typename T>
__device__ __forceinline__ at_u2 at_split(float x, float y) {
  constexpr bool F16 = std::is_same<T, _Float16>::value;
  constexpr float SHORT = F16 ? 1.f - 0x1p-10f : 1.f - 0x1p-7f;
  const unsigned first = at_pack<T>(x * SHORT, y * SHORT);
  const float x0 = F16 ? (float)__builtin_bit_cast(_Float16, (uint16_t)(first & 0xffffu)) : __uint_as_float(first << 16);
  const float y0 = F16 ? (float)__builtin_bit_cast(_Float16, (uint16_t)(first >> 16)) : __uint_as_float(first & 0xffff0000u);
  return at_u2{first, at_pack<T>(x - x0, y - y0)};
}
template <typename T>
__device__ __forceinline__ at_f4 at_mma(at_u4 x, at_u4 y, at_f4 c) {
  if constexpr (std::is_same<T, _Float16>::value)
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(at_h8, x), __builtin_bit_cast(at_h8, y), c, 0, 0, 0);
  else return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(at_b8, x), __builtin_bit_cast(at_b8, y), c, 0, 0, 0);
}

// A value of the output where a model's next product wants it (the fragments' type takes +-65504 at most).
template <typename A>
__device__ __forceinline__ void at_store_row(const A &a, int b, int col, float y) {
  if (a.kind == AT_OUT_FLOAT) {
    ((float *)a.out)[b * a.ldo + col] = y;
  } else {
    _Float16 *to = (_Float16 *)a.out + (((size_t)(col >> 5) * a.q_tiles + (b >> 4)) * 64 + (b & 15) + 16 * ((col & 31) >> 3)) * 8 + (col & 7);
    *to = (_Float16)fminf(fmaxf(y, -65504.f), 65504.f);
  }
}

}  // namespace la
