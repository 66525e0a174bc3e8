// Sums over a wave's lanes by moves between lanes that do not go through LDS (a shuffle takes some sixty cycles, such a move eight).
#pragma once
#include <hip/hip_runtime.h>

namespace la {

// The value of the lane that CTRL names; 0 in lanes without one, and in rows of 16 lanes that ROWS leaves out.
template <int CTRL, int ROWS>
__device__ __forceinline__ int lane_from(int v) { return __builtin_amdgcn_update_dpp(0, v, CTRL, ROWS, 0xf, false); }
template <int CTRL, int ROWS>
__device__ __forceinline__ unsigned lane_from(unsigned v) { return (unsigned)lane_from<CTRL, ROWS>((int)v); }
template <int CTRL, int ROWS>
__device__ __forceinline__ unsigned long long lane_from(unsigned long long v) {
  return (unsigned long long)lane_from<CTRL, ROWS>((unsigned)(v >> 32)) << 32 | lane_from<CTRL, ROWS>((unsigned)v);
}
template <int CTRL, int ROWS>
__device__ __forceinline__ long long lane_from(long long v) { return (long long)lane_from<CTRL, ROWS>((unsigned long long)v); }
template <int CTRL, int ROWS>
__device__ __forceinline__ double lane_from(double v) { return __builtin_bit_cast(double, lane_from<CTRL, ROWS>(__builtin_bit_cast(unsigned long long, v))); }

// Lane l's value, in every lane (l alike in all of them).
__device__ __forceinline__ int lane_value(int v, int l) { return __builtin_amdgcn_readlane(v, l); }
__device__ __forceinline__ unsigned lane_value(unsigned v, int l) { return (unsigned)__builtin_amdgcn_readlane((int)v, l); }
__device__ __forceinline__ unsigned long long lane_value(unsigned long long v, int l) {
  return (unsigned long long)lane_value((unsigned)(v >> 32), l) << 32 | lane_value((unsigned)v, l);
}
__device__ __forceinline__ long long lane_value(long long v, int l) { return (long long)lane_value((unsigned long long)v, l); }
__device__ __forceinline__ double lane_value(double v, int l) { return __builtin_bit_cast(double, lane_value(__builtin_bit_cast(unsigned long long, v), l)); }

// Sum over a row's lanes in front and this one; over all lanes in front and this one.  Every lane of the wave takes part.
template <typename N>
__device__ __forceinline__ N row_through(N v) {
  v += lane_from<0x111, 0xf>(v);  // row_shr by 1, 2, 4, 8
  v += lane_from<0x112, 0xf>(v);
  v += lane_from<0x114, 0xf>(v);
  v += lane_from<0x118, 0xf>(v);
  return v;
}
template <typename N>
__device__ __forceinline__ N lane_through(N v) {
  v = row_through(v);
  v += lane_from<0x142, 0xa>(v);  // the last lane of rows 0 and 2 onto rows 1 and 3, of row 1 onto 2 and 3
  v += lane_from<0x143, 0xc>(v);
  return v;
}
// The largest of a wave's numbers, none of them negative.
__device__ __forceinline__ int lane_most(int v) {
  auto most = [](int x, int y) { return x > y ? x : y; };
  v = most(v, lane_from<0x111, 0xf>(v));
  v = most(v, lane_from<0x112, 0xf>(v));
  v = most(v, lane_from<0x114, 0xf>(v));
  v = most(v, lane_from<0x118, 0xf>(v));
  v = most(v, lane_from<0x142, 0xa>(v));
  return lane_value(most(v, lane_from<0x143, 0xc>(v)), 63);
}
// The sum of the first n <= 16 of an array in LDS, in every lane.
template <typename N>
__device__ __forceinline__ N sum_of(const N *a, int n) {
  const int lane = threadIdx.x & 63;
  return lane_value(row_through(lane < n ? a[lane] : N(0)), 15);
}

// What all threads have alike, as scalars: branches around barriers are then jumps, not masks.
__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }
__device__ __forceinline__ unsigned long long uniform(unsigned long long v) {
  return (unsigned long long)(unsigned)__builtin_amdgcn_readfirstlane((int)(v >> 32)) << 32 | (unsigned)__builtin_amdgcn_readfirstlane((int)v);
}
__device__ __forceinline__ double uniform(double v) { return __builtin_bit_cast(double, uniform(__builtin_bit_cast(unsigned long long, v))); }

}  // namespace la
