// Attention of single tokens over a paged cache (la_paged_attend): the keys of a row are split into items, an item is a workgroup, and a second launch joins
// the items of rows that have several.  K and V are read once for the up to 16 query heads of a kv head that share a tile, and their bytes bound it where they are many: two rows
// of 131000 positions, 1.07 GB, 165 us, 6.5 TB/s (a large copy here: 5.2); 512 rows of 1000, 2.1 GB, 328 us, 6.4.  A row of 500, 2 MB, takes 9 us, of which the bytes are 0.4: a launch, the
// positions, the table, K and V, the waves' meeting, each waiting for the one before.  Pages that 16 does not divide, and float: the table is looked up for every block of keys, a trip to memory
// that the block's loads wait for (17 rows of up to 1008, float, pages of 24: 3.6 MB, 8 us).
#include <algorithm>

#include "la_attend.h"

namespace la {

struct PagedAttend {
  const void *K, *V;  // of the layer
  int n_pages, page, Hkv, dh;
  const void *q;
  int64_t ldq;
  int Hq;
  float scale;
  const int32_t *table;
  int64_t ldt;
  int n_req, max_blocks;
  const int32_t *req, *pos;
  int B;
  void *out;
  int64_t ldo;
  int target;    // items that all keys together are cut into, about; 0: every row is one item
  int q_tiles;   // > 0: q lies in operand fragments, [head][q_tiles][dh / 32][lane][8] of a 16-bit type; 0: rows
  int kind;      // PagedOut
  int rec;       // floats of a head's record of an item: running maximum, sum, two of padding, dh sums
  float *part;   // [item][Hq][rec]
  AtItem *list;  // the items as paged_plan_kernel leaves them; NULL: every wave finds its own
  int32_t *firsts;  // ... and the rows' first ones
};

constexpr int AT_WAVES = 4, AT_WHOLE_WAVES = 8;  // of a workgroup; where rows are not cut and heads are few
constexpr int AT_JOIN_WAVES = 4;

// Keys that row b sees (none where it is padding or names no request), and its request.
__device__ __forceinline__ int at_keys(const PagedAttend &a, int b, int &r) {
  r = a.req ? a.req[b] : b;
  const long long n = (long long)a.pos[b] + 1, cap = (long long)a.max_blocks * a.page;
  return (unsigned)r >= (unsigned)a.n_req || n < 0 ? 0 : (int)(n < cap ? n : cap);
}

// A workgroup takes an item's keys for one kv head and up to 16 of its query heads; its waves take blocks of KEYS keys in turn and meet once, at the end.
// Scores are formed as K q^T (a lane holds one query head's scores of four keys of each 16-key tile), the output as V^T p^T: the contraction runs over the
// keys in the order in which the lanes hold the scores, so the probabilities go from one product into the other without leaving their lanes.  V's operand
// wants eight keys of one channel in a lane: a lane loads eight channels of its eight keys and turns them around in its registers (half an instruction per
// element); which channels make up a tile of the output is free, so neighbouring channels of V end up in neighbouring registers.
//   float: 16 keys a block and the float matrix instruction, whose contraction takes one key per lane: nothing to turn around.
// Scores, running maximum and sum, and both products' sums are float.  A weight goes into the second product as two 16-bit numbers (at_split), which costs a product more for each
// of V's: rounded to one, its half step comes out as large as the output's own (a row of 500, bfloat16: 1.8e-3 off as a whole, now 1.6e-3, which is what rounding the exact output leaves).
// Half precision has no small numbers: below 2^-14 its step is 2^-24, below 2^-25 nothing is left, while many such weights beside a large one whose V is small are the output.  So
// its weights are up to 2^15 instead of 1 (UP; the sums carry the factor too, and it cancels): a step below 2^-29 of the largest is 2^-39 of it.  Keys behind a first one of 2^22.5,
// 2^25 and 2^30 times their weight: 512 of them off by 0.8, 12 and 12 % without it, by half a step of the output with it.
// PAGED16: page_size is a multiple of 16, so that a 16-key tile lies in one page and its address is a scalar; otherwise a lane looks up its own keys' places.
// FULL: head_dim = DH; otherwise what a lane would load behind a row's end is replaced by zeros.
// ONCE: K and V are more than the last-level cache holds, so what goes through it is not kept there.
template <typename T, int DH, bool PAGED16, bool FULL, int WAVES, bool ONCE>
__global__ __launch_bounds__(64 * WAVES, DH > 128 ? 1 : 2) void paged_attend_kernel(PagedAttend a) {
  constexpr bool F32 = sizeof(T) == 4;
  constexpr int E = sizeof(T), TILES = F32 ? 1 : 2, KEYS = 16 * TILES;
  constexpr int KP = DH * E / 64;                  // 16-byte pieces of a key row per lane (four lanes a row)
  constexpr int VW = DH * E / 16 < 16 ? 8 : 16;    // bytes of a V load: a row's share of each of 16 lanes, at most 16
  constexpr int VH = DH * E / 16 / VW;             // such loads a row
  constexpr int VC = VW / E;                       // channels of one
  constexpr int DT = DH / 16;                      // tiles of the output: channel VH-th part, one of VC
  constexpr int VK = 4 * TILES;                    // keys whose V a lane loads
  constexpr float UP = std::is_same<T, _Float16>::value ? 15.f : 0.f;  // all weights carry 2^UP
  extern __shared__ __attribute__((aligned(16))) float at_lds[];
  const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), lane = threadIdx.x & 63, q4 = lane >> 4, c16 = lane & 15;
  const int g = uniform(a.Hq / a.Hkv), tiles = uniform((g + AT_ROWS - 1) / AT_ROWS), item = uniform((int)blockIdx.x / (a.Hkv * tiles)), share = (int)blockIdx.x - item * a.Hkv * tiles;
  const AtItem it = at_find<false, false>(a, item);
  if (it.b < 0) return;  // (all waves)
  const int h = uniform(share / tiles), g0 = share % tiles * AT_ROWS, dh = FULL ? DH : a.dh;
  const int rows = g - g0 < AT_ROWS ? g - g0 : AT_ROWS, head0 = h * g + g0;
  const int k_first = it.index * it.C, k_end = at_item_end(it);  // (C is a multiple of the block)
  // this lane's query head as an operand column
  at_u4 q[KP];
  {
    const int head = head0 + (c16 < rows ? c16 : 0);
    const char *qp = (const char *)a.q + (a.q_tiles ? (((int64_t)head * a.q_tiles + (it.b >> 4)) * (dh / 32) * 64 + (it.b & 15)) * 16 : (it.b * a.ldq + (int64_t)head * dh) * E);
#pragma unroll
    for (int i = 0; i < KP; ++i) {
      const int at = 64 * i + 16 * q4;
      q[i] = FULL || at < dh * E ? *(const at_u4 *)(qp + (a.q_tiles ? 1024 * i + 256 * q4 : at)) : at_u4{0, 0, 0, 0};
    }
  }
  const float to_log2 = a.scale * AT_LOG2E;
  const int row_bytes = dh * E;
  const int32_t *tab = a.table + it.r * a.ldt;
  const int n_blocks = (int)(((unsigned)(k_end - k_first) + KEYS - 1u) / KEYS), mine = n_blocks > wave ? (n_blocks - wave + WAVES - 1) / WAVES : 0;
  // Where the tiles lie: PAGED16: lane i holds byte offset and number of keys of tile i of the next 64 of this wave; else lane j < KEYS the offset of key j of the block, -1: none.
  unsigned off_lo = 0, off_hi = 0;
  int n_keys = 0;
  auto place = [&](long long key) {  // byte offset of the key's row, -1: not in a page
    const int block = (int)key / a.page, pg = tab[block];
    return (unsigned)pg < (unsigned)a.n_pages ? (((long long)pg * a.Hkv + h) * a.page + ((int)key - block * a.page)) * row_bytes : -1ll;
  };
  auto look_up = [&](int i) {  // for block i of this wave
    if (PAGED16 ? i % (64 / TILES) == 0 : true) {
      const long long key = PAGED16 ? k_first + (long long)KEYS * (wave + (long long)WAVES * (i + lane / TILES)) + 16 * (lane % TILES)
                                    : k_first + (long long)KEYS * (wave + (long long)WAVES * i) + lane;
      long long at = -1;
      if (key < k_end && (PAGED16 || lane < KEYS)) at = place(key);
      off_lo = (unsigned)at;
      off_hi = (unsigned)(at >> 32);
      if (PAGED16) n_keys = at < 0 ? 0 : k_end - key < 16 ? (int)(k_end - key) : 16;
    }
  };
  at_u4 kr[TILES][KP];
  unsigned vr[VK][VH][VW / 4];
  const char *kb = (const char *)a.K, *vb = (const char *)a.V;
  unsigned seen = 0;  // bit j: key j of the block whose K is in the registers
  long long tile_at[TILES];  // PAGED16
  auto locate = [&](int i) {
    seen = 0;
    if constexpr (PAGED16) {
#pragma unroll
      for (int t = 0; t < TILES; ++t) {
        const int l = i % (64 / TILES) * TILES + t, n = __builtin_amdgcn_readlane(n_keys, l);
        const long long at = (long long)(unsigned)__builtin_amdgcn_readlane((int)off_lo, l) | (long long)__builtin_amdgcn_readlane((int)off_hi, l) << 32;
        seen |= ((1u << n) - 1u) << (16 * t);
        tile_at[t] = n > 0 ? at : 0;
      }
    } else {
      seen = (unsigned)__ballot((int)off_hi >= 0) & (F32 ? 0xffffu : 0xffffffffu);
    }
  };
  // (a key that is not seen is read as the first row of all: its score and its V are replaced)
  auto key_at = [&](int j) {
    const unsigned lo = __shfl((int)off_lo, j, 64), hi = __shfl((int)off_hi, j, 64);
    return (int)hi < 0 ? 0ll : (long long)lo | (long long)hi << 32;
  };
  auto load = [](auto *p) {
    if constexpr (ONCE) return __builtin_nontemporal_load(p);
    else return *p;
  };
  auto load_k = [&]() {
#pragma unroll
    for (int t = 0; t < TILES; ++t) {
      const bool in = PAGED16 ? (seen >> (16 * t + c16)) & 1u : true;
      const char *p = kb + (PAGED16 ? tile_at[t] + (unsigned)((in ? c16 : 0) * row_bytes) : key_at(16 * t + c16));
#pragma unroll
      for (int i = 0; i < KP; ++i) {
        const int at = 64 * i + 16 * q4;
        const bool there = FULL || at < row_bytes;
        kr[t][i] = load((const at_u4 *)(p + (there ? at : 0)));
        if (!there) kr[t][i] = at_u4{0, 0, 0, 0};
      }
    }
  };
  auto load_v = [&]() {
#pragma unroll
    for (int j = 0; j < VK; ++j) {
      const int t = j >> 2, key = 4 * q4 + (j & 3);
      const bool in = (seen >> (16 * t + key)) & 1u;
      const char *p = vb + (PAGED16 ? tile_at[t] + (unsigned)((in ? key : 0) * row_bytes) : key_at(16 * t + key));
#pragma unroll
      for (int u = 0; u < VH; ++u) {
        const int at = 16 * VW * u + VW * c16;
        const char *from = p + (FULL || at < row_bytes ? at : 0);  // (channels behind the row's end are never stored)
        if constexpr (VW == 16) *(at_u4 *)vr[j][u] = load((const at_u4 *)from);
        else *(at_u2 *)vr[j][u] = load((const at_u2 *)from);
      }
    }
  };
  at_f4 o[DT];
#pragma unroll
  for (int d = 0; d < DT; ++d) o[d] = at_f4{0.f, 0.f, 0.f, 0.f};
  float m_run = -INFINITY, l_run = 0.f;
  if (mine > 0) {
    look_up(0);
    locate(0);
    load_k();
    load_v();
  }
  for (int i = 0; i < mine; ++i) {
    const unsigned now = seen;
    at_f4 s[TILES];
#pragma unroll
    for (int t = 0; t < TILES; ++t) {
      s[t] = at_f4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int k = 0; k < KP; ++k) {
        if constexpr (F32) {
#pragma unroll
          for (int e = 0; e < 4; ++e)
            s[t] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(kr[t][k][e]), __uint_as_float(q[k][e]), s[t], 0, 0, 0);
        } else {
          s[t] = at_mma<T>(kr[t][k], q[k], s[t]);
        }
      }
    }
    const unsigned all = F32 ? 0xffffu : 0xffffffffu;
    float mx = -INFINITY;
#pragma unroll
    for (int t = 0; t < TILES; ++t)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        s[t][e] *= to_log2;
        if (now != all && !((now >> (16 * t + 4 * q4 + e)) & 1u)) s[t][e] = -INFINITY;
        mx = fmaxf(mx, s[t][e]);
      }
    mx = at_max4(mx);
    const float m_new = fmaxf(m_run, mx), base = m_new > -INFINITY ? m_new : 0.f;
    if (__any(m_new > m_run)) {
      const float corr = __builtin_amdgcn_exp2f(m_run - base);
      m_run = m_new;
      l_run *= corr;
#pragma unroll
      for (int d = 0; d < DT; ++d) o[d] *= corr;
    }
#pragma unroll
    for (int t = 0; t < TILES; ++t)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        s[t][e] = __builtin_amdgcn_exp2f(s[t][e] - base + UP);
        l_run += s[t][e];
      }
    if (now != all) {
#pragma unroll
      for (int j = 0; j < VK; ++j)
        if (!((now >> (16 * (j >> 2) + 4 * q4 + (j & 3))) & 1u))
#pragma unroll
          for (int u = 0; u < VH; ++u)
#pragma unroll
            for (int w = 0; w < VW / 4; ++w) vr[j][u][w] = 0u;
    }
    if constexpr (F32) {
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int u = 0; u < VH; ++u)
#pragma unroll
          for (int w = 0; w < VC; ++w)
            o[u * VC + w] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(vr[e][u][w]), s[0][e], o[u * VC + w], 0, 0, 0);
    } else {
      at_u4 p, rest;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const at_u2 both = at_split<T>(s[j / 2 % TILES][2 * (j & 1)], s[j / 2 % TILES][2 * (j & 1) + 1]);
        p[j] = both[0];
        rest[j] = both[1];
      }
#pragma unroll
      for (int u = 0; u < VH; ++u)
#pragma unroll
        for (int w = 0; w < VW / 4; ++w)
#pragma unroll
          for (int half = 0; half < 2; ++half) {
            at_u4 v;
#pragma unroll
            for (int j = 0; j < 4; ++j)
              v[j] = __builtin_amdgcn_perm(vr[(2 * j + 1) % VK][u][w], vr[2 * j % VK][u][w], half ? 0x07060302u : 0x05040100u);
            o[u * VC + 2 * w + half] = at_mma<T>(v, rest, at_mma<T>(v, p, o[u * VC + 2 * w + half]));
          }
    }
    if (i + 1 < mine) {
      look_up(i + 1);
      locate(i + 1);
      load_k();
      load_v();
    }
  }
  l_run = at_sum4(l_run);
  // The waves' sums meet in LDS, a part of 16 VC channels at a time: [wave][row][channels + 4], and in front of them [wave][row] maximum and sum; a thread adds the waves'
  // sums of four channels, in order.  Output tile (u, w), lane, register e is channel 16 VC u + VC (4 q4 + e) + w.
  constexpr int PART = 16 * VC, PITCH = PART + 4, QUADS = PART / 4;
  float *stat = at_lds, *sums = at_lds + 2 * WAVES * AT_ROWS;
  if (q4 == 0) {
    stat[2 * (wave * AT_ROWS + c16)] = m_run;
    stat[2 * (wave * AT_ROWS + c16) + 1] = l_run;
  }
#pragma unroll
  for (int u = 0; u < VH; ++u) {
    if (u > 0) __syncthreads();
    if (c16 < rows) {
      float *to = sums + (size_t)(wave * rows + c16) * PITCH;
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int w = 0; w < VC; w += 4) {
          at_f4 v;
#pragma unroll
          for (int x = 0; x < 4; ++x) v[x] = o[u * VC + w + x][e];
          *(at_f4 *)(to + VC * (4 * q4 + e) + w) = v;
        }
    }
    __syncthreads();
    for (int i = threadIdx.x; i < rows * QUADS; i += 64 * WAVES) {
      const int row = i / QUADS, at = 4 * (i - row * QUADS), ch = PART * u + at, head = head0 + row;
      if (!FULL && ch >= dh) continue;
      float m = stat[2 * row];
#pragma unroll
      for (int w = 1; w < WAVES; ++w) m = fmaxf(m, stat[2 * (w * AT_ROWS + row)]);
      const float base = m > -INFINITY ? m : 0.f;
      float l = 0.f;
      at_f4 y = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < WAVES; ++w) {
        const float f = __builtin_amdgcn_exp2f(stat[2 * (w * AT_ROWS + row)] - base);
        l += stat[2 * (w * AT_ROWS + row) + 1] * f;
        y += *(const at_f4 *)(sums + (size_t)(w * rows + row) * PITCH + at) * f;
      }
      if (it.count > 1) {
        float *to = a.part + ((size_t)item * a.Hq + head) * a.rec;
        if (u == 0 && at == 0) *(float2 *)to = float2{m, l};
        *(at_f4 *)(to + 4 + ch) = y;
        continue;
      }
      y *= l > 0.f || l != l ? 1.f / l : 0.f;  // (nothing seen: zeros)
      if (a.kind != AT_OUT_ROWS) {
#pragma unroll
        for (int x = 0; x < 4; ++x) at_store_row(a, it.b, head * dh + ch + x, y[x]);
      } else {
        T *to = (T *)a.out + it.b * a.ldo + (int64_t)head * dh + ch;
        if constexpr (F32) *(at_f4 *)to = y;
        else *(at_u2 *)to = at_u2{at_pack<T>(y[0], y[1]), at_pack<T>(y[2], y[3])};
      }
    }
  }
}

// The items of a row and head, in item order: a workgroup each, whose waves take every fourth item; a lane takes up to four channels.  What it reads does not wait for what
// the rows' maxima are: they are applied to it.  5.6 to 6.2 us for 32 rows of 64 items together (1 MB of records): the rows' positions and the cut, formed anew by every workgroup, then two
// loads' latencies.
template <typename T>
__global__ __launch_bounds__(64 * AT_JOIN_WAVES) void paged_join_kernel(PagedAttend a) {
  __shared__ float sums[AT_JOIN_WAVES][256];
  const AtItem it = at_find<true, false>(a, blockIdx.x);
  if (it.count < 2) return;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, head = blockIdx.y;
  const size_t step = (size_t)a.Hq * a.rec;
  const float *rec = a.part + ((size_t)it.first * a.Hq + head) * a.rec;
  const int parts = (a.dh + 63) / 64;
  constexpr int N = 4;
  float v[N][4], s[N];  // channels lane, lane + 64, ... of items i0, i0 + AT_JOIN_WAVES, ...
  auto fetch = [&](int i0) {
#pragma unroll
    for (int k = 0; k < N; ++k) {
      const int i = i0 + AT_JOIN_WAVES * k < it.count ? i0 + AT_JOIN_WAVES * k : 0;
      s[k] = rec[i * step];
#pragma unroll
      for (int c = 0; c < 4; ++c) v[k][c] = c < parts ? rec[i * step + 4 + (lane + 64 * c < a.dh ? lane + 64 * c : 0)] : 0.f;
    }
  };
  fetch(wave);
  float m = -INFINITY, l = 0.f;
  for (int i0 = 0; i0 < it.count; i0 += 64) {
    const float2 s = i0 + lane < it.count ? *(const float2 *)(rec + (i0 + lane) * step) : float2{-INFINITY, 0.f};
    const float m_new = fmaxf(m, s.x), base = m_new > -INFINITY ? m_new : 0.f;
    l = l * __builtin_amdgcn_exp2f(m - base) + s.y * __builtin_amdgcn_exp2f(s.x - base);
    m = m_new;
  }
  float top = m;
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor(top, o, 64));
  const float base = top > -INFINITY ? top : 0.f;
  l *= __builtin_amdgcn_exp2f(m - base);
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) l += __shfl_xor(l, o, 64);
  float acc[4] = {0.f, 0.f, 0.f, 0.f};
  for (int i0 = wave; i0 < it.count; i0 += N * AT_JOIN_WAVES) {
    if (i0 > wave) fetch(i0);
#pragma unroll
    for (int k = 0; k < N; ++k) {
      const float f = i0 + AT_JOIN_WAVES * k < it.count ? __builtin_amdgcn_exp2f(s[k] - base) : 0.f;
#pragma unroll
      for (int c = 0; c < 4; ++c) acc[c] += f > 0.f || f != f ? v[k][c] * f : 0.f;
    }
  }
#pragma unroll
  for (int c = 0; c < 4; ++c) sums[wave][lane + 64 * c] = acc[c];
  __syncthreads();
  const float inv = l > 0.f || l != l ? 1.f / l : 0.f;
  for (int ch = threadIdx.x; ch < a.dh; ch += 64 * AT_JOIN_WAVES) {
    float y = sums[0][ch];
#pragma unroll
    for (int w = 1; w < AT_JOIN_WAVES; ++w) y += sums[w][ch];
    y *= inv;
    if (a.kind != AT_OUT_ROWS) {
      at_store_row(a, it.b, head * a.dh + ch, y);
      continue;
    }
    T *to = (T *)a.out + it.b * a.ldo + (int64_t)head * a.dh + ch;
    if constexpr (sizeof(T) == 4) *to = y;
    else *(uint16_t *)to = (uint16_t)at_pack<T>(y, 0.f);
  }
}

// ---- host side ------------------------------------------------------------------------------------------
// Where rows that are not cut leave every CU at most one workgroup (AT_WIDE), it has eight waves, 8 kv heads of 128 channels: one row of 300 7.9 -> 7.5 us, 16 rows of 500
// 10.4 -> 10.1, but 64 rows of 500 24.3 -> 26.4.
// ONCE where a layer's K and V pages are more than AT_CACHED bytes, in kernels whose loads are all of whole rows: two rows of 131072 (1.07 GB) 167 us, 189 without.  The pages' bytes, not
// those that the rows read, which only the device knows: a batch of 32 that reads 99 MB of a large pool has it too, 41.9 us (39.5 in a pool of its own size) where other work went through the
// caches in between, 36.6 (29.8) where its keys would stay cached from call to call, which other layers' keys and weights prevent in a program.
constexpr int AT_WIDE = 256;
static AtPlan at_plan(const la_pages_desc &p, int Hq, int max_blocks, int B) { return at_plan(p.head_dim, p.n_kv_heads, p.page_size, Hq, max_blocks, B); }

template <typename T, int DH, bool PAGED16, bool FULL>
static int at_launch(const PagedAttend &a, const AtPlan &plan, hipStream_t s) {
  const int g = a.Hq / a.Hkv, rows = std::min(g, AT_ROWS);
  constexpr int VC = (DH * (int)sizeof(T) / 16 < 16 ? 8 : 16) / (int)sizeof(T);
  auto lds = [&](int waves) { return (2 * waves * AT_ROWS + waves * rows * (16 * VC + 4)) * 4; };  // (37 KB at most)
  const unsigned grid = (unsigned)plan.items * a.Hkv * plan.tiles;
  bool wide = false;
  if constexpr (DH <= 128) wide = plan.target == 0 && rows <= 8 && (long long)plan.items * a.Hkv * plan.tiles <= AT_WIDE;
  if (a.list) {
    ProfScope ps("paged_plan", s);
    paged_plan_kernel<false><<<1, AT_PLAN_THREADS, 0, s>>>(a, plan.items);
  }
  {
    ProfScope ps("paged_attend", s);
    bool once = false;
    if constexpr (PAGED16 && FULL) once = 2 * (size_t)a.n_pages * a.Hkv * a.page * a.dh * sizeof(T) > AT_CACHED;
    if constexpr (DH <= 128)
      if (wide) paged_attend_kernel<T, DH, PAGED16, FULL, AT_WHOLE_WAVES, false><<<grid, 64 * AT_WHOLE_WAVES, lds(AT_WHOLE_WAVES), s>>>(a);
    if constexpr (PAGED16 && FULL)
      if (!wide && once) paged_attend_kernel<T, DH, PAGED16, FULL, AT_WAVES, true><<<grid, 64 * AT_WAVES, lds(AT_WAVES), s>>>(a);
    if (!wide && !once) paged_attend_kernel<T, DH, PAGED16, FULL, AT_WAVES, false><<<grid, 64 * AT_WAVES, lds(AT_WAVES), s>>>(a);
  }
  if (plan.target > 0) {
    ProfScope ps("paged_join", s);
    paged_join_kernel<T><<<dim3(a.B, a.Hq), 64 * AT_JOIN_WAVES, 0, s>>>(a);
  }
  LA_HIP(hipGetLastError());
  return LA_OK;
}
template <typename T>
static int at_launch(const PagedAttend &a, const AtPlan &plan, hipStream_t s) {
  auto sized = [&](auto dh) {
    constexpr int DH = decltype(dh)::value;
    if constexpr (sizeof(T) == 4) {  // (not a type of large models: the one general kernel)
      return at_launch<T, DH, false, false>(a, plan, s);
    } else {
      const bool in16 = a.page % 16 == 0;
      if (a.dh == DH) return in16 ? at_launch<T, DH, true, true>(a, plan, s) : at_launch<T, DH, false, true>(a, plan, s);
      return in16 ? at_launch<T, DH, true, false>(a, plan, s) : at_launch<T, DH, false, false>(a, plan, s);
    }
  };
  if (a.dh <= 64) return sized(std::integral_constant<int, 64>{});
  if (a.dh <= 128) return sized(std::integral_constant<int, 128>{});
  return sized(std::integral_constant<int, 256>{});
}

static int at_run(PagedAttend a, int dtype, const AtPlan &plan, hipStream_t s) {
  if (plan.list) {
    a.list = (AtItem *)((char *)a.part + plan.list);
    a.firsts = (int32_t *)(a.list + plan.items);
  }
  if (dtype == LA_F32) return at_launch<float>(a, plan, s);
  if (dtype == LA_F16) return at_launch<_Float16>(a, plan, s);
  return at_launch<uint16_t>(a, plan, s);
}

size_t paged_attend_bytes(const la_pages_desc &p, int Hq, int B) { return at_plan(p, Hq, 0x7fffffff / p.page_size, B).bytes; }

int paged_attend_rows(const la_pages_desc &p, int layer, const void *q, int q_tiles, int Hq, float scale, const PagedRows &r, PagedOut kind, void *out, void *workspace,
                      hipStream_t s) {
  const size_t at = layer * layer_bytes(&p);
  const int64_t ld = (int64_t)Hq * p.head_dim;
  const AtPlan plan = at_plan(p, Hq, r.max_blocks, r.B);
  const PagedAttend a{(const char *)p.k + at, (const char *)p.v + at, p.n_pages, p.page_size, p.n_kv_heads, p.head_dim, q, ld, Hq, scale, r.table, r.ldt,
                      r.n_req, r.max_blocks, r.req, r.pos, r.B, out, ld, plan.target, q_tiles, kind, p.head_dim + 4, (float *)workspace, nullptr, nullptr};
  return at_run(a, p.dtype, plan, s);
}

}  // namespace la

using namespace la;

extern "C" size_t la_paged_attend_workspace(const la_pages_desc *pages, int n_q_heads, int max_blocks, int B) {
  if (check_pages(pages, 0) || n_q_heads < 1 || n_q_heads % pages->n_kv_heads || max_blocks < 1 || B < 1) return 0;  // (what the call itself refuses)
  return at_plan(*pages, n_q_heads, max_blocks, B).bytes;
}

extern "C" int la_paged_attend(const la_pages_desc *pages, int layer, const void *q, int64_t q_stride, int n_q_heads, float scale, const int32_t *table,
                               int64_t table_stride, int n_requests, int max_blocks, const int32_t *req, const int32_t *pos, int B, void *out, int64_t out_stride,
                               void *workspace, size_t workspace_bytes, void *stream) {
  if (const int rc = check_pages(pages, layer)) return rc;
  const la_pages_desc &p = *pages;
  const size_t e = esize(&p);
  LA_REQUIRE(B >= 0, LA_EINVAL, "B=%d is negative", B);
  if (B == 0) return LA_OK;
  LA_REQUIRE(q && table && pos && out, LA_EINVAL, "NULL argument");
  LA_REQUIRE(n_q_heads > 0 && n_q_heads % p.n_kv_heads == 0, LA_EINVAL, "n_q_heads %d is not a multiple of n_kv_heads %d", n_q_heads, p.n_kv_heads);
  LA_REQUIRE(n_requests >= 1 && max_blocks >= 1 && (table_stride >= max_blocks || n_requests == 1), LA_EINVAL, "bad table dimensions");
  LA_REQUIRE((long long)max_blocks * p.page_size < (1ll << 31), LA_EINVAL, "%d blocks of %d positions: positions are 32-bit numbers", max_blocks, p.page_size);
  LA_REQUIRE(req || B <= n_requests, LA_EINVAL, "%d rows for %d requests and no row map", B, n_requests);
  LA_REQUIRE(B <= LA_MAX_ATTEND_ROWS && n_q_heads <= 65535, LA_EINVAL, "%d rows of %d heads, at most %d of 65535", B, n_q_heads, LA_MAX_ATTEND_ROWS);
  LA_REQUIRE(aligned16({q, out}) && q_stride * e % 16 == 0 && out_stride * e % 16 == 0, LA_EINVAL, "q and out rows must be 16-byte aligned");
  LA_REQUIRE(scale - scale == 0.f, LA_EINVAL, "scale is not finite");
  const AtPlan plan = at_plan(p, n_q_heads, max_blocks, B);
  LA_REQUIRE((long long)plan.items * p.n_kv_heads * plan.tiles < 1ll << 24, LA_EINVAL, "%d rows of %d kv heads are more than one launch takes", B, p.n_kv_heads);  // (2^32 threads)
  LA_REQUIRE(workspace_bytes >= plan.bytes && (workspace || !plan.bytes), LA_ENOMEM, "workspace of %zu bytes, %zu needed", workspace_bytes, plan.bytes);
  LA_REQUIRE(aligned16({workspace}), LA_EINVAL, "workspace must be 16-byte aligned");
  hipStream_t s = (hipStream_t)stream;
  const size_t at = layer * layer_bytes(&p);
  const PagedAttend a{(const char *)p.k + at, (const char *)p.v + at, p.n_pages, p.page_size, p.n_kv_heads, p.head_dim, q, q_stride, n_q_heads, scale, table, table_stride,
                      n_requests, max_blocks, req, pos, B, out, out_stride, plan.target, 0, AT_OUT_ROWS, p.head_dim + 4, (float *)workspace, nullptr, nullptr};
  return at_run(a, p.dtype, plan, s);
}
