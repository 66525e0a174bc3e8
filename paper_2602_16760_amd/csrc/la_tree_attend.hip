// Attention of trees of drafted tokens over the pages of their requests (la_paged_tree_attend).
#include <algorithm>

#include "la_tree.h"

namespace la {

constexpr int TA_WAVES = 4, TA_WHOLE_WAVES = 8;  // of a workgroup; where requests are not cut and workgroups are few

// A row i of request r at position p sees the committed keys 0 .. len - 1 and row j of its block, at key len + j, where bit j of vis is set:
//   out_i = sum_k w_k V_k / sum_k w_k,  w_k = 2^(log2(e) scale q_i K_k - m),  m a column's offset, which the factor cancels.
// One pass over K and V: m follows the largest score (la_tree.h), the sum and the output's sums are rescaled when it moves.
// A workgroup takes an item's keys for one kv head and 16 of its columns; column c of a kv head is query head c % g of the request's row c / g, so that those of a block of few rows lie
// together and a small tree is one or two matrix operands wide.  The waves take blocks of KEYS keys in turn and meet once, at the end: no barrier in the loop, K and V straight to registers, the
// next block's K asked for under this one's V.  Products, types and pages as in la_attend.hip.  Bound by latency: one tree of eight rows and two query heads a kv head at 500 keys, 10.2 us of
// which a launch is 3.8; the rest is a chain of offset, page, K, V, and the waves' meeting.
template <typename T, int DH, bool FAST, int WAVES, bool ONCE>
__global__ __launch_bounds__(64 * WAVES) void tree_attend_kernel(TreeAttend a) {
  constexpr bool F32 = sizeof(T) == 4;
  constexpr int E = sizeof(T), TILES = F32 ? 1 : 2, KEYS = 16 * TILES;
  constexpr int KP = DH * E / 64;                  // 16-byte pieces of a key row per lane (four lanes a row)
  constexpr int VW = DH * E / 16 < 16 ? 8 : 16;    // bytes of a V load: a row's share of each of 16 lanes, at most 16
  constexpr int VH = DH * E / 16 / VW;             // such loads a row
  constexpr int VC = VW / E;                       // channels of one
  constexpr int DT = DH / 16;                      // tiles of the output: channel VH-th part, one of VC
  constexpr int VK = 4 * TILES;                    // keys whose V a lane loads
  constexpr float UP = TA_UP<T>, LAZY = TA_LAZY<T>;
  extern __shared__ __attribute__((aligned(16))) float at_lds[];
  const int wave = uniform((int)(threadIdx.x >> 6)), lane = threadIdx.x & 63, q4 = lane >> 4, c16 = lane & 15;
  const int g = uniform(a.Hq / a.Hkv), dh = FAST ? DH : a.dh;
  int item, h, tile;
  ta_share(a, (int)blockIdx.x, item, h, tile);
  ta_zero_outside<T>(a, 64 * WAVES);
  if (item < 0) return;
  const AtItem it = at_find<false, true>(a, item);
  if (it.b < 0) return;  // (all waves)
  ta_note(a, it, h, tile);
  int f0;
  const int n_rows = uniform(tree_rows(a, it.b, f0)), first = uniform(f0), L = uniform(a.len[it.b]);
  if (it.index == 0 && tile == 0) ta_zero_behind<T>(a, it.b, first, n_rows, h * g * dh, g * dh, 64 * WAVES);
  const int cols = n_rows * g - 16 * tile;  // of this workgroup, if it had room for all
  if (cols <= 0) return;
  const int k_first = it.index * it.C, k_end = at_item_end(it);  // (C is a multiple of the block)
  // this lane's column: its row of all, and the query head
  const int col = 16 * tile + (c16 < cols ? c16 : 0), col_row = first + col / g, col_head = h * g + col % g;
  at_u4 q[KP];
  {
    const char *qp = (const char *)a.q + (a.q_tiles ? (((int64_t)col_head * a.q_tiles + (col_row >> 4)) * (dh / 32) * 64 + (col_row & 15)) * 16 : (col_row * a.ldq + (int64_t)col_head * dh) * E);
#pragma unroll
    for (int p = 0; p < KP; ++p) {
      const int at = 64 * p + 16 * q4;
      q[p] = FAST || at < dh * E ? *(const at_u4 *)(qp + (a.q_tiles ? 1024 * p + 256 * q4 : at)) : at_u4{0, 0, 0, 0};
    }
    if (a.scale < 0.f)  // (scores are multiplied by what is not negative: the largest stays the largest)
#pragma unroll
      for (int p = 0; p < KP; ++p) q[p] ^= F32 ? 0x80000000u : 0x80008000u;
  }
  const float to_log2 = fabsf(a.scale) * AT_LOG2E;
  const int row_bytes = dh * E;
  const int32_t *tab = a.table + it.r * a.ldt;
  const int n_blocks = (int)(((unsigned)(k_end - k_first) + KEYS - 1u) / KEYS), mine = n_blocks > wave ? (n_blocks - wave + WAVES - 1) / WAVES : 0;
  // Where the tiles lie: FAST: lane i holds byte offset and number of keys of tile i of the next 64 of this wave; else lane j < KEYS the offset of key j of the block, -1: none.
  unsigned off_lo = 0, off_hi = 0;
  int n_keys = 0;
  auto place = [&](long long key) {  // byte offset of the key's row, -1: not in a page
    const int block = (int)key / a.page, pg = tab[block];
    return (unsigned)pg < (unsigned)a.n_pages ? (((long long)pg * a.Hkv + h) * a.page + ((int)key - block * a.page)) * row_bytes : -1ll;
  };
  auto look_up = [&](int i) {  // for block i of this wave
    if (FAST ? i % (64 / TILES) == 0 : true) {
      const long long key = FAST ? k_first + (long long)KEYS * (wave + (long long)WAVES * (i + lane / TILES)) + 16 * (lane % TILES)
                                 : k_first + (long long)KEYS * (wave + (long long)WAVES * i) + lane;
      long long at = -1;
      if (key < k_end && (FAST || lane < KEYS)) at = place(key);
      off_lo = (unsigned)at;
      off_hi = (unsigned)(at >> 32);
      if (FAST) n_keys = at < 0 ? 0 : k_end - key < 16 ? (int)(k_end - key) : 16;
    }
  };
  at_u4 kr[TILES][KP];
  unsigned vr[VK][VH][VW / 4];
  const char *kb = (const char *)a.K, *vb = (const char *)a.V;
  unsigned seen = 0;  // bit j: key j of the block is in a page
  long long tile_at[TILES];  // FAST
  auto locate = [&](int i) {
    seen = 0;
    if constexpr (FAST) {
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
      const bool in = FAST ? (seen >> (16 * t + c16)) & 1u : true;
      const char *p = kb + (FAST ? tile_at[t] + (unsigned)((in ? c16 : 0) * row_bytes) : key_at(16 * t + c16));
#pragma unroll
      for (int i = 0; i < KP; ++i) {
        const int at = 64 * i + 16 * q4;
        const bool there = FAST || at < row_bytes;
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
      const char *p = vb + (FAST ? tile_at[t] + (unsigned)((in ? key : 0) * row_bytes) : key_at(16 * t + key));
#pragma unroll
      for (int u = 0; u < VH; ++u) {
        const int at = 16 * VW * u + VW * c16;
        const char *from = p + (FAST || at < row_bytes ? at : 0);  // (channels behind the row's end are never stored)
        if constexpr (VW == 16) *(at_u4 *)vr[j][u] = load((const at_u4 *)from);
        else *(at_u2 *)vr[j][u] = load((const at_u2 *)from);
      }
    }
  };
  at_f4 o[DT];
#pragma unroll
  for (int d = 0; d < DT; ++d) o[d] = at_f4{0.f, 0.f, 0.f, 0.f};
  float m_run = -INFINITY, l_run = 0.f;
  bool far = false;
  if (mine > 0) {
    look_up(0);
    locate(0);
    load_k();
    load_v();
  }
  const unsigned long long vis = a.vis[col_row];  // (asked for here, behind the first keys: where it is needed first, at the request's end, everybody would wait for it)
  unsigned long long odd_rows = 0;  // drafted rows, of those whose keys this wave has, whose V has an infinity or NaN
  constexpr unsigned ALL = F32 ? 0xffffu : 0xffffffffu;
  for (int i = 0; i < mine; ++i) {
    const unsigned now = seen;
    const int key0 = k_first + KEYS * (wave + WAVES * i);
    const bool drafted = (long long)key0 + KEYS > L;  // keys of the request's own rows among them
    at_f4 s[TILES];
#pragma unroll
    for (int t = 0; t < TILES; ++t) {
      s[t] = at_f4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int k = 0; k < KP; ++k) {
        if constexpr (F32) {
#pragma unroll
          for (int e = 0; e < 4; ++e) s[t] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(kr[t][k][e]), __uint_as_float(q[k][e]), s[t], 0, 0, 0);
        } else {
          s[t] = at_mma<T>(kr[t][k], q[k], s[t]);
        }
      }
    }
    float factor = to_log2;
    unsigned odd = 0;  // such keys of the block
    if (drafted || now != ALL) {
      factor = 1.f;
      unsigned mask = now;  // keys that the column sees
      if (drafted) {
        const int at = key0 - L;  // of the block's first key in the request's rows
        mask &= at >= 0 ? (at < 64 ? (unsigned)(vis >> at) : 0u) : (unsigned)(vis << -at) | ((1u << -at) - 1u);  // (at > -KEYS)
      }
      mask >>= 4 * q4;
#pragma unroll
      for (int t = 0; t < TILES; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) s[t][e] = mask >> (16 * t + e) & 1u ? s[t][e] * to_log2 : -INFINITY;
      if (drafted) {
#pragma unroll
        for (int j = 0; j < VK; ++j) {
          bool any = false;
#pragma unroll
          for (int u = 0; u < VH; ++u)
#pragma unroll
            for (int w = 0; w < VW / 4; ++w) any = any || ((FAST || 16 * VW * u + VW * c16 < row_bytes) && ta_odd<T>(vr[j][u][w]));
          const unsigned long long lanes = __ballot(any);
#pragma unroll
          for (int x = 0; x < 4; ++x) odd |= (lanes >> (16 * x) & 0xffff) != 0 ? 1u << (16 * (j >> 2) + 4 * x + (j & 3)) : 0u;
        }
        odd &= now;
        const int committed = L - key0;  // (their infinities are seen by every row that sees anything)
        if (committed > 0) odd &= ~((1u << committed) - 1u);  // (< KEYS)
        odd_rows |= committed > 0 ? (unsigned long long)odd >> committed : (unsigned long long)odd << -committed;
      }
      const unsigned zero = ~now | odd;
#pragma unroll
      for (int j = 0; j < VK; ++j)
        if (zero >> (16 * (j >> 2) + 4 * q4 + (j & 3)) & 1u)
#pragma unroll
          for (int u = 0; u < VH; ++u)
#pragma unroll
            for (int w = 0; w < VW / 4; ++w) vr[j][u][w] = 0u;
    }
    if (i + 1 < mine) {
      look_up(i + 1);
      locate(i + 1);
      load_k();
    }
    float mx = -INFINITY;
#pragma unroll
    for (int t = 0; t < TILES; ++t)
#pragma unroll
      for (int e = 0; e < 4; ++e) mx = fmaxf(mx, s[t][e]);
    mx *= factor;
    if (__any(mx > m_run + LAZY)) {
      const float m_new = fmaxf(m_run, at_max4(mx)), corr = __builtin_amdgcn_exp2f(m_run - (m_new > -INFINITY ? m_new : 0.f));
      m_run = m_new;
      far = ta_far(m_new);
      l_run *= corr;
#pragma unroll
      for (int d = 0; d < DT; ++d) o[d] *= corr;
    }
    const float base = m_run > -INFINITY ? m_run : 0.f;
    float by = factor, add = UP - base;
    if (far) {
#pragma unroll
      for (int t = 0; t < TILES; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) s[t][e] = ta_exponent<T>(s[t][e], factor, base);
      by = 1.f;
      add = 0.f;
    }
#pragma unroll
    for (int t = 0; t < TILES; ++t)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        s[t][e] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[t][e], by, add));
        l_run += s[t][e];
      }
    if constexpr (F32) {
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int u = 0; u < VH; ++u)
#pragma unroll
          for (int w = 0; w < VC; ++w) o[u * VC + w] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(vr[e][u][w]), s[0][e], o[u * VC + w], 0, 0, 0);
    } else {
      at_u4 p, rest;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const at_u2 both = ta_split<T>(s[j / 2 % TILES][2 * (j & 1)], s[j / 2 % TILES][2 * (j & 1) + 1]);
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
    if (i + 1 < mine) load_v();
  }
  // Those V's, which the products took as zeros (a weight of zero would have made NaN of them in every column), for the columns that see them alone.
  for (; odd_rows; odd_rows &= odd_rows - 1) {
    const int row = __builtin_ctzll(odd_rows);
    const long long at = place((long long)L + row);
    at_f4 score = {0.f, 0.f, 0.f, 0.f};  // (added up as the tile's were: the weight has to be the one in the sum)
#pragma unroll
    for (int i = 0; i < KP; ++i) {
      const int b = 64 * i + 16 * q4;
      at_u4 k = *(const at_u4 *)(kb + at + (FAST || b < row_bytes ? b : 0));
      if (!FAST && b >= row_bytes) k = at_u4{0, 0, 0, 0};
      if constexpr (F32) {
#pragma unroll
        for (int e = 0; e < 4; ++e) score = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(k[e]), __uint_as_float(q[i][e]), score, 0, 0, 0);
      } else {
        score = at_mma<T>(k, q[i], score);
      }
    }
    const float p = __builtin_amdgcn_exp2f(ta_from(score[0], to_log2, m_run > -INFINITY ? m_run : 0.f) + UP) * (1.f + TA_REST<T>);
    if (!(vis >> row & 1u)) continue;
#pragma unroll
    for (int u = 0; u < VH; ++u)
#pragma unroll
      for (int w = 0; w < VC; ++w)
#pragma unroll
        for (int y = 0; y < 4; ++y) {
          const int ch = 16 * VC * u + VC * (4 * q4 + y) + w;
          if (FAST || ch < dh) o[u * VC + w][y] += p * load_as_float<T>((const T *)(vb + at) + ch);
        }
  }
  if (vis == 0) {  // (zeros, whatever was multiplied)
    m_run = -INFINITY;
    l_run = 0.f;
#pragma unroll
    for (int d = 0; d < DT; ++d) o[d] = at_f4{0.f, 0.f, 0.f, 0.f};
  }
  // The waves' sums meet in LDS, a part of 16 VC channels at a time: [wave][column][channels + 4], and in front of them [wave][column] offset and sum; a thread adds the waves' sums of four
  // channels, in order.  Output tile (u, w), lane, register e is channel 16 VC u + VC (4 q4 + e) + w.
  constexpr int PART = 16 * VC, PITCH = PART + 4, QUADS = PART / 4;
  float *stat = at_lds, *sums = at_lds + 2 * WAVES * AT_ROWS;
  const int columns = cols < 16 ? cols : 16;
  const float l = at_sum4(l_run) * (1.f + TA_REST<T>);
  if (q4 == 0) {
    stat[2 * (wave * AT_ROWS + c16)] = m_run;
    stat[2 * (wave * AT_ROWS + c16) + 1] = l;
  }
#pragma unroll
  for (int u = 0; u < VH; ++u) {
    if (u > 0) __syncthreads();
    if (c16 < columns) {
      float *to = sums + (size_t)(wave * AT_ROWS + c16) * PITCH;
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
    for (int x = threadIdx.x; x < columns * QUADS; x += 64 * WAVES) {
      const int row = x / QUADS, at = 4 * (x - row * QUADS), ch = PART * u + at, c = 16 * tile + row, j = c / g, head = h * g + c - j * g;
      if (!FAST && ch >= dh) continue;
      float m = stat[2 * row];
#pragma unroll
      for (int w = 1; w < WAVES; ++w) m = fmaxf(m, stat[2 * (w * AT_ROWS + row)]);
      const float base = m > -INFINITY ? m : 0.f;
      float sum = 0.f;
      at_f4 y = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < WAVES; ++w) {
        const float f = __builtin_amdgcn_exp2f(stat[2 * (w * AT_ROWS + row)] - base);
        sum += stat[2 * (w * AT_ROWS + row) + 1] * f;
        y += *(const at_f4 *)(sums + (size_t)(w * AT_ROWS + row) * PITCH + at) * f;
      }
      if (it.count > 1) {
        float *to = a.part + (((size_t)it.record * a.Hq + head) * a.max_rows + j) * a.rec;
        if (u == 0 && at == 0) *(float2 *)to = float2{m, sum};
        *(at_f4 *)(to + 4 + ch) = y;
        continue;
      }
      y *= sum > 0.f || sum != sum ? 1.f / sum : 0.f;  // (nothing seen: zeros)
      if (a.kind != AT_OUT_ROWS) {
#pragma unroll
        for (int z = 0; z < 4; ++z) at_store_row(a, first + j, head * dh + ch + z, y[z]);
      } else {
        T *to = (T *)a.out + (first + j) * a.ldo + (int64_t)head * dh + ch;
        if constexpr (F32) *(at_f4 *)to = y;
        else *(at_u2 *)to = at_u2{at_pack<T>(y[0], y[1]), at_pack<T>(y[2], y[3])};
      }
    }
  }
}

// The items of a request's row and query head, in item order: a wave each, a lane takes up to four channels.  Eight records at a time are on their way, since a wave's reads are a chain (one after
// the other 16 requests' join took 8 us, so 5).  Bound by the records' bytes where they are many: two requests of 64 rows at 65000 keys leave 34 KB an item and kv head, 10 us.
constexpr int TA_JOIN_WAVES = 4;
template <typename T, int PARTS, bool SPLIT>
__global__ __launch_bounds__(64 * TA_JOIN_WAVES) void tree_join_kernel(TreeAttend a) {
  const int lane = threadIdx.x & 63, wave = uniform((int)(threadIdx.x >> 6)), head = SPLIT ? (int)blockIdx.y : (int)blockIdx.y * TA_JOIN_WAVES + wave;
  const int r = uniform((int)(blockIdx.x / a.max_rows)), j = (int)blockIdx.x - r * a.max_rows;
  int first;
  const int2 note = a.notes[r];
  const int n_rows = tree_rows(a, r, first), all = note.y;
  if (all < 2 || j >= n_rows || head >= a.Hq) return;  // (SPLIT: all waves)
  const int own = SPLIT ? (all + TA_JOIN_WAVES - 1) / TA_JOIN_WAVES : all, skip = SPLIT ? wave * own : 0, count = all - skip < own ? all - skip : own;  // this wave's records
  const size_t step = (size_t)a.Hq * a.max_rows * a.rec;
  const float *rec = a.part + (((size_t)(note.x + skip) * a.Hq + head) * a.max_rows + j) * a.rec;
  const bool sees = a.vis[first + j] != 0;
  float top = -INFINITY, l = 0.f, acc[PARTS] = {};
  constexpr int N = 8;
  for (int i0 = 0; i0 < count; i0 += N) {
    float v[N][PARTS], m[N], s[N], most = top;
#pragma unroll
    for (int k = 0; k < N; ++k) {
      const float *p = rec + (i0 + k < count ? i0 + k : i0) * step;
      m[k] = p[0];
      s[k] = i0 + k < count ? p[1] : 0.f;
#pragma unroll
      for (int c = 0; c < PARTS; ++c) v[k][c] = p[4 + (lane + 64 * c < a.dh ? lane + 64 * c : 0)];
    }
#pragma unroll
    for (int k = 0; k < N; ++k) most = fmaxf(most, m[k]);
    const float base = most > -INFINITY ? most : 0.f, corr = __builtin_amdgcn_exp2f(top - base);
    top = most;
    l *= corr;
#pragma unroll
    for (int c = 0; c < PARTS; ++c) acc[c] *= corr;
#pragma unroll
    for (int k = 0; k < N; ++k) {
      const float f = i0 + k < count ? __builtin_amdgcn_exp2f(m[k] - base) : 0.f;
      l += s[k] * f;  // (scores that are all NaN leave an offset of -inf and a sum of NaN)
      if (!(f > 0.f || f != f)) continue;
#pragma unroll
      for (int c = 0; c < PARTS; ++c) acc[c] += v[k][c] * f;
    }
  }
  if constexpr (SPLIT) {  // the waves' sums, in order
    __shared__ float sums[TA_JOIN_WAVES][PARTS + 2][64];
#pragma unroll
    for (int c = 0; c < PARTS; ++c) sums[wave][c][lane] = acc[c];
    sums[wave][PARTS][lane] = top;
    sums[wave][PARTS + 1][lane] = l;
    __syncthreads();
    if (wave > 0) return;
    float most = top;
    for (int w = 1; w < TA_JOIN_WAVES; ++w) most = fmaxf(most, sums[w][PARTS][lane]);
    const float base = most > -INFINITY ? most : 0.f;
    l = 0.f;
#pragma unroll
    for (int c = 0; c < PARTS; ++c) acc[c] = 0.f;
    for (int w = 0; w < TA_JOIN_WAVES; ++w) {
      const float f = __builtin_amdgcn_exp2f(sums[w][PARTS][lane] - base);
      l += sums[w][PARTS + 1][lane] * f;
      if (!(f > 0.f || f != f)) continue;
#pragma unroll
      for (int c = 0; c < PARTS; ++c) acc[c] += sums[w][c][lane] * f;
    }
  }
  const float inv = sees && (l > 0.f || l != l) ? 1.f / l : 0.f;
#pragma unroll
  for (int c = 0; c < PARTS; ++c) {
    const int ch = lane + 64 * c;
    if (ch >= a.dh) continue;
    const float y = sees ? acc[c] * inv : 0.f;
    if (a.kind != AT_OUT_ROWS) {
      at_store_row(a, first + j, head * a.dh + ch, y);
      continue;
    }
    T *to = (T *)a.out + (first + j) * a.ldo + (int64_t)head * a.dh + ch;
    if constexpr (sizeof(T) == 4) *to = y;
    else *(uint16_t *)to = (uint16_t)at_pack<T>(y, 0.f);
  }
}

// ---- host side ------------------------------------------------------------------------------------------
// Which kernel, and what is cut; each rule with both sides as measured, in microseconds, 32 query heads of 128 channels unless said.
// TA_FEW: where no request is cut and workgroups of 16 columns are no more than the CUs, eight waves share a workgroup's keys (1 tree of 8 rows at 500 keys: 11.7, with four waves 14.7; 1 of 16:
//   13.5 and 16.4).  More than 32 columns, or more workgroups, go through LDS.
// Wide from 17 columns: 1 x 8 rows at 1000, 11.7 and with the other kernel 14.4; at 2000, 13.7 and 16.2; 8 x 8 at 4000, 35.8 both; 2 x 57 at 19000 with pages of 8, 50 and 134.  At 16 columns and
// fewer three quarters of its waves would idle.
constexpr int TA_FEW = 256;
// Requests are left whole up to AT_WHOLE keys (16 x 16 rows at 400: 16.4, cut 21.4; 16 x 64 at 500: 35 and 46), float ones up to half as many, their products being 1/16 as fast (3 x 8 at 500: cut
//   11.0, 13.5 whole).  Where wide workgroups of whole requests are fewer than TA_MANY, only up to TA_WHOLE_WIDE keys (1 x 64 at 500: cut 23, 34 whole; 4 x 16 at 500, 64 workgroups: 18.6 whole and
//   cut 16.5, but 4 x 32 at 600, 22.6 and 26.5), and so always for heads of 256 channels (22 of 1 to 12 rows at up to 747: cut 21, whole 34; one row at 500 14.3 and 18.3).
constexpr int TA_WHOLE_WIDE = 256, TA_MANY = 64;
// 128 columns a workgroup rather than 64 (K and V pass through LDS half as often) where one of 512 then has this many keys, if all requests are as long as the table: 4 x 64 rows at 500, 128
//   columns 26.4 and 64 20.0, 1 x 40 at 3000, 28.9 and 23.5, 4 x 64 at 4000, 512 keys, 49.9 and 48.3, 4 x 40 of three heads of 96 channels at 16000, 930 keys, 57.4 and 64.5, 16 x 64 at 4000,
//   2000 keys, 129 and 134, 4 x 64 at 16000, 119 and 134, 2 x 64 at 65000, 230 and 284.  Heads of 256 channels (one of 16 query heads), one workgroup a CU: 1 x 10 at 15800,
//   38 keys, 28.5 and 26.9, 8 x 33 at 2000, 129 keys, 38.2 and 44.1, 4 x 30 at 5000, 146 keys, 39.6 and 42.2.
constexpr int TA_LONG = 768, TA_LONG_256 = 128;
// Workgroups that items are cut for: one of 64 columns a CU (16 of 1 to 16 rows at up to 4096, 25.5; 384 of them 27.4, 512 26.1; 32 x 16 rows at 2000 62, 75 and 69), or two where a request has
//   several and each keeps TA_SHARE keys (1 x 64 rows of 64 heads at 8000: 48.1, one 54.9; 1 x 40 at 3000, 117 keys: 23.5 and 21.9); two of 128; at_workgroups' for the kernel above.
constexpr int TA_SHARE = 256;
// Bytes of the items' records at most; fewer items keep to it.  A record is written and read again: 4 us and 10 us at 34 KB an item and kv head of two requests of 64 rows.
constexpr size_t TA_RECORDS = (size_t)64 << 20;
// The join's waves share a row's and head's records where a request may have that many items and rows and heads are fewer than waves that fill the chip: one row of 8 heads at 30000 keys 37.6, shared
//   21.0, 1 x 10 of 16 heads of 256 channels at 15800, 37.7 and 28.3, 1 x 8 of 32 at 4000, 17.8 and 16.1; from 8 or 4 items a request on: no difference; 2 x 64 of 32 heads: 231 both.
constexpr int TA_MANY_RECORDS = 16, TA_PAIRS = 2048;
struct TreePlan {
  int wide, waves, tiles, uncut, target, items;
  bool split;  // the join's waves share a row's records
  unsigned grid;
  size_t notes, list, bytes;
};
// Kernel, columns of a workgroup and workgroups of an item and kv head; how many items are resident at once.  cap: positions that the table has room for.
static TreePlan ta_shape(const la_pages_desc &p, int Hq, int max_rows, int R, long long cap) {
  TreePlan r{};
  const int columns = Hq / p.n_kv_heads * max_rows;
  const bool few = cap <= AT_WHOLE && p.head_dim <= 128 && columns <= 32 && (long long)R * p.n_kv_heads * ceil_div(columns, 16) <= TA_FEW;
  const double share = (double)R * p.n_kv_heads * columns * (double)cap / 512;  // columns times keys of one of 512 workgroups
  if (columns > 16 && !few && tree_wide(p.dtype, p.head_dim, p.page_size)) r.wide = columns > 64 && share >= 128. * (p.head_dim <= 128 ? TA_LONG : TA_LONG_256) ? 128 : 64;
  r.waves = few ? TA_WHOLE_WAVES : TA_WAVES;
  r.tiles = ceil_div(columns, r.wide ? r.wide : 16);
  const int groups = !r.wide ? at_workgroups(p.head_dim) : p.head_dim <= 128 && (r.wide == 128 || (r.tiles > 1 && share >= 64. * TA_SHARE)) ? 512 : 256;
  r.target = std::max(1, groups / (p.n_kv_heads * r.tiles));
  return r;
}
static TreePlan ta_plan(const la_pages_desc &p, int Hq, int max_blocks, int R, int max_rows) {
  const long long cap = (long long)max_blocks * p.page_size;
  TreePlan r = ta_shape(p, Hq, max_rows, R, cap);
  const int target = r.target;
  r.target = 0;
  const bool sparse = (long long)R * p.n_kv_heads * r.tiles < TA_MANY;
  r.uncut = p.head_dim > 128 || (r.wide && sparse) ? TA_WHOLE_WIDE : p.dtype == LA_F32 ? AT_WHOLE / 2 : AT_WHOLE;
  const bool whole = cap <= r.uncut;
  if (!whole) r.waves = TA_WAVES;
  if (!whole && sparse && p.dtype == LA_F32) r.uncut = std::min(r.uncut, TA_WHOLE_WIDE);  // (the join is launched anyway, and four waves have the keys: 1 x 8 rows at 402, 16.4 and 11.8)
  r.items = R;
  if (!whole) {
    const size_t record = (size_t)Hq * max_rows * (p.head_dim + 4) * 4;
    const long long pieces = R * ((cap + AT_PIECE - 1) / AT_PIECE);
    for (r.target = target;; r.target = r.target * 3 / 4) {
      const int cut = (2 * R > r.target ? AT_FINE : 1) * r.target;
      r.items = (int)std::min((long long)cut + R, pieces);
      r.bytes = std::min(r.items, 2 * cut) * record;  // (of requests that are cut: fewer than `cut`, with one item more than their share of `cut` each)
      if (r.bytes <= TA_RECORDS || r.target == 1) break;
    }
    r.split = std::min((long long)r.target, (cap + AT_PIECE - 1) / AT_PIECE) >= TA_MANY_RECORDS * (long long)R && (long long)R * max_rows * Hq < TA_PAIRS;
    r.notes = r.bytes;
    r.bytes += ((size_t)R * sizeof(int2) + 15) / 16 * 16;
    if (R > 64) {
      r.list = r.bytes;
      r.bytes += r.items * sizeof(AtItem) + (size_t)R * 4;
    }
  }
  const long long groups = (long long)r.items * p.n_kv_heads, grid = r.tiles > 1 ? (groups + 7) / 8 * 8 * r.tiles : groups;
  r.grid = grid < 1ll << 24 ? (unsigned)grid : 1u << 24;
  return r;
}

template <typename T, int DH, bool FAST, int WAVES, bool ONCE>
static int ta_launch(const TreeAttend &a, const TreePlan &plan, hipStream_t s) {
  constexpr int VC = (DH * (int)sizeof(T) / 16 < 16 ? 8 : 16) / (int)sizeof(T);
  constexpr int LDS = (2 * WAVES * AT_ROWS + WAVES * AT_ROWS * (16 * VC + 4)) * 4;
  if constexpr (LDS > 64 * 1024)
    if (const int rc = ta_allow_lds<tree_attend_kernel<T, DH, FAST, WAVES, ONCE>>(LDS)) return rc;
  tree_attend_kernel<T, DH, FAST, WAVES, ONCE><<<plan.grid, 64 * WAVES, LDS, s>>>(a);
  return LA_OK;
}
template <typename T, int DH, int WAVES>
static int ta_launch(const TreeAttend &a, const TreePlan &plan, hipStream_t s) {
  if constexpr (sizeof(T) == 2)
    if (a.dh == DH && a.page % 16 == 0) {
      if constexpr (WAVES == TA_WAVES)
        if (a.once) return ta_launch<T, DH, true, WAVES, true>(a, plan, s);
      return ta_launch<T, DH, true, WAVES, false>(a, plan, s);
    }
  return ta_launch<T, DH, false, WAVES, false>(a, plan, s);
}
template <typename T, int DH>
static int ta_launch(const TreeAttend &a, const TreePlan &plan, hipStream_t s) {
  if constexpr (DH <= 128)
    if (plan.waves == TA_WHOLE_WAVES) return ta_launch<T, DH, TA_WHOLE_WAVES>(a, plan, s);
  return ta_launch<T, DH, TA_WAVES>(a, plan, s);
}
template <typename T, bool SPLIT>
static void ta_join(const TreeAttend &a, int heads, hipStream_t s) {
  const dim3 grid((unsigned)a.B * a.max_rows, heads);
  if (a.dh <= 64) tree_join_kernel<T, 1, SPLIT><<<grid, 64 * TA_JOIN_WAVES, 0, s>>>(a);
  else if (a.dh <= 128) tree_join_kernel<T, 2, SPLIT><<<grid, 64 * TA_JOIN_WAVES, 0, s>>>(a);
  else tree_join_kernel<T, 4, SPLIT><<<grid, 64 * TA_JOIN_WAVES, 0, s>>>(a);
}
template <typename T>
static int ta_launch(const TreeAttend &a, const TreePlan &plan, hipStream_t s) {
  if (a.list) {
    ProfScope ps("tree_plan", s);
    paged_plan_kernel<true><<<1, AT_PLAN_THREADS, 0, s>>>(a, plan.items);
  }
  int rc;
  if (plan.wide) {
    ProfScope ps("tree_attend", s);
    rc = tree_attend_wide(a, std::is_same<T, _Float16>::value ? LA_F16 : LA_BF16, plan.wide, plan.grid, s);
  } else {
    ProfScope ps("tree_attend", s);
    rc = a.dh <= 64 ? ta_launch<T, 64>(a, plan, s) : a.dh <= 128 ? ta_launch<T, 128>(a, plan, s) : ta_launch<T, 256>(a, plan, s);
  }
  if (rc) return rc;
  if (plan.target > 0) {
    ProfScope ps("tree_join", s);
    if (plan.split) ta_join<T, true>(a, a.Hq, s);
    else ta_join<T, false>(a, ceil_div(a.Hq, TA_JOIN_WAVES), s);
  }
  LA_HIP(hipGetLastError());
  return LA_OK;
}
static int ta_run(TreeAttend a, int dtype, const TreePlan &plan, hipStream_t s) {
  a.target = plan.target;
  a.tiles = plan.tiles;
  a.items = plan.items;
  a.uncut = plan.uncut;
  // (32 x 8 rows at 4000, 537 MB: 98.9 us, kept 104; 16 x 8 at 16000 190 and 200; where two workgroups read what one of them has asked for it has to stay)
  a.once = plan.tiles == 1 && 2 * (size_t)a.n_pages * a.Hkv * a.page * a.dh * (dtype == LA_F32 ? 4 : 2) > AT_CACHED;
  a.rec = a.dh + 4;
  a.notes = plan.target > 0 ? (int2 *)((char *)a.part + plan.notes) : nullptr;
  if (plan.list) {
    a.list = (AtItem *)((char *)a.part + plan.list);
    a.firsts = (int32_t *)(a.list + plan.items);
  }
  if (dtype == LA_F32) return ta_launch<float>(a, plan, s);
  if (dtype == LA_F16) return ta_launch<_Float16>(a, plan, s);
  return ta_launch<uint16_t>(a, plan, s);
}

size_t tree_attend_bytes(const la_pages_desc &p, int Hq) {
  size_t most = 0;
  la_pages_desc d = p;
  for (int page : {16, 17})  // (a page size that the wide kernel takes, one that it does not; the longest table, for which the most items are resident)
    for (int rows = 1; rows <= LA_MAX_ROWS; ++rows) {
      d.page_size = page;
      const size_t record = (size_t)Hq * rows * (p.head_dim + 4) * 4;
      most = std::max(most, std::min(2 * AT_FINE * (size_t)ta_shape(d, Hq, rows, 1, 1ll << 62).target, std::max(TA_RECORDS / record, (size_t)2 * AT_FINE)) * record);
    }
  return most + LA_MAX_ROWS * sizeof(int2);
}
int tree_attend_rows(const la_pages_desc &p, int layer, const void *q, int q_tiles, int Hq, float scale, const PagedRows &r, PagedOut kind, void *out, void *workspace, hipStream_t s) {
  const size_t at = layer * layer_bytes(&p);
  const int64_t ld = (int64_t)Hq * p.head_dim;
  TreeAttend a{(const char *)p.k + at, (const char *)p.v + at, p.n_pages, p.page_size, p.n_kv_heads, p.head_dim, q, ld, Hq, scale, r.table, r.ldt, r.n_req, r.max_blocks,
               r.first, r.len, r.vis, r.max_rows, r.B, out, ld};
  a.q_tiles = q_tiles;
  a.kind = kind;
  a.part = (float *)workspace;
  return ta_run(a, p.dtype, ta_plan(p, Hq, r.max_blocks, r.n_req, r.max_rows), s);
}

}  // namespace la

using namespace la;

extern "C" size_t la_paged_tree_attend_workspace(const la_pages_desc *pages, int n_q_heads, int max_blocks, int n_requests, int max_rows) {
  if (check_pages(pages, 0) || n_q_heads < 1 || n_q_heads % pages->n_kv_heads || max_blocks < 1 || n_requests < 1 || max_rows < 1 || max_rows > LA_MAX_ROWS) return 0;
  return ta_plan(*pages, n_q_heads, max_blocks, n_requests, max_rows).bytes;
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
  const TreePlan plan = ta_plan(p, n_q_heads, max_blocks, n_requests, max_rows);
  LA_REQUIRE(plan.grid < 1u << 24 && (long long)n_requests * max_rows * ceil_div(n_q_heads, TA_JOIN_WAVES) < 1ll << 24, LA_EINVAL,
             "%d requests of %d rows and %d heads are more than one launch takes", n_requests, max_rows, n_q_heads);  // (2^32 threads)
  LA_REQUIRE(workspace_bytes >= plan.bytes && (workspace || !plan.bytes), LA_ENOMEM, "workspace of %zu bytes, %zu needed", workspace_bytes, plan.bytes);
  LA_REQUIRE(aligned16({workspace}), LA_EINVAL, "workspace must be 16-byte aligned");
  hipStream_t s = (hipStream_t)stream;
  const size_t at = layer * layer_bytes(&p);
  TreeAttend a{(const char *)p.k + at, (const char *)p.v + at, p.n_pages, p.page_size, p.n_kv_heads, p.head_dim, q, q_stride, n_q_heads, scale, table, table_stride, n_requests,
               max_blocks, first, len, vis, max_rows, B, out, out_stride};
  a.kind = AT_OUT_ROWS;
  a.part = (float *)workspace;
  return ta_run(a, p.dtype, plan, s);
}
