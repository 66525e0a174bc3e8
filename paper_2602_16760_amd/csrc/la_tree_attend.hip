// Attention of trees of drafted tokens over the pages of their requests (la_paged_tree_attend).
#include "la_tree.h"

namespace la {

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
