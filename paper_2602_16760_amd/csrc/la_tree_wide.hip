// Attention of trees whose rows and query heads are many: a workgroup of four or eight waves has a kv head's K and V go through LDS once for all of its columns.
#include "la_tree.h"

#define LDS_AS __attribute__((address_space(3)))

namespace la {

typedef short __attribute__((ext_vector_type(4))) tw_s4;

template <int DH> constexpr int TW_KEYS = DH <= 128 ? 64 : 32;  // of a stage
template <int DH> constexpr int TW_PITCH = DH <= 64 ? 128 : DH <= 128 ? 256 : 512;  // bytes of a row in LDS
template <int DH> constexpr int TW_STAGE = 2 * TW_KEYS<DH> * TW_PITCH<DH>;

// 16 bytes a lane from base + offset to LDS at `to` + 16 lane.  In assembly, as is the wait for them: the compiler does not know which LDS reads they concern, and waits for all of them in
// front of every transposing read; what it waits for of its own loads is then waited for with them, which is safe.
// m0 is set anew by the compiler where it needs it, and is no register that it gives out (as a clobber it is refused).  The wait states are those between a vector instruction's write of a scalar and a load that takes it.
template <bool ONCE>
__device__ __forceinline__ void tw_load(unsigned to, const char *base, unsigned offset) {
  if constexpr (ONCE) asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tglobal_load_lds_dwordx4 %1, %2 nt" : : "s"(to), "v"(offset), "s"(base) : "memory");
  else asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tglobal_load_lds_dwordx4 %1, %2" : : "s"(to), "v"(offset), "s"(base) : "memory");
}
template <int N>
__device__ __forceinline__ void tw_wait_loads() {  // at most N of this wave's loads on their way
  asm volatile("s_waitcnt vmcnt(%0)" : : "n"(N) : "memory");
}
__device__ __forceinline__ void tw_wait_lds() { asm volatile("s_waitcnt lgkmcnt(0)" : : : "memory"); }
__device__ __forceinline__ void tw_barrier() {
  __atomic_signal_fence(__ATOMIC_SEQ_CST);
  __builtin_amdgcn_s_barrier();
  __atomic_signal_fence(__ATOMIC_SEQ_CST);
}

// Keys go through a ring of NS stages in LDS, K rows and V rows of a stage's keys, brought by direct-to-LDS loads of 1 KB; a wave has 16 NT columns of its own and all keys, so nothing is left
// to add up but the items.  One barrier a stage: past it every wave's part of the stage is in, and nobody reads the stage any more that the next requests overwrite.
// The 16-byte pieces of a row are permuted by its key, so that sixteen keys' equal pieces, and four keys' neighbouring ones, lie in different banks.  V's operand, eight keys of a channel in a
// lane, comes out of LDS by transposing reads.
// Bound by the matrix unit and the power it draws at long requests: two of 64 rows at 65000 keys, 32 query heads of 128 channels, are 137 GFLOP, 205 with V's products with the weights' second
// numbers: half precision 220 us, 0.93 PFLOP/s of the 205 where a large library product reaches 1.16 (0.62 of the 137), 267 in the mean where the call repeats at once and the clock falls; bfloat16
// 198, its offsets being moved less often.  Without the weights' instructions it would be 190.  These go first (s_setprio), so that one workgroup's fill the gaps of
// the other's products: 8 x 64 rows at 16000 227 -> 210, 16 x 64 at 4000 133 -> 124.  The next stage's scores in front of a stage's weights took 353; products of 32 by 32, V asked for in front of the
// weights, priority for the products: no difference.  At 16 requests of 1 to 16 rows at 64 to 4096, 41 MB, 19 us: the chain to a workgroup's first stage, five stages, and 34 KB of sums out of it.
template <typename T, int DH, int WAVES, int NT, int NS>
__global__ __launch_bounds__(64 * WAVES, 2) void tree_wide_kernel(TreeAttend a) {
  constexpr int KEYS = TW_KEYS<DH>, TILES = KEYS / 16, KP = DH / 32, DT = DH / 16, ROWB = DH * 2, PITCH = TW_PITCH<DH>, HALF = KEYS * PITCH, STAGE = 2 * HALF;
  constexpr int PPR = PITCH / 16, KPI = 1024 / PITCH;        // pieces of a row; rows of a request
  constexpr int LPW = STAGE / 1024 / WAVES, HALF_N = HALF / 1024;  // a wave's requests of a stage; requests of its K
  constexpr int EIGHTS = KEYS / 8, WINDOW = 64 / EIGHTS;     // page boundaries lie between eights of keys; stages whose eights a wave's lanes look up at once
  constexpr float UP = TA_UP<T>, LAZY = TA_LAZY<T>;
  static_assert(LPW * WAVES * 1024 == STAGE && (NS - 1) * LPW <= 63, "requests");
  extern __shared__ __attribute__((aligned(1024))) uint8_t tw_lds[];
  const unsigned lds0 = (unsigned)(uintptr_t)(LDS_AS uint8_t *)tw_lds;
  const int wave = uniform((int)(threadIdx.x >> 6)), lane = threadIdx.x & 63, q4 = lane >> 4, c16 = lane & 15;
  const int g = uniform(a.Hq / a.Hkv);
  int item, h, tile;
  ta_share(a, (int)blockIdx.x, item, h, tile);
  ta_zero_outside<T>(a, 64 * WAVES);
  if (item < 0) return;
  const AtItem it = at_find<false, true>(a, item);
  if (it.b < 0) return;  // (all waves)
  ta_note(a, it, h, tile);
  int f0;
  const int n_rows = uniform(tree_rows(a, it.b, f0)), first = uniform(f0), L = uniform(a.len[it.b]);
  if (it.index == 0 && tile == 0) ta_zero_behind<T>(a, it.b, first, n_rows, h * g * DH, g * DH, 64 * WAVES);
  const int all_cols = n_rows * g - tile * 16 * NT * WAVES;  // of this workgroup, if it had room for all
  if (all_cols <= 0) return;
  const int col0 = tile * 16 * NT * WAVES + wave * 16 * NT, cols = n_rows * g - col0;  // of this wave
  const int k_first = it.index * it.C, k_end = at_item_end(it), n_stages = (int)(((unsigned)(k_end - k_first) + KEYS - 1u) / KEYS);
  at_u4 q[NT][KP];
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    const int c = 16 * t + c16 < cols ? col0 + 16 * t + c16 : 0, j = c / g, i = first + j, head = h * g + c - j * g;
    const char *qp = (const char *)a.q + (a.q_tiles ? (((int64_t)head * a.q_tiles + (i >> 4)) * (DH / 32) * 64 + (i & 15)) * 16 : (i * a.ldq + (int64_t)head * DH) * 2);
#pragma unroll
    for (int p = 0; p < KP; ++p) q[t][p] = *(const at_u4 *)(qp + (a.q_tiles ? 1024 * p + 256 * q4 : 64 * p + 16 * q4));
    if (a.scale < 0.f)  // (scores are multiplied by what is not negative: the largest stays the largest)
#pragma unroll
      for (int p = 0; p < KP; ++p) q[t][p] ^= 0x80008000u;
  }
  unsigned long long early = 0;  // the column's mask: asked for here, since where it is needed first, at the request's end, everybody would wait for it (of two there are no registers for them)
  if constexpr (NT == 1) early = a.vis[first + (c16 < cols ? col0 + c16 : 0) / g];
  const float to_log2 = fabsf(a.scale) * AT_LOG2E;
  const int32_t *tab = a.table + it.r * a.ldt;
  // Lane i: where eight keys, the i-th of the next WINDOW stages', lie (the first page where they lie in none: they are not seen, whatever they hold).
  unsigned off_lo = 0, off_hi = 0;
  unsigned long long paged = 0, paged_next = 0;  // bit i: they lie in a page
  int next_page, next_place;
  auto ask = [&](int stage) {  // for the window from this stage on: the entry is here when the stage before that has been waited for
    const long long key = k_first + (long long)KEYS * stage + 8 * lane;
    const int k = key < k_end ? (int)key : k_end - 1, block = k / a.page;
    next_page = tab[block];
    next_place = key < k_end ? k - block * a.page : -1;
  };
  auto look_up = [&]() {
    long long at = next_place >= 0 && (unsigned)next_page < (unsigned)a.n_pages ? (((long long)next_page * a.Hkv + h) * a.page + next_place) * ROWB : -1;
    paged_next = __ballot(at >= 0);
    at = at < 0 ? 0 : at;
    off_lo = (unsigned)at;
    off_hi = (unsigned)(at >> 32);
  };
  auto swz_k = [](int key) { return DH == 64 ? (key >> 1) & 7 : key & 15; };
  auto swz_v = [](int key) { return DH == 64 ? 2 * ((key >> 1) & 3) : 2 * (key & 7); };
  // what this wave brings of a stage: requests wave LPW .., the first HALF_N of a stage are K's (places behind a row's end hold its pieces again; nothing reads them as channels)
  unsigned voff[LPW];
#pragma unroll
  for (int i = 0; i < LPW; ++i) {
    const int n = wave * LPW + i, key = n % HALF_N * KPI % 16 + lane / PPR, piece = lane % PPR ^ (n < HALF_N ? swz_k(key) : swz_v(key));
    voff[i] = (unsigned)(key % 8 * ROWB + piece % (ROWB / 16) * 16);
  }
  int nx = 0;
  unsigned nx_slot = 0;
  auto request = [&]() {
    if (nx < n_stages) {
      if (nx > 0 && nx % WINDOW == 0) {
        look_up();
        ask(nx + WINDOW);
      }
      auto all = [&](auto once) {
#pragma unroll
        for (int i = 0; i < LPW; ++i) {
          const int n = wave * LPW + i, l = nx % WINDOW * EIGHTS + n % HALF_N * KPI / 8;
          const long long at = (long long)(unsigned)__builtin_amdgcn_readlane((int)off_lo, l) | (long long)__builtin_amdgcn_readlane((int)off_hi, l) << 32;
          tw_load<decltype(once)::value>(lds0 + nx_slot + (unsigned)n * 1024u, (const char *)(n < HALF_N ? a.K : a.V) + at, voff[i]);
        }
      };
      a.once ? all(std::true_type{}) : all(std::false_type{});
    }
    ++nx;
    nx_slot = nx_slot + STAGE == NS * STAGE ? 0u : nx_slot + STAGE;
  };
  at_f4 o[NT][DT];
  float m_run[NT], l_run[NT];
  bool far[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t) {
#pragma unroll
    for (int d = 0; d < DT; ++d) o[t][d] = at_f4{0.f, 0.f, 0.f, 0.f};
    m_run[t] = -INFINITY;
    l_run[t] = 0.f;
    far[t] = false;
  }
  ask(0);
  look_up();
  ask(WINDOW);
  __builtin_amdgcn_s_waitcnt(0xf70);  // (vmcnt(0): q is in, and the compiler knows it)
#pragma unroll
  for (int i = 0; i < NS - 1; ++i) request();
  const unsigned rd_k = (unsigned)(c16 * PITCH) + (unsigned)((q4 ^ swz_k(c16)) * 16);  // piece 4 p + q4 of key c16 of a tile: ^ 64 p
  const int v_key = 4 * q4 + (c16 >> 2);
  const unsigned rd_v = (unsigned)(HALF + v_key * PITCH + (((c16 >> 1) & 1) ^ swz_v(v_key)) * 16 + 8 * (c16 & 1));  // channels 16 d ..: ^ 32 d
  LDS_AS unsigned *odd_lds = (LDS_AS unsigned *)(uintptr_t)(lds0 + NS * STAGE);
  unsigned long long odd_rows = 0;  // drafted rows, of those whose keys this item has, whose V has an infinity or NaN
  unsigned slot = 0;
  for (int i = 0; i < n_stages; ++i) {
    if (i + NS - 1 <= n_stages) tw_wait_loads<(NS - 2) * LPW>();
    else tw_wait_loads<0>();
    tw_wait_lds();
    tw_barrier();
    if (i % WINDOW == 0) paged = paged_next;  // (the window after it is not looked up before the next request but NS - 2)
    request();
    const int key0 = k_first + KEYS * i;
    // keys of the stage that lie in a page, in front of the item's end
    constexpr unsigned long long ALL = KEYS == 64 ? ~0ull : (1ull << (KEYS & 63)) - 1;
    const unsigned in = (unsigned)(paged >> (i % WINDOW * EIGHTS)) & ((1u << EIGHTS) - 1u);
    unsigned long long now = ALL;
    if (in != (1u << EIGHTS) - 1u)
#pragma unroll
      for (int t = 0; t < EIGHTS; ++t) now &= in >> t & 1 ? ~0ull : ~(0xffull << (8 * t));
    if (k_end - key0 < KEYS) now &= (1ull << (k_end - key0)) - 1;
    const bool drafted = (long long)key0 + KEYS > L;  // keys of the request's own rows among them
    const unsigned base = lds0 + slot;
    slot = slot + STAGE == NS * STAGE ? 0u : slot + STAGE;
    if (now != ALL || drafted) {  // what V has in places that not all columns see becomes zeros, where it is not seen at all or no number
      if (threadIdx.x == 0) odd_lds[0] = odd_lds[1] = 0;
      __syncthreads();
      const int committed = L - key0;
      for (int x = threadIdx.x; x < KEYS * PPR; x += 64 * WAVES) {
        const int key = x / PPR;
        LDS_AS at_u4 *p = (LDS_AS at_u4 *)(uintptr_t)(base + HALF + (unsigned)x * 16u);
        const at_u4 v = *p;
        if (!(now >> key & 1)) *p = at_u4{0, 0, 0, 0};
        else if (key >= committed && (ta_odd<T>(v[0]) || ta_odd<T>(v[1]) || ta_odd<T>(v[2]) || ta_odd<T>(v[3]))) __hip_atomic_fetch_or(odd_lds + (key >> 5), 1u << (key & 31), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
      }
      __syncthreads();
      const unsigned long long odd = uniform((unsigned long long)odd_lds[0] | (unsigned long long)odd_lds[1] << 32);
      if (odd) {
        odd_rows |= committed > 0 ? odd >> committed : odd << -committed;
        for (int x = threadIdx.x; x < KEYS * PPR; x += 64 * WAVES)
          if (odd >> (x / PPR) & 1) *(LDS_AS at_u4 *)(uintptr_t)(base + HALF + (unsigned)x * 16u) = at_u4{0, 0, 0, 0};
      }
      __syncthreads();
    }
    if (cols <= 0) continue;
    at_f4 s[NT][TILES];
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int t = 0; t < TILES; ++t) s[n][t] = at_f4{0.f, 0.f, 0.f, 0.f};
    {
      at_u4 kf[2][TILES];
      auto read_k = [&](int k) {
        unsigned from = base + (rd_k ^ (unsigned)(64 * k));
        asm("" : "+v"(from));  // (one address for all tiles: what differs fits into the instructions)
#pragma unroll
        for (int t = 0; t < TILES; ++t) kf[k & 1][t] = *(LDS_AS const at_u4 *)(uintptr_t)(from + (unsigned)(16 * t * PITCH));
      };
      read_k(0);
#pragma unroll
      for (int k = 0; k < KP; ++k) {
        if (k + 1 < KP) read_k(k + 1);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int t = 0; t < TILES; ++t)
#pragma unroll
          for (int n = 0; n < NT; ++n) s[n][t] = at_mma<T>(kf[k & 1][t], q[n][k], s[n][t]);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    float factor = to_log2;
    if (now != ALL || drafted) {
      factor = 1.f;
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        unsigned long long mask = now;  // keys that the column sees
        if (drafted) {
          const int c = 16 * n + c16 < cols ? col0 + 16 * n + c16 : 0;
          const unsigned long long vis = NT == 1 ? early : a.vis[first + c / g];
          const int at = key0 - L;  // of the stage's first key in the request's rows
          mask &= at >= 0 ? (at < 64 ? vis >> at : 0ull) : vis << -at | ((1ull << -at) - 1);  // (at > -KEYS)
        }
        mask >>= 4 * q4;
#pragma unroll
        for (int t = 0; t < TILES; ++t)
#pragma unroll
          for (int e = 0; e < 4; ++e) s[n][t][e] = mask >> (16 * t + e) & 1 ? s[n][t][e] * to_log2 : -INFINITY;
      }
    }
    __builtin_amdgcn_s_setprio(1);  // (the other workgroup's products run beside these instructions, and go last where both have one to issue)
    at_u4 p[NT][TILES / 2], rest[NT][TILES / 2];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      float mx = -INFINITY;
#pragma unroll
      for (int t = 0; t < TILES; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) mx = fmaxf(mx, s[n][t][e]);
      mx *= factor;
      if (__any(mx > m_run[n] + LAZY)) {
        const float m_new = fmaxf(m_run[n], at_max4(mx)), corr = __builtin_amdgcn_exp2f(m_run[n] - (m_new > -INFINITY ? m_new : 0.f));
        m_run[n] = m_new;
        far[n] = ta_far(m_new);
        l_run[n] *= corr;
#pragma unroll
        for (int d = 0; d < DT; ++d) o[n][d] *= corr;
      }
      const float offset = m_run[n] > -INFINITY ? m_run[n] : 0.f;
      float by = factor, add = UP - offset;
      if (far[n]) {
#pragma unroll
        for (int t = 0; t < TILES; ++t)
#pragma unroll
          for (int e = 0; e < 4; ++e) s[n][t][e] = ta_exponent<T>(s[n][t][e], factor, offset);
        by = 1.f;
        add = 0.f;
      }
#pragma unroll
      for (int t = 0; t < TILES; ++t) {
        float w[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          w[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[n][t][e], by, add));
          l_run[n] += w[e];
        }
        const at_u2 x = ta_split<T>(w[0], w[1]), y = ta_split<T>(w[2], w[3]);
        p[n][t / 2][2 * (t & 1)] = x[0];
        p[n][t / 2][2 * (t & 1) + 1] = y[0];
        rest[n][t / 2][2 * (t & 1)] = x[1];
        rest[n][t / 2][2 * (t & 1) + 1] = y[1];
      }
    }
    __builtin_amdgcn_s_setprio(0);
    {
      constexpr int DG = DT % 4 ? 3 : 4, GROUPS = TILES / 2 * DT / DG;  // V's fragments of some tiles of channels at a time, the next ones on their way
      at_u4 vf[2][DG];
      auto read_v = [&](int x) {
        const int m = x * DG / DT, d0 = x * DG % DT;
#pragma unroll
        for (int y = 0; y < DG; ++y) {
          unsigned at = base + (rd_v ^ (unsigned)(32 * (d0 + y)));
          asm("" : "+v"(at));
          const at_u2 lo = __builtin_bit_cast(at_u2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((LDS_AS tw_s4 *)(uintptr_t)(at + (unsigned)(32 * m * PITCH))));
          const at_u2 hi = __builtin_bit_cast(at_u2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((LDS_AS tw_s4 *)(uintptr_t)(at + (unsigned)(32 * m * PITCH) + 16u * PITCH)));
          vf[x & 1][y] = at_u4{lo[0], lo[1], hi[0], hi[1]};
        }
      };
      read_v(0);
#pragma unroll
      for (int x = 0; x < GROUPS; ++x) {
        const int m = x * DG / DT, d0 = x * DG % DT;
        if (x + 1 < GROUPS) read_v(x + 1);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int y = 0; y < DG; ++y)
#pragma unroll
          for (int n = 0; n < NT; ++n) o[n][d0 + y] = at_mma<T>(vf[x & 1][y], p[n][m], o[n][d0 + y]);
#pragma unroll
        for (int y = 0; y < DG; ++y)
#pragma unroll
          for (int n = 0; n < NT; ++n) o[n][d0 + y] = at_mma<T>(vf[x & 1][y], rest[n][m], o[n][d0 + y]);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
  }
  if (cols <= 0) return;
  // Those V's, which the products took as zeros (a weight of zero would have made NaN of them in every column), for the columns that see them alone.
  for (; odd_rows; odd_rows &= odd_rows - 1) {
    const int row = __builtin_ctzll(odd_rows), key = L + row, block = key / a.page;
    const long long at = (((long long)tab[block] * a.Hkv + h) * a.page + (key - block * a.page)) * ROWB;
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      const int c = 16 * n + c16 < cols ? col0 + 16 * n + c16 : 0;
      at_f4 score = {0.f, 0.f, 0.f, 0.f};  // (added up as the tile's were: the weight has to be the one in the sum)
#pragma unroll
      for (int k = 0; k < KP; ++k) score = at_mma<T>(*(const at_u4 *)((const char *)a.K + at + 64 * k + 16 * q4), q[n][k], score);
      const float w = __builtin_amdgcn_exp2f(ta_from(score[0], to_log2, m_run[n] > -INFINITY ? m_run[n] : 0.f) + UP) * (1.f + TA_REST<T>);
      if (!((NT == 1 ? early : a.vis[first + c / g]) >> row & 1u)) continue;
#pragma unroll
      for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[n][d][e] += w * load_as_float<T>((const T *)((const char *)a.V + at) + 16 * d + 4 * q4 + e);
    }
  }
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    const float l = at_sum4(l_run[n]) * (1.f + TA_REST<T>);
    if (16 * n + c16 >= cols) continue;
    const int c = col0 + 16 * n + c16, j = c / g, head = h * g + c - j * g;
    if (it.count > 1) {
      float *to = a.part + (((size_t)it.record * a.Hq + head) * a.max_rows + j) * a.rec;
      if (q4 == 0) *(float2 *)to = float2{m_run[n], l};
#pragma unroll
      for (int d = 0; d < DT; ++d) *(at_f4 *)(to + 4 + 16 * d + 4 * q4) = o[n][d];
      continue;
    }
    const bool sees = (NT == 1 ? early : a.vis[first + j]) != 0;
    const float inv = l > 0.f || l != l ? 1.f / l : 0.f;
#pragma unroll
    for (int d = 0; d < DT; ++d) {
      const at_f4 y = sees ? o[n][d] * inv : at_f4{0.f, 0.f, 0.f, 0.f};
      const int ch = 16 * d + 4 * q4;
      if (a.kind != AT_OUT_ROWS) {
#pragma unroll
        for (int e = 0; e < 4; ++e) at_store_row(a, first + j, head * DH + ch + e, y[e]);
      } else {
        *(at_u2 *)((uint16_t *)a.out + (first + j) * a.ldo + (int64_t)head * DH + ch) = at_u2{at_pack<T>(y[0], y[1]), at_pack<T>(y[2], y[3])};
      }
    }
  }
}

// ---- host side ------------------------------------------------------------------------------------------
template <typename T, int DH, int WAVES, int NT, int NS>
static int tw_launch(const TreeAttend &a, unsigned grid, hipStream_t s) {
  constexpr int LDS = NS * TW_STAGE<DH> + 16;
  if constexpr (LDS > 64 * 1024)
    if (const int rc = ta_allow_lds<tree_wide_kernel<T, DH, WAVES, NT, NS>>(LDS)) return rc;
  tree_wide_kernel<T, DH, WAVES, NT, NS><<<grid, 64 * WAVES, LDS, s>>>(a);
  return LA_OK;
}
template <typename T, int DH>
static int tw_launch(const TreeAttend &a, int columns, unsigned grid, hipStream_t s) {
  constexpr int NS = 2;  // (64 KB at 128 channels, two workgroups a CU; four stages, one workgroup: 16 ragged requests 27.5 us, so 25.3; four of 64 channels, 4 x 64 rows at 32000 135, so 130)
  if (columns == 64) return tw_launch<T, DH, 4, 1, NS>(a, grid, s);
  if constexpr (DH <= 128) return tw_launch<T, DH, 4, 2, NS>(a, grid, s);
  else return tw_launch<T, DH, 8, 1, 4>(a, grid, s);
}
template <typename T>
static int tw_launch(const TreeAttend &a, int columns, unsigned grid, hipStream_t s) {
  if (a.dh == 64) return tw_launch<T, 64>(a, columns, grid, s);
  if (a.dh == 96) return tw_launch<T, 96>(a, columns, grid, s);
  if (a.dh == 128) return tw_launch<T, 128>(a, columns, grid, s);
  return tw_launch<T, 256>(a, columns, grid, s);
}

// (128 by four waves of 32, two workgroups a CU, and 256 by eight, one: 16 x 64 rows at 500 keys 28 us and 35, 1 x 64 19.6 and 22.6, 2 x 64 at 65000 244 and 237)
int tree_attend_wide(const TreeAttend &a, int dtype, int columns, unsigned grid, hipStream_t s) {
  return dtype == LA_F16 ? tw_launch<_Float16>(a, columns, grid, s) : tw_launch<uint16_t>(a, columns, grid, s);
}

}  // namespace la
