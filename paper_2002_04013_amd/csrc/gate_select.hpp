// Exact TopK of one token over the expert grid by one wave, from its fp64 scores in LDS (Sec.
// 3.2, Eq. 1, App. C): the selection of dmoe_gate_topk's exact routes and of dmoe_layer_few_fwd.
#pragma once

#include "common.hpp"

namespace dmoe {

struct GateArgs {
  const void* x; const void* Wg; const void* bg; const uint8_t* alive;
  int32_t* idx; float* w; float* g; float* scores;
  int T, D, d, M, k, dM, N;
};

// Order-preserving 64-bit image of an fp64 value (larger value, larger key; no NaN).
__device__ __forceinline__ uint64_t ord64(double v) {
  const uint64_t b = (uint64_t)__double_as_longlong(v);
  return (b >> 63) ? ~b : (b | 0x8000000000000000ull);
}
// Cell keys (live, total, ~flat) compared lexicographically: alive first (when ranked
// that way), then the larger total, then the lower flat index (larger ~flat).
__device__ __forceinline__ bool cell_gt(uint32_t al, uint64_t at, uint32_t an, uint32_t bl, uint64_t bt,
                                        uint32_t bn) {
  return (al > bl) | ((al == bl) & ((at > bt) | ((at == bt) & (an > bn))));
}

// Element q (compile-time after unrolling) of a 16-byte vector, as a float.
template <typename E> __device__ __forceinline__ float vec_elem(const uint4& v, int q);
template <> __device__ __forceinline__ float vec_elem<float>(const uint4& v, int q) {
  return __uint_as_float(q == 0 ? v.x : q == 1 ? v.y : q == 2 ? v.z : v.w);
}
template <> __device__ __forceinline__ float vec_elem<bf16>(const uint4& v, int q) {
  const uint32_t w = (q >> 1) == 0 ? v.x : (q >> 1) == 1 ? v.y : (q >> 1) == 2 ? v.z : v.w;
  return __uint_as_float((q & 1) ? (w & 0xffff0000u) : (w << 16));
}

template <int CTRL, int ROWS>
__device__ __forceinline__ uint64_t u64_max_dpp(uint64_t v) {
  const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp((int)(uint32_t)v, (int)(uint32_t)v, CTRL, ROWS, 0xf, false);
  const uint32_t hi = (uint32_t)__builtin_amdgcn_update_dpp((int)(uint32_t)(v >> 32), (int)(uint32_t)(v >> 32), CTRL,
                                                            ROWS, 0xf, false);
  const uint64_t o = ((uint64_t)hi << 32) | lo;
  return o > v ? o : v;
}

// Maximum of a 64-bit value over the wave (every lane gets it): within each row of 16
// lanes by DPP exchanges (lane i with i^1, i^2, 7-i, 15-i), then row r-1's last lane into
// row r (rows 1 and 3) and lane 31 into rows 2 and 3, so that lane 63 holds the maximum.
__device__ __forceinline__ uint64_t wave_max_u64(uint64_t v) {
  v = u64_max_dpp<0xB1, 0xf>(v);       // quad_perm [1,0,3,2]
  v = u64_max_dpp<0x4E, 0xf>(v);       // quad_perm [2,3,0,1]
  v = u64_max_dpp<0x141, 0xf>(v);      // row_half_mirror
  v = u64_max_dpp<0x140, 0xf>(v);      // row_mirror
  v = u64_max_dpp<0x142, 0xa>(v);      // row_bcast:15
  v = u64_max_dpp<0x143, 0xc>(v);      // row_bcast:31
  return ((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(v >> 32), 63) << 32) |
         (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)v, 63);
}

// The rank tuples (r_0 .. r_{d-1}) with prod(r_i + 1) <= K1, in order of the product: the
// cells of a grid that can be among its K1 best (a cell with per-dimension ranks r_i is
// beaten by the prod(r_i + 1) - 1 cells that take an equal or better index in every
// dimension).  Those of a smaller K1 are a prefix.  4 bits per digit.
constexpr int RANK_KMAX = KMAX + 3;      // largest K1
constexpr int RANK_TUPLES = 96;          // 93 tuples for d = 4, K1 = 11
struct RankTable {
  uint16_t tup[DMAX][RANK_TUPLES];
  uint8_t cnt[DMAX][RANK_KMAX + 1];
};
constexpr RankTable make_rank_table() {
  RankTable q{};
  for (int d = 1; d <= DMAX; ++d) {
    int n = 0;
    for (int prod = 1; prod <= RANK_KMAX; ++prod) {
      for (int r0 = 0; r0 < prod; ++r0)
        for (int r1 = 0; r1 < (d > 1 ? prod : 1); ++r1)
          for (int r2 = 0; r2 < (d > 2 ? prod : 1); ++r2)
            for (int r3 = 0; r3 < (d > 3 ? prod : 1); ++r3)
              if ((r0 + 1) * (r1 + 1) * (r2 + 1) * (r3 + 1) == prod)
                q.tup[d - 1][n++] = (uint16_t)(r0 | (r1 << 4) | (r2 << 8) | (r3 << 12));
      q.cnt[d - 1][prod] = (uint8_t)n;
    }
  }
  return q;
}
static __device__ const RankTable rank_table = make_rank_table();

// Orders the LDS operations of one wave for the compiler; the hardware keeps their order.
__device__ __forceinline__ void wave_lds_sync() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }

// This lane's candidate tuples (the cells ranked for K1) and how many there are.
struct RankTuples { int cnt, tup[2]; };
template <bool ALIVE> __device__ __forceinline__ int rank_k1(const GateArgs& a) {
  return ALIVE ? min(a.N, RANK_KMAX) : a.k;
}
template <bool ALIVE> __device__ __forceinline__ RankTuples rank_tuples(const GateArgs& a) {
  const int lane = threadIdx.x & 63;
  RankTuples r;
  r.cnt = rank_table.cnt[a.d - 1][rank_k1<ALIVE>(a)];
  r.tup[0] = rank_table.tup[a.d - 1][lane];
  r.tup[1] = rank_table.tup[a.d - 1][min(lane + 64, RANK_TUPLES - 1)];
  return r;
}

// Per-wave LDS of the selection.
constexpr int RANK_LIVE = 1 << 30;       // N <= 16384
constexpr int DEC_ZERO = DM_MAX + 4 * DMAX;
struct SelectScratch {
  float dec[DEC_ZERO + 4];               // decision scores, each dimension padded to 4 with -inf; a 0
  float lv[DMAX][RANK_KMAX + 1];         // per dimension, the best indices: score and index
  int li[DMAX][RANK_KMAX + 1];
  double tot[RANK_TUPLES];               // candidate cells: total, flat index
  int flat[RANK_TUPLES];
  int rf[RANK_KMAX + 1], ru[RANK_KMAX + 1];   // by rank: flat index (bit 30: the expert responds), grid indices (8 bits each)
  int own[RANK_KMAX + 1];                     // by rank: the candidate that wrote it
};

template <int CTRL, int ROWS>
__device__ __forceinline__ uint32_t u32_max_dpp(uint32_t v) {
  const uint32_t o = (uint32_t)__builtin_amdgcn_update_dpp((int)v, (int)v, CTRL, ROWS, 0xf, false);
  return o > v ? o : v;
}
// As wave_max_u64, of 32 bits.
__device__ __forceinline__ uint32_t wave_max_u32(uint32_t v) {
  v = u32_max_dpp<0xB1, 0xf>(v);
  v = u32_max_dpp<0x4E, 0xf>(v);
  v = u32_max_dpp<0x141, 0xf>(v);
  v = u32_max_dpp<0x140, 0xf>(v);
  v = u32_max_dpp<0x142, 0xa>(v);
  v = u32_max_dpp<0x143, 0xc>(v);
  return (uint32_t)__builtin_amdgcn_readlane((int)v, 63);
}

// This lane takes the previous lane's value (lane 0 its own); the list below lies in a row of 16.
__device__ __forceinline__ uint32_t shift_up(uint32_t v) {
  return (uint32_t)__builtin_amdgcn_update_dpp((int)v, (int)v, 0x111, 0xf, 0xf, false);   // row_shr:1
}

// TopK by its definition for one token, by one wave, in one pass over every cell of the grid:
// lane l takes the cells l, l + 64, ... (mixed-radix digits advanced by 64 per cell), the
// totals adding the d decision scores in fp64 in dimension order, ranked (alive first when
// ALIVE, total desc, flat asc).  The k best so far lie in lanes 0 .. k - 1, best first; the
// few cells of a step that beat the k-th (a ballot) are inserted one by one, at their count of
// better entries; of the first 64 cells, most of which would be, the k best are taken by k rounds
// of a maximum (ranking them by counting is 64 steps, which the four waves of a SIMD share).  A
// step's alive flags are loaded RA_U steps at a time.
// Reached where a ranking of the likely cells does not decide: fewer than k alive among them,
// or totals that may round.  Bound by the latency of a step's and of an insertion's chain.  The
// gate call with a fifth of the experts alive, D = 512, fp32, as k rounds over every cell /
// with a sorted list of k cells in every lane / this form: T = 8192, 15625 experts, k = 8
// 3412 / 1072 / 381 us; 14641 experts, k = 4 1498 / 702 / 294 us; 4096 experts, k = 8
// 622 / 451 / 138 us.  T = 836, D = 1984, 256 experts, k = 6, 30% alive: 54 / 32 / 35 us (42 with
// the first cells ranked by counting).
constexpr int RA_U = 4;
template <bool ALIVE>
__device__ __forceinline__ void rank_all_wave(const GateArgs& a, const float* dec, int M4, int* rf, int* ru) {
  const int lane = threadIdx.x & 63;
  const int d = a.d, M = a.M, N = a.N, k = a.k;
  int u[DMAX], st[DMAX], at[DMAX];                                   // digits, their steps, the dimensions' scores
  {
    int rl = lane, rs = 64;
#pragma unroll
    for (int i = DMAX - 1; i >= 0; --i) {
      u[i] = 0; st[i] = 0; at[i] = DEC_ZERO;                         // dimensions past d add 0
      if (i < d) { u[i] = rl % M; rl /= M; st[i] = rs % M; rs /= M; at[i] = i * M4; }
    }
  }
  uint32_t el = 0u, en = 0u;                                         // this lane's entry: below every cell
  uint64_t et = 0ull;
  uint32_t kl = 0u, kn = 0u;                                         // the k-th entry
  uint64_t kt = 0ull;
  auto kth = [&]() {
    kl = (uint32_t)__builtin_amdgcn_readlane((int)el, k - 1);
    kn = (uint32_t)__builtin_amdgcn_readlane((int)en, k - 1);
    kt = ((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(et >> 32), k - 1) << 32) |
         (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)et, k - 1);
  };
  for (int f0 = 0; f0 < N; f0 += 64 * RA_U) {
    uint32_t live[RA_U];
    uint64_t tt[RA_U];
#pragma unroll
    for (int q = 0; q < RA_U; ++q) {
      live[q] = 1u;
      if (ALIVE && a.alive != nullptr) live[q] = a.alive[min(f0 + 64 * q + lane, N - 1)];
    }
#pragma unroll
    for (int q = 0; q < RA_U; ++q) {
      double tot = 0.0;
      int carry = 0;
#pragma unroll
      for (int i = 0; i < DMAX; ++i) tot += (double)dec[at[i] + u[i]];   // digits stay in [0, M)
      tt[q] = ord64(tot == tot ? tot + 0.0 : -INFINITY);             // -0 and +0 are one value
#pragma unroll
      for (int i = DMAX - 1; i >= 0; --i) {                          // digits of f + 64
        u[i] += st[i] + carry;
        carry = u[i] >= M;
        u[i] -= carry ? M : 0;
      }
    }
#pragma unroll
    for (int q = 0; q < RA_U; ++q) {
      const int f = f0 + 64 * q + lane;
      const uint32_t n = ~(uint32_t)f, l = live[q] != 0u ? 1u : 0u;
      auto take = [&](int s, uint32_t& cl, uint64_t& ct, uint32_t& cn) {     // the cell of lane s
        cl = (uint32_t)__builtin_amdgcn_readlane((int)l, s);
        cn = (uint32_t)__builtin_amdgcn_readlane((int)n, s);
        ct = ((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(tt[q] >> 32), s) << 32) |
             (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)tt[q], s);
      };
      if (q == 0 && f0 == 0) {                                       // the first cells: k rounds of a maximum
        bool in = f < N;
        for (int j = 0; j < min(N, k); ++j) {
          const bool alive = __ballot(in && l != 0u) != 0ull;
          const bool cand = in && (!alive || l != 0u);
          const uint64_t best = wave_max_u64(cand ? tt[q] : 0ull);   // no image is 0
          const int s = __builtin_ctzll(__ballot(cand && tt[q] == best));
          if (lane == j) { el = alive ? 1u : 0u; et = best; en = ~(uint32_t)s; }
          in = in && lane != s;
        }
        kth();
        continue;
      }
      uint64_t in = __ballot(f < N && cell_gt(l, tt[q], n, kl, kt, kn));
      while (in) {
        const int s = __builtin_ctzll(in);
        in &= in - 1;
        uint32_t cl, cn;
        uint64_t ct;
        take(s, cl, ct, cn);
        if (!cell_gt(cl, ct, cn, kl, kt, kn)) continue;              // a cell of this step took its place
        const int pos = __popcll(__ballot(lane < k && cell_gt(el, et, en, cl, ct, cn)));
        const uint32_t pl = shift_up(el), pn = shift_up(en);
        const uint64_t pt = ((uint64_t)shift_up((uint32_t)(et >> 32)) << 32) | shift_up((uint32_t)et);
        el = lane == pos ? cl : lane > pos ? pl : el;
        et = lane == pos ? ct : lane > pos ? pt : et;
        en = lane == pos ? cn : lane > pos ? pn : en;
        kth();
      }
    }
  }
  if (lane < k) {                                                    // k <= N: every entry is a cell
    const int f = (int)~en;
    int rem = f, uu = 0;
#pragma unroll
    for (int i = DMAX - 1; i >= 0; --i)
      if (i < d) { uu |= (rem % M) << (8 * i); rem /= M; }
    rf[lane] = f | (a.alive == nullptr || a.alive[f] != 0 ? RANK_LIVE : 0);
    ru[lane] = uu;
  }
  wave_lds_sync();
}

// One token's exact selection by one wave from its fp64 scores sc[d*M] in LDS: the same
// definition as select_token_cap without a certificate (the scores are exact).  Nothing is
// serial in k or M: a lane holds one or two gate columns and counts the columns of its
// dimension that beat it, which is the column's rank; a lane holds one or two candidate
// tuples and counts the candidates that beat its total.  Equal values are found by reading
// the rank slots back, and ranked again by (value desc, index asc).
// ALIVE: K1 = min(N, 11) cells are ranked and the first k alive ones taken; with
// fewer alive among them, or where fp64 totals may round (nonzero scores spanning more than
// 2^26), every cell of the grid is ranked.
template <bool ALIVE>
__device__ __forceinline__ void select_wave(const GateArgs& a, const RankTuples& rt, const double* sc,
                                            SelectScratch& q, int t) {
  const int lane = threadIdx.x & 63;
  const int d = a.d, M = a.M, k = a.k, N = a.N, dM = a.dM;
  const int M4 = (M + 3) & ~3;
  const int K1 = rank_k1<ALIVE>(a);
  const int L = min(K1, M);
  // decision scores (a NaN ranks with -inf, last), their span, and safe contents for the
  // rank slots
  int ci[2], cu[2];
  float cv[2];
  float amax = 0.f, amin = 3.4e38f;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int c = lane + 64 * h;
    ci[h] = (c >= M) + (c >= 2 * M) + (c >= 3 * M);
    cu[h] = c - ci[h] * M;
    cv[h] = 0.f;
    if (c < dM) {
      const float v = (float)sc[c], av = fabsf(v);
      cv[h] = v == v ? v : -INFINITY;
      q.dec[ci[h] * M4 + cu[h]] = cv[h];
      if (av > 0.f) { amax = fmaxf(amax, av); amin = fminf(amin, av); }
    }
  }
  if (lane == 0) q.dec[DEC_ZERO] = 0.f;
  for (int p = lane; p < d * (M4 - M); p += 64) q.dec[(p / (M4 - M)) * M4 + M + p % (M4 - M)] = -INFINITY;
  if (lane < DMAX * (RANK_KMAX + 1)) { (&q.lv[0][0])[lane] = -INFINITY; (&q.li[0][0])[lane] = 0; }
  if (lane <= RANK_KMAX) { q.rf[lane] = min(lane, N - 1); q.ru[lane] = 0; q.own[lane] = -1; }
  // magnitudes are not negative, so their bit patterns are ordered as they are
  amax = __uint_as_float(wave_max_u32(__float_as_uint(amax)));
  amin = __uint_as_float(~wave_max_u32(~__float_as_uint(amin)));
  bool full = amax > 0.f && !(amax <= amin * 67108864.f);            // span 2^26
  wave_lds_sync();
  // rank of each column in its dimension
  int rk[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    rk[h] = L;
    if (lane + 64 * h < dM) {
      const float* dv = q.dec + ci[h] * M4;
      int r = 0;
#pragma unroll 8
      for (int u = 0; u < M4; u += 4) {
        const float4 o = *reinterpret_cast<const float4*>(dv + u);
        r += (o.x > cv[h]) + (o.y > cv[h]) + (o.z > cv[h]) + (o.w > cv[h]);
      }
      rk[h] = r;
    }
  }
  auto put_lists = [&]() {
#pragma unroll
    for (int h = 0; h < 2; ++h)
      if (rk[h] < L) { q.lv[ci[h]][rk[h]] = cv[h]; q.li[ci[h]][rk[h]] = cu[h]; }
    wave_lds_sync();
  };
  put_lists();
  bool clash = false;
#pragma unroll
  for (int h = 0; h < 2; ++h) clash |= rk[h] < L && q.li[ci[h]][rk[h]] != cu[h];
  if (__ballot(clash)) {                                             // equal scores: by index
#pragma unroll
    for (int h = 0; h < 2; ++h)
      if (rk[h] < L) {
        const float* dv = q.dec + ci[h] * M4;
        for (int u = 0; u < cu[h]; ++u) rk[h] += dv[u] == cv[h];
      }
    put_lists();
  }
  // candidate cells
  const int cnt = rt.cnt;
  double tv[2];
  int tf[2], tu[2];
  bool tk[2], lv[2] = {false, false};   // lv: alive, loaded while the ranks are counted
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int p = lane + 64 * h;
    tv[h] = -INFINITY; tf[h] = 0x7fffffff; tu[h] = 0; tk[h] = p < cnt;
    if (p < cnt) {
      const int tup = rt.tup[h];
      double tot = 0.0;
      int flat = 0, uu = 0;
#pragma unroll
      for (int i = 0; i < DMAX; ++i) {
        if (i < d) {
          const int r = (tup >> (4 * i)) & 15;
          if (r >= L) { tk[h] = false; continue; }
          const int u = q.li[i][r];
          tot += (double)q.lv[i][r];
          flat = flat * M + u;
          uu |= u << (8 * i);
        }
      }
      if (tk[h]) {
        tv[h] = tot == tot ? tot : -INFINITY;                        // inf - inf
        tf[h] = flat; tu[h] = uu;
        lv[h] = a.alive == nullptr || a.alive[flat] != 0;
      }
      q.tot[p] = tv[h];
      q.flat[p] = tf[h];
    }
  }
  wave_lds_sync();
  int rc[2] = {0, 0};
#pragma unroll 8
  for (int o = 0; o < cnt; ++o) {
    const double v = q.tot[o];
    rc[0] += v > tv[0];
    rc[1] += v > tv[1];
  }
  auto put_cells = [&]() {
#pragma unroll
    for (int h = 0; h < 2; ++h)
      if (tk[h] && rc[h] < K1) {
        q.rf[rc[h]] = tf[h] | (lv[h] ? RANK_LIVE : 0);
        q.ru[rc[h]] = tu[h];
        q.own[rc[h]] = lane + 64 * h;
      }
    wave_lds_sync();
  };
  put_cells();
  clash = false;
#pragma unroll
  for (int h = 0; h < 2; ++h) clash |= tk[h] && rc[h] < K1 && q.own[rc[h]] != lane + 64 * h;
  if (__ballot(clash)) {                                             // equal totals: by flat index
    for (int o = 0; o < cnt; ++o) {
      const double v = q.tot[o];
      const int fo = q.flat[o];
      rc[0] += (v == tv[0]) & (fo < tf[0]);
      rc[1] += (v == tv[1]) & (fo < tf[1]);
    }
    put_cells();
  }
  if constexpr (ALIVE) {
    // the first k alive of the K1 ranked cells, in order
    const int cf = lane < K1 ? q.rf[lane] : 0, cuu = lane < K1 ? q.ru[lane] : 0;
    const uint64_t am = __ballot(lane < K1 && (cf & RANK_LIVE));
    full |= __popcll(am) < k;
    const int pos = __popcll(am & ((1ull << lane) - 1ull));
    if ((am >> lane) & 1ull) { q.rf[pos] = cf; q.ru[pos] = cuu; }
    wave_lds_sync();
  }
  if (full) rank_all_wave<ALIVE>(a, q.dec, M4, q.rf, q.ru);
  const int fl = lane < k ? q.rf[lane] : 0, uu = lane < k ? q.ru[lane] : 0;
  const int f = fl & (RANK_LIVE - 1);
  // Eq. 1 weights from the fp64 totals of the chosen experts, over the alive ones: lane j
  // holds the j-th, sums in slot order
  const bool live = (fl & RANK_LIVE) != 0;
  double gx = 0.0;
#pragma unroll
  for (int i = 0; i < DMAX; ++i) if (i < d) gx += sc[i * M + ((uu >> (8 * i)) & 0xff)];
  double m = live ? gx : -1.0e308;
#pragma unroll
  for (int o = 1; o < KMAX; o <<= 1) {
    const double om = __shfl_xor(m, o, 64);
    m = om > m ? om : m;
  }
  const float ex = live ? expf((float)(gx - m)) : 0.f;
  float sum = 0.f;
#pragma unroll
  for (int j = 0; j < KMAX; ++j) sum += __shfl(ex, j, 64);
  const bool any = (__ballot(live) & 0xffull) != 0ull;
  if (lane < k) {
    a.idx[(int64_t)t * k + lane] = f;
    a.w[(int64_t)t * k + lane] = any ? ex / sum : 0.f;
    if (a.g) a.g[(int64_t)t * k + lane] = (float)gx;
  }
}

}  // namespace dmoe
