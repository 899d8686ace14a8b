// Layer normalisation of the sub-layer around a DMoE layer (pre-norm, residual), forward and
// backward, over T rows of D features:
//   s = x + r,  mean = mean_f(s),  rstd = 1 / sqrt(mean_f((s - mean)^2) + eps),
//   n = (s - mean) rstd,  y = gamma n + beta;
//   dn = dy gamma,  dx = rstd (dn - mean_f(dn) - n mean_f(dn n)) + dr,
//   dgamma = sum_t dy n,  dbeta = sum_t dy.
// Both directions are one pass over the rows, bound by memory: GS consecutive lanes hold a
// row in registers, CH 16-byte chunks to a lane, the next row's chunks loaded ahead; the row
// sums meet by lane exchanges (GS <= 64) or through LDS.  Sums are fp32; the variance is
// summed about the mean, from the registers.  The backward keeps its columns' dgamma and
// dbeta sums in registers over all rows of a group, adds the block's groups in LDS, and a
// second kernel adds the blocks' sums in block order.
#include <algorithm>

#include "common.hpp"

namespace dmoe {

constexpr float LAYER_NORM_EPS = 1e-5f;
constexpr int64_t LNORM_DMAX = 16384;    // widest row: 1024 lanes of four fp32 chunks

constexpr int lnorm_threads(int GS) { return GS > 256 ? GS : 256; }

// Lanes and chunks of a row of `nch` chunks (at most 2048 in bf16, 4096 in fp32): a lane to a
// chunk up to a wave, two up to two waves' worth.  Wider rows: the forward has up to four chunks to a lane
// of one wave (no barrier), then of four to sixteen waves; the backward, whose column sums take
// 2 VEC registers to a chunk, at most two up to 1024 chunks (8192 rows x 4096 fp32 118 -> 106 us, 8000 x 8192
// bf16 158 -> 118 with four a lane / two; 4000 x 16384 bf16 179 with four, 252 with two).
struct RowShape { int gs, ch; };
static RowShape row_shape(int64_t nch, bool bwd) {
  for (int gs = 8; gs <= 64; gs *= 2)
    if (nch <= gs) return {gs, 1};
  if (nch <= 64 * 2) return {64, 2};
  if (nch <= 64 * 4) return bwd ? RowShape{256, 1} : RowShape{64, 4};
  if (nch <= 256 * 2) return {256, 2};
  if (nch <= 256 * 4) return bwd ? RowShape{512, 2} : RowShape{256, 4};
  if (nch <= 512 * 4) return {512, 4};
  return {1024, 4};
}

// Sum over the GS lanes of a row.  `red`: two slots of 16 floats per sum, taken in turn: a
// wave passes the barrier of one slot only after it has read the other.
template <int GS, int NV>
__device__ __forceinline__ void row_sum(float (&v)[NV], float (*red)[NV], int slot) {
#pragma unroll
  for (int o = (GS < 64 ? GS : 64) / 2; o > 0; o >>= 1)
#pragma unroll
    for (int i = 0; i < NV; ++i) v[i] += __shfl_xor(v[i], o, WAVE);
  if constexpr (GS > 64) {
    constexpr int NW = GS / 64;
    float (*s)[NV] = red + slot * 16;
    if ((threadIdx.x & 63) == 0)
#pragma unroll
      for (int i = 0; i < NV; ++i) s[threadIdx.x >> 6][i] = v[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      v[i] = s[0][i];
#pragma unroll
      for (int w = 1; w < NW; ++w) v[i] += s[w][i];
    }
  }
}

template <typename E, int GS, int CH>
struct RowPart {
  static constexpr int VEC = Vec<E>::N;
  uint4 v[CH];
  __device__ __forceinline__ void load(const E* row, int l, int nch) {
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      const int c = l + GS * i;
      v[i] = c < nch ? *reinterpret_cast<const uint4*>(row + c * VEC) : make_uint4(0, 0, 0, 0);
    }
  }
};

template <typename E, int GS, int CH, bool RES>
__global__ void __launch_bounds__(lnorm_threads(GS))
layer_norm_fwd_kernel(const E* x, const E* res, const E* gamma, const E* beta, E* s, E* y, float* stats, int T, int D) {
  constexpr int VEC = Vec<E>::N, G = lnorm_threads(GS) / GS;
  __shared__ float red[32][1];
  const int l = threadIdx.x % GS, grp = threadIdx.x / GS;
  const int nch = D / VEC;
  const float invD = 1.f / (float)D;
  RowPart<E, GS, CH> gv, bv, xv, rv, xn, rn;
  gv.load(gamma, l, nch);
  if (beta) bv.load(beta, l, nch);
  else
#pragma unroll
    for (int i = 0; i < CH; ++i) bv.v[i] = make_uint4(0, 0, 0, 0);
  const int64_t step = (int64_t)gridDim.x * G;
  // r0 is the block's first row: the loop is uniform in the block, a group past the last row
  // works on that row and stores nothing
  int64_t r0 = (int64_t)blockIdx.x * G;
  auto at = [&](int64_t q) { return min(q + grp, (int64_t)T - 1) * D; };
  xv.load(x + at(r0), l, nch);
  if constexpr (RES) rv.load(res + at(r0), l, nch);
  for (; r0 < T; r0 += step) {
    const int64_t row = r0 + grp;
    const bool live = row < T;
    if (r0 + step < T) {
      xn.load(x + at(r0 + step), l, nch);
      if constexpr (RES) rn.load(res + at(r0 + step), l, nch);
    }
    float sum[1] = {0.f};
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      float f[VEC];
      Vec<E>::unpack(xv.v[i], f);
      if constexpr (RES) {
        // the sum is rounded to the layer's type once, as it is stored, and normalised as stored
        float q[VEC];
        Vec<E>::unpack(rv.v[i], q);
#pragma unroll
        for (int j = 0; j < VEC; ++j) f[j] += q[j];
        xv.v[i] = Vec<E>::pack(f);
        Vec<E>::unpack(xv.v[i], f);
        if (live && l + GS * i < nch) *reinterpret_cast<uint4*>(s + row * D + (l + GS * i) * VEC) = xv.v[i];
      }
#pragma unroll
      for (int j = 0; j < VEC; ++j) sum[0] += f[j];
    }
    row_sum<GS, 1>(sum, red, 0);
    const float mean = sum[0] * invD;
    float sq[1] = {0.f};
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      float f[VEC];
      Vec<E>::unpack(xv.v[i], f);
      if (l + GS * i < nch)
#pragma unroll
        for (int j = 0; j < VEC; ++j) sq[0] += (f[j] - mean) * (f[j] - mean);
    }
    row_sum<GS, 1>(sq, red, 1);
    const float rstd = 1.f / sqrtf(sq[0] * invD + LAYER_NORM_EPS);
    if (live) {
#pragma unroll
      for (int i = 0; i < CH; ++i) {
        const int c = l + GS * i;
        if (c >= nch) continue;
        float f[VEC], g[VEC], b[VEC];
        Vec<E>::unpack(xv.v[i], f);
        Vec<E>::unpack(gv.v[i], g);
        Vec<E>::unpack(bv.v[i], b);
#pragma unroll
        for (int j = 0; j < VEC; ++j) f[j] = fmaf(g[j], (f[j] - mean) * rstd, b[j]);
        *reinterpret_cast<uint4*>(y + row * D + c * VEC) = Vec<E>::pack(f);
      }
      if (stats && l == 0) *reinterpret_cast<float2*>(stats + 2 * row) = make_float2(mean, rstd);
    }
    xv = xn;
    if constexpr (RES) rv = rn;
  }
}

// part: [gridDim.x][2][D], the block's sums of dy n and of dy
template <typename E, int GS, int CH, bool RES>
__global__ void __launch_bounds__(lnorm_threads(GS))
layer_norm_bwd_kernel(const E* s, const float* stats, const E* gamma, const E* dy, const E* dres, E* dx, float* part,
                      int T, int D) {
  constexpr int VEC = Vec<E>::N, NT = lnorm_threads(GS), G = NT / GS;
  __shared__ float red[32][2];
  const int l = threadIdx.x % GS, grp = threadIdx.x / GS;
  const int nch = D / VEC;
  const float invD = 1.f / (float)D;
  RowPart<E, GS, CH> gv, sv, dv, rv, sn, dn, rn;
  float2 st, stn;
  gv.load(gamma, l, nch);
  float ag[CH][VEC], ab[CH][VEC];
#pragma unroll
  for (int i = 0; i < CH; ++i)
#pragma unroll
    for (int j = 0; j < VEC; ++j) ag[i][j] = ab[i][j] = 0.f;
  const int64_t step = (int64_t)gridDim.x * G;
  int64_t r0 = (int64_t)blockIdx.x * G;
  auto load = [&](RowPart<E, GS, CH>& a, RowPart<E, GS, CH>& b, RowPart<E, GS, CH>& c, float2& t, int64_t q) {
    const int64_t row = min(q + grp, (int64_t)T - 1);
    a.load(s + row * D, l, nch);
    b.load(dy + row * D, l, nch);
    if constexpr (RES) c.load(dres + row * D, l, nch);
    t = *reinterpret_cast<const float2*>(stats + 2 * row);
  };
  load(sv, dv, rv, st, r0);
  int slot = 0;
  for (; r0 < T; r0 += step) {
    const int64_t row = r0 + grp;
    const bool live = row < T;
    if (r0 + step < T) load(sn, dn, rn, stn, r0 + step);
    float m[2] = {0.f, 0.f};
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      float f[VEC], d[VEC], g[VEC];
      Vec<E>::unpack(sv.v[i], f);
      Vec<E>::unpack(dv.v[i], d);
      Vec<E>::unpack(gv.v[i], g);
      if (live && l + GS * i < nch) {
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
          const float n = (f[j] - st.x) * st.y, q = d[j] * g[j];
          m[0] += q;
          m[1] += q * n;
          ag[i][j] += d[j] * n;
          ab[i][j] += d[j];
        }
      }
    }
    row_sum<GS, 2>(m, red, slot);
    slot ^= 1;
    const float m1 = m[0] * invD, m2 = m[1] * invD;
    if (live) {
#pragma unroll
      for (int i = 0; i < CH; ++i) {
        const int c = l + GS * i;
        if (c >= nch) continue;
        float f[VEC], d[VEC], g[VEC];
        Vec<E>::unpack(sv.v[i], f);
        Vec<E>::unpack(dv.v[i], d);
        Vec<E>::unpack(gv.v[i], g);
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
          const float n = (f[j] - st.x) * st.y;
          f[j] = st.y * (d[j] * g[j] - m1 - n * m2);
        }
        if constexpr (RES) {
          Vec<E>::unpack(rv.v[i], d);
#pragma unroll
          for (int j = 0; j < VEC; ++j) f[j] += d[j];
        }
        *reinterpret_cast<uint4*>(dx + row * D + c * VEC) = Vec<E>::pack(f);
      }
    }
    sv = sn; dv = dn; st = stn;
    if constexpr (RES) rv = rn;
  }
  // the block's groups, added in group order
  if constexpr (G > 1) {
    constexpr int W = GS * CH * VEC;                 // a group's columns
    __shared__ float sums[G][W + 4];
    for (int k = 0; k < 2; ++k) {
      __syncthreads();
#pragma unroll
      for (int i = 0; i < CH; ++i)
#pragma unroll
        for (int j = 0; j < VEC; ++j) sums[grp][(l + GS * i) * VEC + j] = k ? ab[i][j] : ag[i][j];
      __syncthreads();
      for (int c = threadIdx.x; c < D; c += NT) {
        float t = sums[0][c];
#pragma unroll
        for (int g = 1; g < G; ++g) t += sums[g][c];
        part[((int64_t)blockIdx.x * 2 + k) * D + c] = t;
      }
    }
  } else {
    float* p = part + (int64_t)blockIdx.x * 2 * D;
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      const int c = (l + GS * i) * VEC;
      if (c >= D) continue;
#pragma unroll
      for (int j = 0; j < VEC; j += 4) {
        *reinterpret_cast<float4*>(p + c + j) = make_float4(ag[i][j], ag[i][j + 1], ag[i][j + 2], ag[i][j + 3]);
        *reinterpret_cast<float4*>(p + D + c + j) = make_float4(ab[i][j], ab[i][j + 1], ab[i][j + 2], ab[i][j + 3]);
      }
    }
  }
}

// dgamma, dbeta = the nb blocks' sums in block order.  A block takes 32 of the 2 D columns, 16 bytes
// to a thread (128-byte pieces of the sums); slice threadIdx / LR_C adds a contiguous run of the
// blocks, the slices meet in LDS.
constexpr int LR_NT = 512, LR_C = 8, LR_S = LR_NT / LR_C;
template <typename E>
__global__ void __launch_bounds__(LR_NT)
layer_norm_reduce_kernel(const float* part, int nb, int D, E* dgamma, E* dbeta) {
  __shared__ float4 sums[LR_S][LR_C + 1];
  const int cc = threadIdx.x % LR_C, sl = threadIdx.x / LR_C;
  const int64_t c = ((int64_t)blockIdx.x * LR_C + cc) * 4;      // 2 D is a multiple of 128
  const int per = (nb + LR_S - 1) / LR_S;
  const int b1 = min(nb, (sl + 1) * per);
  float4 t = make_float4(0.f, 0.f, 0.f, 0.f);
  auto add = [&](const float4& v) { t.x += v.x; t.y += v.y; t.z += v.z; t.w += v.w; };
#pragma unroll 8
  for (int b = sl * per; b < b1; ++b) add(*reinterpret_cast<const float4*>(part + (int64_t)b * 2 * D + c));
  sums[sl][cc] = t;
  __syncthreads();
  if (threadIdx.x >= 4 * LR_C) return;
  // a thread to a column
  const int q = threadIdx.x;
  float s = 0.f;
#pragma unroll 8
  for (int i = 0; i < LR_S; ++i) s += reinterpret_cast<const float*>(&sums[i][0])[q];
  const int64_t o = (int64_t)blockIdx.x * LR_C * 4 + q;
  if (o < D) dgamma[o] = cvt<E>(s);
  else if (dbeta) dbeta[o - D] = cvt<E>(s);
}

// Blocks of the backward: as many as stay resident (three of 256 threads to a compute unit), each at
// least one row per group; more would only add sums for the second kernel.
static int64_t lnorm_bwd_blocks(const Shape& s) {
  const RowShape q = row_shape(s.D * (int64_t)s.esz / 16, true);
  const int64_t nt = lnorm_threads(q.gs), groups = nt / q.gs;
  return std::min<int64_t>((s.T + groups - 1) / groups, nt == 256 ? 768 : nt == 512 ? 512 : 256);
}

// f(integral_constant GS, integral_constant CH) of a row shape
template <typename E, bool BWD, typename F>
static void with_row_shape(const RowShape& q, F&& f) {
  auto go = [&](auto GSc, auto CHc) {
    if (q.gs == GSc.value && q.ch == CHc.value) f(GSc, CHc);
  };
  const std::integral_constant<int, 1> c1;
  const std::integral_constant<int, 2> c2;
  const std::integral_constant<int, 4> c4;
  go(std::integral_constant<int, 8>{}, c1);
  go(std::integral_constant<int, 16>{}, c1);
  go(std::integral_constant<int, 32>{}, c1);
  go(std::integral_constant<int, 64>{}, c1);
  go(std::integral_constant<int, 64>{}, c2);
  go(std::integral_constant<int, 256>{}, c2);
  if constexpr (BWD) {
    go(std::integral_constant<int, 256>{}, c1);
    go(std::integral_constant<int, 512>{}, c2);
  } else {
    go(std::integral_constant<int, 64>{}, c4);
    go(std::integral_constant<int, 256>{}, c4);
  }
  go(std::integral_constant<int, 512>{}, c4);
  if constexpr (sizeof(E) == 4) go(std::integral_constant<int, 1024>{}, c4);
}

template <typename E>
static void layer_norm_fwd(const Shape& s, const void* x, const void* res, const void* gamma, const void* beta, void* sum,
                           void* y, float* stats, hipStream_t st) {
  const RowShape q = row_shape(s.D / Vec<E>::N, false);
  auto c = [](const void* p) { return reinterpret_cast<const E*>(p); };
  with_row_shape<E, false>(q, [&](auto GSc, auto CHc) {
    constexpr int GS = decltype(GSc)::value, CH = decltype(CHc)::value, NT = lnorm_threads(GS), G = NT / GS;
    const int64_t blocks = std::min<int64_t>((s.T + G - 1) / G, 256 * (2048 / NT));
    auto kern = res ? layer_norm_fwd_kernel<E, GS, CH, true> : layer_norm_fwd_kernel<E, GS, CH, false>;
    DMOE_LAUNCH_NAMED("layer_norm_fwd_kernel", kern, dim3((unsigned)blocks), dim3(NT), 0, st, c(x), c(res), c(gamma),
                      c(beta), reinterpret_cast<E*>(sum), reinterpret_cast<E*>(y), stats, (int)s.T, (int)s.D);
  });
}

template <typename E>
static void layer_norm_bwd(const Shape& s, const void* sum, const float* stats, const void* gamma, const void* dy,
                           const void* dres, void* dx, void* dgamma, void* dbeta, float* part, hipStream_t st) {
  const RowShape q = row_shape(s.D / Vec<E>::N, true);
  const int nb = (int)lnorm_bwd_blocks(s);
  auto c = [](const void* p) { return reinterpret_cast<const E*>(p); };
  if (nb > 0)
    with_row_shape<E, true>(q, [&](auto GSc, auto CHc) {
      constexpr int GS = decltype(GSc)::value, CH = decltype(CHc)::value, NT = lnorm_threads(GS);
      auto kern = dres ? layer_norm_bwd_kernel<E, GS, CH, true> : layer_norm_bwd_kernel<E, GS, CH, false>;
      DMOE_LAUNCH_NAMED("layer_norm_bwd_kernel", kern, dim3(nb), dim3(NT), 0, st, c(sum), stats, c(gamma), c(dy),
                        c(dres), reinterpret_cast<E*>(dx), part, (int)s.T, (int)s.D);
    });
  DMOE_LAUNCH_NAMED("layer_norm_reduce_kernel", layer_norm_reduce_kernel<E>, dim3((unsigned)(2 * s.D / (4 * LR_C))), dim3(LR_NT),
                    0, st, part, nb, (int)s.D, reinterpret_cast<E*>(dgamma), reinterpret_cast<E*>(dbeta));
}

}  // namespace dmoe

using namespace dmoe;

extern "C" size_t dmoe_layer_norm_workspace_bytes(const dmoe_dims* dims) {
  Shape s;
  if (check_dims(dims, &s) != DMOE_OK || s.D > LNORM_DMAX) return 0;
  return (size_t)std::max<int64_t>(1, lnorm_bwd_blocks(s)) * 2 * s.D * sizeof(float);
}

extern "C" int dmoe_layer_norm_fwd(const dmoe_dims* dims, const void* x, const void* res, const void* gamma,
                                   const void* beta, void* s_out, void* y, float* stats, void* stream) {
  Shape s;
  int rc = check_dims(dims, &s);
  if (rc) return rc;
  if (s.D > LNORM_DMAX) return DMOE_EUNSUPPORTED;
  if ((res == nullptr) != (s_out == nullptr)) return DMOE_EINVAL;
  if (s.T == 0) return DMOE_OK;
  if (!x || !gamma || !y) return DMOE_EINVAL;
  if (y == s_out) return DMOE_EINVAL;
  for (const void* q : {x, res, gamma, beta, (const void*)s_out, (const void*)y, (const void*)stats})
    if (!aligned16(q)) return DMOE_EUNSUPPORTED;
  hipStream_t st = reinterpret_cast<hipStream_t>(stream);
  if (s.dtype == DMOE_BF16) layer_norm_fwd<bf16>(s, x, res, gamma, beta, s_out, y, stats, st);
  else layer_norm_fwd<float>(s, x, res, gamma, beta, s_out, y, stats, st);
  return launch_status();
}

extern "C" int dmoe_layer_norm_bwd(const dmoe_dims* dims, const void* s_in, const float* stats, const void* gamma,
                                   const void* dy, const void* dres, void* dx, void* dgamma, void* dbeta, void* ws,
                                   void* stream) {
  Shape s;
  int rc = check_dims(dims, &s);
  if (rc) return rc;
  if (s.D > LNORM_DMAX) return DMOE_EUNSUPPORTED;
  if (!dgamma || !ws) return DMOE_EINVAL;
  if (s.T > 0 && (!s_in || !stats || !gamma || !dy || !dx)) return DMOE_EINVAL;
  for (const void* q : {s_in, (const void*)stats, gamma, dy, dres, (const void*)dx, (const void*)dgamma, (const void*)dbeta,
                        (const void*)ws})
    if (!aligned16(q)) return DMOE_EUNSUPPORTED;
  hipStream_t st = reinterpret_cast<hipStream_t>(stream);
  float* part = reinterpret_cast<float*>(ws);
  if (s.dtype == DMOE_BF16) layer_norm_bwd<bf16>(s, s_in, stats, gamma, dy, dres, dx, dgamma, dbeta, part, st);
  else layer_norm_bwd<float>(s, s_in, stats, gamma, dy, dres, dx, dgamma, dbeta, part, st);
  return launch_status();
}
