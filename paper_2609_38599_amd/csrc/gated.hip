// The gated feed-forward block y = act(a) * b, a = x Wg^T, b = x Wu^T, and its
// backward pass, for 16-bit x [T][D], Wg, Wu [F][D] (row-major).
//
// Forward: one kernel forms both products of a tile of y from one staging of x
// (the tile's P rows are Wg's and Wu's of the same channels, so a lane ends up with
// a and b of the same entry) and stores act(a) b, rounded once from fp32 sums.
//
// Backward: da = dy b act'(a), db = dy act(a) from the saved fp32 a and b, rounded
// to 16 bits as the matrix cores take them (the only rounding beside the
// outputs'; in float16 what passes 65504 is an infinity, as in any gradient held
// so); then dx = [da db] [Wg; Wu] in one product over 2 F, and
// [dWg; dWu] = [da db]^T x in one over T.

#include "skinny.h"

namespace jarq {

namespace {

constexpr float kInvSqrt2Pi = 0.39894228040143268f;
constexpr float kSqrt2OverPi = 0.79788456080286536f;

// The normal distribution function of a, e = exp(-a^2 / 2).  Phi(-u) = e v r(v) for u >= 0,
// v = 1 / (1 + 0.36 u): r is the polynomial of degree 8 of the least largest relative error
// on 0 <= u <= 40 (9e-8; 4e-7 in fp32 for u < 1, then what e is off by).  The tail stays
// right to itself where (1 + erf) / 2 cancels (4 % off at -5), and takes less than erfc: 611 x
// 1000 -> 2752 20 us, 22.
__device__ __forceinline__ float normal_cdf(float a, float e) {
  const float v = __builtin_amdgcn_rcpf(fmaf(0.36f, fabsf(a), 1.f));
  float r = -0.030238334f;
  r = fmaf(r, v, 0.13950869f);
  r = fmaf(r, v, -0.22360012f);
  r = fmaf(r, v, 0.10736972f);
  r = fmaf(r, v, -0.00038668368f);
  r = fmaf(r, v, 0.096037455f);
  r = fmaf(r, v, 0.12400974f);
  r = fmaf(r, v, 0.14368188f);
  r = fmaf(r, v, 0.14361766f);
  const float tail = e * v * r;
  return a < 0.f ? tail : 1.f - tail;
}

// act(a), and act'(a) where `d` is given
template <int ACT>
__device__ __forceinline__ float activation(float a, float* d) {
  if constexpr (ACT == 0) {          // silu
    const float sig = __builtin_amdgcn_rcpf(1.f + __expf(-a));   // to an ulp
    if (d) *d = sig * (1.f + a * (1.f - sig));
    return a * sig;
  } else if constexpr (ACT == 1) {   // gelu
    const float e = __expf(-0.5f * a * a), cdf = normal_cdf(a, e);
    if (d) *d = cdf + a * kInvSqrt2Pi * e;
    return a * cdf;
  } else {                           // gelu, tanh form: (1 + tanh z) / 2 = 1 / (1 + exp(-2 z))
    const float aa = fminf(a * a, 1e30f);   // (0 times it stays 0)
    const float z = kSqrt2OverPi * (a + 0.044715f * a * aa);
    const float sig = __builtin_amdgcn_rcpf(1.f + __expf(-2.f * z));
    if (d)
      *d = sig + sig * (1.f - sig) * a * (2.f * kSqrt2OverPi * (1.f + 3.f * 0.044715f * aa));
    return a * sig;
  }
}
__device__ __forceinline__ float activation(int act, float a, float* d) {   // act is uniform
  if (act == 0) return activation<0>(a, d);
  if (act == 1) return activation<1>(a, d);
  return activation<2>(a, d);
}

}  // namespace

// ---- forward, many tokens ----
// WI x WJ wavefronts, each BI blocks of 16 P rows (half Wg's, half Wu's) x BJ blocks
// of 16 tokens.  Bound by the matrix cores at the clock that the card's power allows:
// 4096 tokens, 4096 -> 14336 in bf16 780 us, 1.23 PFLOP/s; with a and b stored as well
// 4096 -> 11008 690 us, as long as 12288 channels: five rounds of 256 tiles and a third of a
// sixth.  53 tokens, 4096 -> 14336: 224 work-groups, 54 us, 4.4 TB/s of weights.
template <int KIND, int S, int WI, int WJ, int BI, int BJ>
__global__ __launch_bounds__(64 * WI * WJ) JARQ_WAVES(2) void gated_tile_kernel(
    const void* __restrict__ X, const void* __restrict__ Wg, const void* __restrict__ Wu, int T,
    int D, int F, int act, uint16_t* __restrict__ Y, float* __restrict__ pre, int ni, int nj) {
  constexpr int TI = 16 * WI * BI, TJ = 16 * WJ * BJ, NW = WI * WJ;
  typedef KContig<TI, NW, kRowHalves> LP;
  typedef KContig<TJ, NW, kOne> LQ;
  constexpr int STAGE = LP::kBytes + LQ::kBytes;
  JARQ_STAGES(S, STAGE);
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wi = wave / WJ, wj = wave % WJ;
  int ti, tj;
  xcd_tile(blockIdx.x, ni, nj, ti, tj);
  const int f0 = ti * (TI / 2), t0 = tj * TJ;
  LP lp;
  LQ lq;
  lp.init(Wg, Wu, 2 * (size_t)D, f0, F, 2 * D, wave, lane);
  lq.init(X, X, 2 * (size_t)D, t0, T, 2 * D, wave, lane);
  f32x4 acc[BI][BJ] = {};
  // block a < BI / 2: Wg, the others: Wu of the same channels
  mma_loop<S, BI, BJ>(lp, lq, 0, (2 * D + kChunk - 1) / kChunk, lane, wi * 8 * BI, wj * 16 * BJ,
                   stages, [](int) {},
                   [&](const u32x4& p, const u32x4& q, int a, int b, int)
                       __attribute__((always_inline)) {
                         acc[a][b] = Mma<KIND>::mul(p, q, acc[a][b]);
                       });
  // Out through LDS, 32 tokens of a wave column at a time: memory gets whole lines (8
  // bytes a lane straight from the registers took 75 us of 800), and the activation's code is
  // there once, not once a value: 10 KB a kernel, which fits the instruction cache, not 57.
  constexpr int RB = TI / 2 * 4, PIECES = RB / 16;   // a row: one projection's fp32
  constexpr bool APART = WJ == 2;                    // two stages a column, else one
  static_assert((APART ? 1 : 2) * 32 * RB <= STAGE && (WJ == 2 || WJ == 4), "stage");
  char* const ga = wj == 0 ? stage0 : wj == 1 ? stage1 : wj == 2 ? stage2 : stage3;
  char* const up = APART ? (wj == 0 ? stage2 : stage3) : ga + 32 * RB;
#pragma unroll
  for (int bb = 0; bb < BJ; bb += 2) {
    if (bb > 0) __syncthreads();
#pragma unroll
    for (int b = bb; b < bb + 2; ++b)
#pragma unroll
      for (int a = 0; a < BI / 2; ++a) {
        const int row = 16 * (b - bb) + (lane & 15);
        const int c = (wi * 8 * BI + 16 * a + 4 * (lane >> 4)) / 4;
        *(f32x4*)out_piece<RB>(ga, row, c) = acc[a][b];
        *(f32x4*)out_piece<RB>(up, row, c) = acc[BI / 2 + a][b];
      }
    __syncthreads();
    const int tb = t0 + wj * 16 * BJ + 16 * bb;
#pragma unroll 1
    for (int p = wi * 64 + lane; p < 32 * PIECES; p += WI * 64) {
      const int r = p / PIECES, c = p % PIECES, t = tb + r, f = f0 + 4 * c;
      const f32x4 g = *(const f32x4*)out_piece<RB>(ga, r, c);
      const f32x4 u = *(const f32x4*)out_piece<RB>(up, r, c);
      if (t < T && f < F) {
        const size_t e = (size_t)t * F + f;
        if (pre) {
          *(f32x4*)(pre + e) = g;
          *(f32x4*)(pre + (size_t)T * F + e) = u;
        }
        float y[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) y[i] = activation(act, g[i], nullptr) * u[i];
        *(u32x2*)(Y + e) = u32x2{pack16<KIND>(y[0], y[1]), pack16<KIND>(y[2], y[3])};
      }
    }
  }
}

// ---- forward, few tokens ----
// A work-group: 16 channels of both projections x up to 16 IB tokens, eight wavefronts
// along k.  One token, 4096 -> 11008: 35 us, 5.2 TB/s of weights (32 channels: 45 us).
template <int KIND, int IB>
__global__ __launch_bounds__(512) void gated_skinny_kernel(
    const void* __restrict__ X, const void* __restrict__ Wg, const void* __restrict__ Wu, int T,
    int D, int F, int act, uint16_t* __restrict__ Y, float* __restrict__ pre) {
  constexpr int NW = 8;
  __shared__ __attribute__((aligned(16))) float red[NW * IB * 2 * 256];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int f0 = blockIdx.x * 16;
  const int row = lane & 15;
  const size_t ld = 2 * (size_t)D, wrow = (size_t)min(f0 + row, F - 1) * ld;
  const char* p[IB];
#pragma unroll
  for (int a = 0; a < IB; ++a) p[a] = (const char*)X + (size_t)min(16 * a + row, T - 1) * ld;
  const char* const q[2] = {(const char*)Wg + wrow, (const char*)Wu + wrow};
  f32x4 acc[IB][2] = {};
  skinny_loop<IB, 2, 4, NW>(
      p, q, 2 * D, wave, lane, [](int, int) {},
      [&](int, int, const u32x4(&fp)[IB], const u32x4(&fq)[2]) __attribute__((always_inline)) {
#pragma unroll
        for (int a = 0; a < IB; ++a)
#pragma unroll
          for (int b = 0; b < 2; ++b) acc[a][b] = Mma<KIND>::mul(fp[a], fq[b], acc[a][b]);
      });
#pragma unroll
  for (int a = 0; a < IB; ++a)
#pragma unroll
    for (int b = 0; b < 2; ++b)
      *(f32x4*)(red + ((wave * IB + a) * 2 + b) * 256 + 4 * lane) = acc[a][b];
  __syncthreads();
  for (int e = threadIdx.x; e < IB * 256; e += 512) {
    const int j = e & 15, i = (e >> 4) & 15, a = e >> 8;
    const int t = 16 * a + i, f = f0 + j;
    if (t < T && f < F) {
      const float g = skinny_sum<NW, 2 * IB>(red, 2 * a, i, j);
      const float u = skinny_sum<NW, 2 * IB>(red, 2 * a + 1, i, j);
      const size_t at = (size_t)t * F + f;
      Y[at] = to16<KIND>(activation(act, g, nullptr) * u);
      if (pre) {
        pre[at] = g;
        pre[(size_t)T * F + at] = u;
      }
    }
  }
}

template <int KIND, int S, int WI, int WJ, int BI, int BJ>
static hipError_t launch_gated_tiles(hipStream_t st, int act, int T, int D, int F, const void* X,
                                     const void* Wg, const void* Wu, uint16_t* Y, float* pre) {
  const int ni = (F + 8 * WI * BI - 1) / (8 * WI * BI);
  const int nj = (T + 16 * WJ * BJ - 1) / (16 * WJ * BJ);
  hipLaunchKernelGGL((gated_tile_kernel<KIND, S, WI, WJ, BI, BJ>), dim3((unsigned)(ni * nj)),
                     dim3(64 * WI * WJ), 0, st, X, Wg, Wu, T, D, F, act, Y, pre, ni, nj);
  return hipGetLastError();
}

// Up to 32 tokens fragments straight from memory (24 tokens, 4096 -> 11008: 48 us, tiles
// of 64 channels 54); beyond, the tiles that tile_cost makes the cheapest.  4096 -> 1000,
// 2752 and 11008 channels, in us with tiles of 128 x 256 (channels x tokens), 64 x 128,
// 64 x 64 and 32 x 64:
//    100 tokens   69 26 19 17    71 31 25 19    73  38  49  48
//    400          72 31 26 19    73 34 44 58    91 113 125 145
//   1600          74 37 51 59    88 104 127 149 280 337 443 515
template <int KIND>
static hipError_t launch_gated_forward_kind(hipStream_t st, int act, int T, int D, int F,
                                            const void* X, const void* Wg, const void* Wu,
                                            void* Y, float* pre) {
  uint16_t* y = (uint16_t*)Y;
  if (T <= 32) {
    const dim3 wg((F + 15) / 16);
    if (T <= 16)
      hipLaunchKernelGGL((gated_skinny_kernel<KIND, 1>), wg, dim3(512), 0, st, X, Wg, Wu, T, D, F,
                         act, y, pre);
    else
      hipLaunchKernelGGL((gated_skinny_kernel<KIND, 2>), wg, dim3(512), 0, st, X, Wg, Wu, T, D, F,
                         act, y, pre);
    return hipGetLastError();
  }
  auto tiles = [&](int f, int t) { return (long long)((F + f - 1) / f) * ((T + t - 1) / t); };
  const int nk = (2 * D + kChunk - 1) / kChunk;
  const double cost[4] = {tile_cost(tiles(128, 256), nk, {6.0, 0.62, 6.0, 0.62}),
                          tile_cost(tiles(64, 128), nk, {3.3, 0.26, 3.3, 0.26}),
                          tile_cost(tiles(64, 64), nk, {2.7, 0.19, 2.7, 0.19}),
                          tile_cost(tiles(32, 64), nk, {2.6, 0.135, 2.6, 0.135})};
  switch ((int)(std::min_element(cost, cost + 4) - cost)) {
    case 0: return launch_gated_tiles<KIND, 4, 2, 4, 8, 4>(st, act, T, D, F, X, Wg, Wu, y, pre);
    case 1: return launch_gated_tiles<KIND, 4, 2, 2, 4, 4>(st, act, T, D, F, X, Wg, Wu, y, pre);
    case 2: return launch_gated_tiles<KIND, 4, 2, 2, 4, 2>(st, act, T, D, F, X, Wg, Wu, y, pre);
    default: return launch_gated_tiles<KIND, 8, 1, 2, 4, 2>(st, act, T, D, F, X, Wg, Wu, y, pre);
  }
}

hipError_t launch_gated_forward(hipStream_t st, int dtype, int act, int T, int D, int F,
                                const void* X, const void* Wg, const void* Wu, void* Y,
                                float* pre) {
  return dtype == kBF16
             ? launch_gated_forward_kind<kBF16>(st, act, T, D, F, X, Wg, Wu, Y, pre)
             : launch_gated_forward_kind<kF16>(st, act, T, D, F, X, Wg, Wu, Y, pre);
}

// ---- backward: da, db ----
// dab [T][2 F]: da in columns 0..F-1, db behind.  Eight entries a thread.  Bound by
// memory, 14 bytes an entry: 4096 x 11008 127 us, 5.0 TB/s.  (Formed inside the two products
// each entry's would be computed D / 256 + 2 F / 256 times.)
template <int KIND>
__global__ __launch_bounds__(256) void gated_grad_kernel(const float* __restrict__ pre,
                                                         const uint16_t* __restrict__ dY, int T,
                                                         int F, int act,
                                                         uint16_t* __restrict__ dab) {
  const size_t n = (size_t)T * F, f8 = (size_t)(F / 8);
  for (size_t e = (size_t)blockIdx.x * 256 + threadIdx.x; e < n / 8;
       e += (size_t)gridDim.x * 256) {
    const size_t t = e / f8, f = (e - t * f8) * 8;
    const size_t at = 8 * e;
    f32x4 g[2], u[2];
    g[0] = *(const f32x4*)(pre + at);
    g[1] = *(const f32x4*)(pre + at + 4);
    u[0] = *(const f32x4*)(pre + n + at);
    u[1] = *(const f32x4*)(pre + n + at + 4);
    const u32x4 dy = *(const u32x4*)(dY + at);
    u32x4 da, db;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      float ga[2], gb[2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int v = 2 * w + h;
        const float d = from16<KIND>((uint16_t)(dy[w] >> (16 * h)));
        float slope;
        const float s = activation(act, g[v >> 2][v & 3], &slope);
        ga[h] = d * u[v >> 2][v & 3] * slope;
        gb[h] = d * s;
      }
      da[w] = pack16<KIND>(ga[0], ga[1]);
      db[w] = pack16<KIND>(gb[0], gb[1]);
    }
    uint16_t* out = dab + t * (2 * (size_t)F) + f;
    *(u32x4*)out = da;
    *(u32x4*)(out + F) = db;
  }
}

// ---- backward: dx = dab [Wg; Wu] ----
// part: fp32 partial sums [split][T][D] where the 2 F are cut over blockIdx.y.  Wg and Wu
// are read as they lie (k down the rows) through the transposing LDS read.  Bound by the
// matrix cores: 4096 tokens, 4096 channels, F = 11008 550 us, 1.35 PFLOP/s: one round of 256
// tiles.
template <int KIND, int S, int WI, int WJ, int BI, int BJ>
__global__ __launch_bounds__(64 * WI * WJ) JARQ_WAVES(2) void gated_dx_kernel(
    const void* __restrict__ dab, const void* __restrict__ Wg, const void* __restrict__ Wu, int T,
    int D, int F, int each, uint16_t* __restrict__ dX, float* __restrict__ part, int ni, int nj) {
  constexpr int TI = 16 * WI * BI, TJ = 16 * WJ * BJ, NW = WI * WJ;
  typedef KStrided<TI, NW, kTwoSpans> LP;
  typedef KContig<TJ, NW, kTwoSpans> LQ;
  constexpr int STAGE = LP::kBytes + LQ::kBytes;
  JARQ_STAGES(S, STAGE);
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wi = wave / WJ, wj = wave % WJ;
  int ti, tj;
  xcd_tile(blockIdx.x, ni, nj, ti, tj);
  const int d0 = ti * TI, t0 = tj * TJ;
  LP lp;
  LQ lq;
  lp.init(Wg, Wu, 2 * (size_t)D, d0, D, F, wave, lane);
  lq.init(dab, (const uint16_t*)dab + F, 4 * (size_t)F, t0, T, 2 * F, wave, lane);
  f32x4 acc[BI][BJ] = {};
  const int nk = 2 * ((2 * F + kChunk - 1) / kChunk);
  const int q0 = blockIdx.y * each, q1 = min(q0 + each, nk);
  mma_loop<S, BI, BJ>(lp, lq, q0, q1, lane, wi * 16 * BI, wj * 16 * BJ, stages,
                   [](int) {},
                   [&](const u32x4& p, const u32x4& q, int a, int b, int)
                       __attribute__((always_inline)) {
                         acc[a][b] = Mma<KIND>::mul(p, q, acc[a][b]);
                       });
  if (part) {   // uniform
#pragma unroll
    for (int b = 0; b < BJ; ++b) {
      const int t = t0 + wj * 16 * BJ + 16 * b + (lane & 15);
#pragma unroll
      for (int a = 0; a < BI; ++a) {
        const int d = d0 + wi * 16 * BI + 16 * a + 4 * (lane >> 4);
        if (t < T && d < D) *(f32x4*)(part + ((size_t)blockIdx.y * T + t) * D + d) = acc[a][b];
      }
    }
    return;
  }
  char* const stage = wj == 0 ? stage0 : wj == 1 ? stage1 : wj == 2 ? stage2 : stage3;
  const int tw = t0 + wj * 16 * BJ;
  store_tile16<KIND, WI, BI, BJ>(acc, stage, wi, lane, [&](int t, int i, const u32x4& w) {
    if (tw + t < T && d0 + i < D) *(u32x4*)(dX + (size_t)(tw + t) * D + d0 + i) = w;
  });
}

// The parts' sums in their order, rounded once.  Bound by a small launch's latency: 611 x
// 1000 in three parts 4 us.
template <int KIND>
__global__ __launch_bounds__(256) void gated_dx_sum_kernel(const float* __restrict__ part,
                                                           int splits, size_t n,
                                                           uint16_t* __restrict__ dX) {
  for (size_t e = 4 * ((size_t)blockIdx.x * 256 + threadIdx.x); e < n;
       e += 4 * (size_t)gridDim.x * 256) {
    f32x4 s = *(const f32x4*)(part + e);
    for (int k = 1; k < splits; ++k) s += *(const f32x4*)(part + k * n + e);
    *(u32x2*)(dX + e) = u32x2{pack16<KIND>(s[0], s[1]), pack16<KIND>(s[2], s[3])};
  }
}

// ---- backward: [dWg; dWu] = dab^T x ----
// Both operands have k (the tokens) down their rows.  Bound by the matrix cores: 4096
// tokens, 4096 channels, F = 11008 580 us, 1.27 PFLOP/s.  What it lacks to dx is its last
// round of tiles, a third full: F = 12288, six whole rounds, 618 us, dx 629.
template <int KIND, int S, int WI, int WJ, int BI, int BJ>
__global__ __launch_bounds__(64 * WI * WJ) JARQ_WAVES(2) void gated_dw_kernel(
    const void* __restrict__ dab, const void* __restrict__ X, int T, int D, int F,
    uint16_t* __restrict__ dWg, uint16_t* __restrict__ dWu, int ni, int nj) {
  constexpr int TI = 16 * WI * BI, TJ = 16 * WJ * BJ, NW = WI * WJ;
  typedef KStrided<TI, NW, kOne> LP;
  typedef KStrided<TJ, NW, kOne> LQ;
  constexpr int STAGE = LP::kBytes + LQ::kBytes;
  JARQ_STAGES(S, STAGE);
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wi = wave / WJ, wj = wave % WJ;
  int ti, tj;
  xcd_tile(blockIdx.x, ni, nj, ti, tj);
  const int d0 = ti * TI, f0 = tj * TJ;
  LP lp;
  LQ lq;
  lp.init(X, X, 2 * (size_t)D, d0, D, T, wave, lane);
  lq.init(dab, dab, 4 * (size_t)F, f0, 2 * F, T, wave, lane);
  f32x4 acc[BI][BJ] = {};
  mma_loop<S, BI, BJ>(lp, lq, 0, (2 * T + kChunk - 1) / kChunk, lane, wi * 16 * BI, wj * 16 * BJ,
                   stages, [](int) {},
                   [&](const u32x4& p, const u32x4& q, int a, int b, int)
                       __attribute__((always_inline)) {
                         acc[a][b] = Mma<KIND>::mul(p, q, acc[a][b]);
                       });
  char* const stage = wj == 0 ? stage0 : wj == 1 ? stage1 : wj == 2 ? stage2 : stage3;
  const int fw = f0 + wj * 16 * BJ;
  store_tile16<KIND, WI, BI, BJ>(acc, stage, wi, lane, [&](int r, int i, const u32x4& w) {
    const int f = fw + r;
    uint16_t* out = f < F ? dWg : dWu;
    if (f < 2 * F && d0 + i < D && out)
      *(u32x4*)(out + (size_t)(f < F ? f : f - F) * D + d0 + i) = w;
  });
}

namespace {

struct DxPlan {
  int kind;   // tiles of 256 x 256 (channels x tokens), 128 x 128, 128 x 64
  int ni, nj, splits, each;
};
// The tiles and the number of parts of the 2 F that cost the least, with the parts'
// fp32 sums written and read again.  4096 channels, F = 11008: 400 tokens 256-wide tiles in
// 4 parts 117 us, 128-wide ones in 1, 2, 4 parts 171, 99, 98; 1600 tokens 256-wide ones in
// 1, 2, 4 parts 388, 229, 288, 128-wide ones 357.
DxPlan dx_plan(int T, int D, int F) {
  const int nk = 2 * ((2 * F + kChunk - 1) / kChunk);
  constexpr int wide[3] = {256, 128, 128}, tall[3] = {256, 128, 64};
  constexpr TileTime time[3] = {
      {8.0, 0.62, 8.0, 0.62}, {4.0, 0.26, 4.0, 0.26}, {3.0, 0.19, 3.0, 0.19}};
  DxPlan best{};
  double least = 0.0;
  for (int kind = 0; kind < 3; ++kind) {
    const int ni = (D + wide[kind] - 1) / wide[kind], nj = (T + tall[kind] - 1) / tall[kind];
    for (int parts = 1; parts <= 16; ++parts) {
      const int each = ((nk + parts - 1) / parts + 3) / 4 * 4;   // whole rounds of stages
      const int splits = (nk + each - 1) / each;
      if (splits != parts) continue;
      double cost = tile_cost((long long)ni * nj * splits, each, time[kind]);
      if (splits > 1) cost += 5.0 + 8e-6 * splits / 4.0 * T * D;
      if (best.splits == 0 || cost < least) {
        least = cost;
        best = {kind, ni, nj, splits, each};
      }
    }
  }
  return best;
}

size_t pad256(size_t n) { return (n + 255) & ~(size_t)255; }

}  // namespace

size_t gated_workspace_bytes(int T, int D, int F) {
  const DxPlan p = dx_plan(T, D, F);
  return pad256(4 * (size_t)T * F) +
         (p.splits > 1 ? pad256(4 * (size_t)p.splits * T * D) : 0);
}

// The weights' gradient of no tokens.
__global__ __launch_bounds__(256) void gated_zero_kernel(u32x4* out, size_t n) {
  for (size_t e = (size_t)blockIdx.x * 256 + threadIdx.x; e < n; e += (size_t)gridDim.x * 256)
    out[e] = u32x4{};
}

template <int KIND>
static hipError_t launch_gated_backward_kind(hipStream_t st, int act, int T, int D, int F,
                                             const void* X, const void* Wg, const void* Wu,
                                             const void* dY, const float* pre, void* dX, void* dWg,
                                             void* dWu, char* ws) {
  if (T == 0) {
    for (void* out : {dWg, dWu}) {
      if (!out) continue;
      hipLaunchKernelGGL(gated_zero_kernel, dim3(1024), dim3(256), 0, st, (u32x4*)out,
                         (size_t)F * D / 8);
      const hipError_t e = hipGetLastError();
      if (e != hipSuccess) return e;
    }
    return hipSuccess;
  }
  uint16_t* dab = (uint16_t*)ws;
  float* part = (float*)(ws + pad256(4 * (size_t)T * F));
  const size_t n8 = (size_t)T * F / 8;
  const size_t blocks = (n8 + 255) / 256 < 16384 ? (n8 + 255) / 256 : 16384;
  hipLaunchKernelGGL((gated_grad_kernel<KIND>), dim3((unsigned)blocks), dim3(256), 0, st, pre,
                     (const uint16_t*)dY, T, F, act, dab);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  if (dX) {
    const DxPlan p = dx_plan(T, D, F);
    float* to = p.splits > 1 ? part : nullptr;
    const dim3 grid((unsigned)(p.ni * p.nj), (unsigned)p.splits);
    if (p.kind == 0)
      hipLaunchKernelGGL((gated_dx_kernel<KIND, 4, 2, 4, 8, 4>), grid, dim3(512), 0, st, dab, Wg,
                         Wu, T, D, F, p.each, (uint16_t*)dX, to, p.ni, p.nj);
    else if (p.kind == 1)
      hipLaunchKernelGGL((gated_dx_kernel<KIND, 4, 2, 2, 4, 4>), grid, dim3(256), 0, st, dab, Wg,
                         Wu, T, D, F, p.each, (uint16_t*)dX, to, p.ni, p.nj);
    else
      hipLaunchKernelGGL((gated_dx_kernel<KIND, 4, 2, 2, 4, 2>), grid, dim3(256), 0, st, dab, Wg,
                         Wu, T, D, F, p.each, (uint16_t*)dX, to, p.ni, p.nj);
    if ((e = hipGetLastError()) != hipSuccess) return e;
    if (to) {
      const size_t n = (size_t)T * D, b = (n / 4 + 255) / 256;
      hipLaunchKernelGGL((gated_dx_sum_kernel<KIND>), dim3((unsigned)(b < 4096 ? b : 4096)),
                         dim3(256), 0, st, part, p.splits, n, (uint16_t*)dX);
      if ((e = hipGetLastError()) != hipSuccess) return e;
    }
  }
  if (dWg || dWu) {
    // 256-wide tiles from 320 on (1600 tokens, 1000 channels, F = 11008, 344 of them: 69 us,
    // 128-wide 74; 4096, F = 1000, 128 of them: 36 and 27), 128-wide ones from 192 on (1000
    // channels, F = 2752, 344 of them: 26, 128 x 64 30; F = 1000, 128 of them: 16 and 14)
    const int ni = (D + 127) / 128, bi = (D + 255) / 256, bj = (2 * F + 255) / 256;
    const int nj = (2 * F + 127) / 128, nh = (2 * F + 63) / 64;
    if ((long long)bi * bj >= 320)
      hipLaunchKernelGGL((gated_dw_kernel<KIND, 4, 2, 4, 8, 4>), dim3((unsigned)(bi * bj)),
                         dim3(512), 0, st, dab, X, T, D, F, (uint16_t*)dWg, (uint16_t*)dWu, bi,
                         bj);
    else if ((long long)ni * nj >= 192)
      hipLaunchKernelGGL((gated_dw_kernel<KIND, 4, 2, 2, 4, 4>), dim3((unsigned)(ni * nj)),
                         dim3(256), 0, st, dab, X, T, D, F, (uint16_t*)dWg, (uint16_t*)dWu, ni,
                         nj);
    else
      hipLaunchKernelGGL((gated_dw_kernel<KIND, 4, 2, 2, 4, 2>), dim3((unsigned)(ni * nh)),
                         dim3(256), 0, st, dab, X, T, D, F, (uint16_t*)dWg, (uint16_t*)dWu, ni,
                         nh);
    e = hipGetLastError();
  }
  return e;
}

hipError_t launch_gated_backward(hipStream_t st, int dtype, int act, int T, int D, int F,
                                 const void* X, const void* Wg, const void* Wu, const void* dY,
                                 const float* pre, void* dX, void* dWg, void* dWu, char* ws) {
  return dtype == kBF16 ? launch_gated_backward_kind<kBF16>(st, act, T, D, F, X, Wg, Wu, dY, pre,
                                                            dX, dWg, dWu, ws)
                        : launch_gated_backward_kind<kF16>(st, act, T, D, F, X, Wg, Wu, dY, pre,
                                                           dX, dWg, dWu, ws);
}

}  // namespace jarq
