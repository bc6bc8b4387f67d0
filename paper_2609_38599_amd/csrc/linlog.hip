// Log probabilities of given tokens straight from hidden states x [T][D] and the output
// layer's weights w [V][D], 16-bit both, and their gradients, without the logits.
//
// Forward: a tile of l = x w^T leaves its maximum and the sum of exponentials beside the
// maximum's own 1 for each token (kept apart, as in the pass over stored logits: where one entry
// takes nearly all, log p of it is log(1 + that sum)), and the target's logit; the tiles' are
// joined in a fixed order.
//
// Backward, in pieces of the vocabulary: the piece's logits again,
//     dl = g 1{v = target} + (h - g) exp(l - lse)
// in 16 bits as the matrix cores take them, then dx += dl w (fp32 sums between the pieces) and
// dw = dl^T x.  Forming the logits twice is a quarter of the work; kept, they would be T V
// values in memory.  In fp16 dl is scaled by a power of two, the largest finite |g|, |h| and
// |h - g| to 2^14, so that what is 2^-38 of it is not lost; the sums are scaled back in fp32.
#include <float.h>

#include "mma_pairs.h"
#include "skinny.h"

namespace jarq {

namespace {

// The maximum (at least -FLT_MAX) and the sum of exp(x - m) beside its own 1; -1: no entry
// above -infinity.
struct Part {
  float m, more;
};
__device__ __forceinline__ Part no_part() { return Part{-FLT_MAX, -1.f}; }
__device__ __forceinline__ Part join(const Part& s, const Part& o) {
  const bool first = s.m >= o.m;
  const Part a = first ? s : o, b = first ? o : s;
  return Part{a.m, fmaf(__expf(b.m - a.m), 1.f + b.more, a.more)};
}
__device__ __forceinline__ Part of_lane(const Part& s, int off) {
  return Part{__shfl_xor(s.m, off), __shfl_xor(s.more, off)};
}
constexpr float kLog2e = 1.44269504088896340736f;
// N entries (a power of two); -infinity has no part, +infinity and NaN make it NaN.  The largest
// by a tournament: every other entry loses once, and the losers' exponentials are the sum beside
// the largest's own 1, ties included.  Differences from it are taken before they are scaled: exact
// near it however far it is from 0.  (Nine issue slots an entry, four of them the exponential;
// thirteen with a maximum first and the entries that equal it counted.)
template <int N>
__device__ __forceinline__ Part part_of(float (&x)[N]) {
#pragma unroll
  for (int s = N / 2; s >= 1; s /= 2)
#pragma unroll
    for (int i = 0; i < s; ++i) {
      const float hi = __builtin_elementwise_maximum(x[i], x[i + s]);   // (NaN wins)
      x[i + s] = __builtin_elementwise_minimum(x[i], x[i + s]);
      x[i] = hi;
    }
  const bool none = x[0] == -INFINITY;
  const float m = none ? 0.f : x[0];
  float more = 0.f;
#pragma unroll
  for (int i = 1; i < N; ++i) more += __builtin_amdgcn_exp2f((x[i] - m) * kLog2e);
  // (one entry has no losers to carry a NaN)
  return Part{none ? -FLT_MAX : m, none ? -1.f : fabsf(m) < INFINITY ? more : NAN};
}

}  // namespace

// ---- forward, many tokens ----
// WI x WJ wavefronts, each BI blocks of 16 rows of w x BJ blocks of 16 tokens.  Bound by the matrix
// cores at the clock that the card's power allows: 4096 tokens, 128000 x 4096 in bf16 3.0 ms,
// 1.43 PFLOP/s (a large library product with the logits stored: 1.45 to 1.52); 2047 x 32001 400 to 420 us.
// On zeros, at the full clock, 1.88 PFLOP/s.  Tiles that go on with the next while they finish one
// (256 work-groups that stay) took as long.
template <int KIND, int SP, int SQ, int WI, int WJ, int BI, int BJ>
__global__ __launch_bounds__(64 * WI * WJ) JARQ_WAVES(2) void linlog_tile_kernel(
    const void* __restrict__ X, const void* __restrict__ W, int T, int D, int V,
    const int64_t* __restrict__ targets, float* __restrict__ target_logit,
    float2* __restrict__ part, int ni, int nj) {
  constexpr int TI = 16 * WI * BI, TJ = 16 * WJ * BJ, NW = WI * WJ;
  typedef PairContig<TI, NW> LP;
  typedef PairContig<TJ, NW> LQ;
  JARQ_SLOTS(SP, SQ, LP::kBytes, LQ::kBytes);
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wi = wave / WJ, wj = wave % WJ;
  int ti, tj;
  xcd_tile(blockIdx.x, ni, nj, ti, tj);
  const int v0 = ti * TI, t0 = tj * TJ;
  LP lp;
  LQ lq;
  lp.init(W, 2 * (size_t)D, v0, V, 2 * D, wave, lane);
  lq.init(X, 2 * (size_t)D, t0, T, 2 * D, wave, lane);
  f32x4 acc[BI][BJ] = {};
  mma_pairs<SP, SQ, BI, BJ>(lp, lq, 0, (2 * D + kChunk - 1) / kChunk, lane, wi * 16 * BI,
                            wj * 16 * BJ, pslots, qslots,
                            [&](const u32x4& p, const u32x4& q, int a, int b)
                                __attribute__((always_inline)) {
                                  acc[a][b] = Mma<KIND>::mul(p, q, acc[a][b]);
                                });
  static_assert(WI <= 2 && TJ * 8 <= LP::kBytes, "the other wave's parts fit a stage");
  float2* const red = (float2*)pslot0;
  const int vw = v0 + wi * 16 * BI + 4 * (lane >> 4);   // this lane's first row of w
  const int tw = wj * 16 * BJ + (lane & 15);            // its first token in the tile
  Part parts[BJ];
#pragma unroll
  for (int b = 0; b < BJ; ++b) {
    const int t = t0 + tw + 16 * b;
    float x[4 * BI];
#pragma unroll
    for (int a = 0; a < BI; ++a)
#pragma unroll
      for (int i = 0; i < 4; ++i) x[4 * a + i] = acc[a][b][i];
    // (rows past the last one are copies of it: only a last tile has any)
    if (v0 + TI > V)
#pragma unroll
      for (int a = 0; a < BI; ++a)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (vw + 16 * a + i >= V) x[4 * a + i] = -INFINITY;
    const int64_t at = t < T ? targets[t] - vw : -1;
    if (__any(at >= 0 && at < 16 * BI && at < V - vw)) {   // of few tiles
#pragma unroll
      for (int a = 0; a < BI; ++a)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (at == 16 * a + i && vw + 16 * a + i < V) target_logit[t] = x[4 * a + i];
    }
    Part s = part_of(x);
    s = join(s, of_lane(s, 16));
    parts[b] = join(s, of_lane(s, 32));
  }
  if constexpr (WI == 2) {
    if (wi == 1)
#pragma unroll
      for (int b = 0; b < BJ; ++b)
        if (lane < 16) red[tw + 16 * b] = make_float2(parts[b].m, parts[b].more);
    __syncthreads();
  }
  if (wi == 0 && lane < 16)
#pragma unroll
    for (int b = 0; b < BJ; ++b) {
      Part s = parts[b];
      if constexpr (WI == 2) {
        const float2 o = red[tw + 16 * b];
        s = join(s, Part{o.x, o.y});
      }
      const int t = t0 + tw + 16 * b;
      if (t < T) part[(size_t)ti * T + t] = make_float2(s.m, s.more);
    }
}

// ---- forward, few tokens ----
// The parts of logits of 16 JB rows of w (of `rows`, from r0 on) and up to 16 IB tokens by eight
// wavefronts along k, for skinny_sum.  The backward pass takes its logits from the same sums: those
// of the tiles above are off by other roundings, which large logits turn into other probabilities.
template <int KIND, int IB, int JB>
__device__ __forceinline__ void few_logits(const void* X, const void* W, int T, int D, int rows,
                                           int r0, float* red) {
  constexpr int NW = 8;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int row = lane & 15;
  const size_t ld = 2 * (size_t)D;
  const char* p[IB];
#pragma unroll
  for (int a = 0; a < IB; ++a) p[a] = (const char*)X + (size_t)min(16 * a + row, T - 1) * ld;
  const char* q[JB];
#pragma unroll
  for (int b = 0; b < JB; ++b)
    q[b] = (const char*)W + (size_t)min(r0 + 16 * b + row, rows - 1) * ld;
  f32x4 acc[IB][JB] = {};
  skinny_loop<IB, JB, 4, NW>(
      p, q, 2 * D, wave, lane, [](int, int) {},
      [&](int, int, const u32x4(&fp)[IB], const u32x4(&fq)[JB]) __attribute__((always_inline)) {
#pragma unroll
        for (int a = 0; a < IB; ++a)
#pragma unroll
          for (int b = 0; b < JB; ++b) acc[a][b] = Mma<KIND>::mul(fp[a], fq[b], acc[a][b]);
      });
#pragma unroll
  for (int a = 0; a < IB; ++a)
#pragma unroll
    for (int b = 0; b < JB; ++b)
      *(f32x4*)(red + ((wave * IB + a) * JB + b) * 256 + 4 * lane) = acc[a][b];
  __syncthreads();
}

// Bound by reading w: one token, 128000 x 4096 166 us, 6.3 TB/s; 181 among other kernels, which
// leave less of w in the last cache (32 rows a work-group 8 % longer).
template <int KIND, int IB, int JB>
__global__ __launch_bounds__(512) void linlog_skinny_kernel(
    const void* __restrict__ X, const void* __restrict__ W, int T, int D, int V,
    const int64_t* __restrict__ targets, float* __restrict__ target_logit,
    float2* __restrict__ part) {
  constexpr int NW = 8;
  __shared__ __attribute__((aligned(16))) float red[NW * IB * JB * 256];
  const int v0 = blockIdx.x * (16 * JB);
  few_logits<KIND, IB, JB>(X, W, T, D, V, v0, red);
  for (int e = threadIdx.x; e < IB * JB * 256; e += 512) {   // 16 JB lanes a token
    const int j = e & (16 * JB - 1), t = e / (16 * JB), v = v0 + j;
    if (t >= T) continue;
    const float x = skinny_sum<NW, JB * IB>(red, JB * (t >> 4) + (j >> 4), t & 15, j & 15);
    Part s = no_part();
    if (v < V) {
      float one[1] = {x};
      s = part_of(one);
      if (targets[t] == v) target_logit[t] = x;
    }
#pragma unroll
    for (int off = 8 * JB; off >= 1; off >>= 1) s = join(s, of_lane(s, off));
    if (j == 0) part[(size_t)blockIdx.x * T + t] = make_float2(s.m, s.more);
  }
}

// A token's parts in a fixed order: `tw` tokens a work-group (a power of two), 256 / tw shares of
// the parts each.
__global__ __launch_bounds__(256) void linlog_join_kernel(
    const float2* __restrict__ part, int parts, int T, int V, int tw,
    const int64_t* __restrict__ targets, const float* __restrict__ target_logit,
    float* __restrict__ logprob, float* __restrict__ lse, float* __restrict__ rest) {
  __shared__ float2 red[256];
  const int shares = 256 / tw, share = threadIdx.x / tw;
  const int t = blockIdx.x * tw + (threadIdx.x & (tw - 1));
  Part s = no_part();
  if (t < T) {
    int p = share;
    for (; p + 3 * shares < parts; p += 4 * shares) {   // four loads in flight
      float2 o[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) o[i] = part[(size_t)(p + i * shares) * T + t];
#pragma unroll
      for (int i = 0; i < 4; ++i) s = join(s, Part{o[i].x, o[i].y});
    }
    for (; p < parts; p += shares) {
      const float2 o = part[(size_t)p * T + t];
      s = join(s, Part{o.x, o.y});
    }
  }
  red[threadIdx.x] = make_float2(s.m, s.more);
  for (int n = 128; n >= tw; n >>= 1) {
    __syncthreads();
    if ((int)threadIdx.x < n) {
      const float2 o = red[threadIdx.x + n];
      s = join(s, Part{o.x, o.y});
      red[threadIdx.x] = make_float2(s.m, s.more);
    }
  }
  if ((int)threadIdx.x >= tw || t >= T) return;
  const bool none = s.more == -1.f;
  const float lz = log1pf(s.more);
  // log sum exp, rounded, and what the rounding left
  const float l = none ? -INFINITY : s.m + lz, d = l - s.m;
  lse[t] = l;
  rest[t] = none ? 0.f : (s.m - (l - d)) + (lz - d);
  const int64_t to = targets[t];
  float lp = 0.f;
  if (to >= V) lp = NAN;
  else if (to >= 0) lp = none ? -INFINITY : (target_logit[t] - s.m) - lz;
  logprob[t] = lp;
}

// ---- backward: dl of a piece ----
// One power of two for all tokens' gradients: scale[0], and its inverse in scale[1].  From the
// largest of their halves, whose differences stay in range; what is infinite or NaN is its own
// token's alone.
__global__ __launch_bounds__(1024) void linlog_scale_kernel(const int64_t* __restrict__ targets,
                                                           const float* __restrict__ dlp,
                                                           const float* __restrict__ dlse, int T,
                                                           float* __restrict__ scale) {
  __shared__ float red[16];
  float m = 0.f;
  for (int t = threadIdx.x; t < T; t += 1024) {
    const float g = targets[t] >= 0 ? 0.5f * dlp[t] : 0.f, h = dlse ? 0.5f * dlse[t] : 0.f;
    for (const float x : {fabsf(g), fabsf(h), fabsf(h - g)})
      if (x < INFINITY) m = fmaxf(m, x);
  }
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) m = fmaxf(m, __shfl_xor(m, off));
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = m;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int w = 1; w < 16; ++w) m = fmaxf(m, red[w]);
    const int e = (int)(__float_as_uint(m) >> 23) - 127;
    // (the scale and its inverse are both normal)
    const int by = m > 0.f ? min(13 - e, 126) : 0;
    scale[0] = ldexpf(1.f, by);
    scale[1] = ldexpf(1.f, -by);
  }
}

// What the backward pass takes of each token.
struct Tokens {
  const int64_t* targets;
  const float *logprob, *lse, *rest, *dlp, *dlse;
};
// dl at the target, g (1 - p) + h p, from its log probability.
__device__ __forceinline__ float at_target(float lt, float lse, float g, float h) {
  return lse == -INFINITY || (g == 0.f && h == 0.f) ? 0.f : fmaf(h, __expf(lt), -g * expm1f(lt));
}
// Token t's row of dl, scaled by `by`.
struct TokenGrad {
  int64_t to;
  float g, h, by_p, l, r;
  __device__ __forceinline__ TokenGrad(const Tokens& k, int t, int V, float by) {
    to = k.targets[t];
    g = to >= 0 ? k.dlp[t] * by : 0.f;
    h = k.dlse ? k.dlse[t] * by : 0.f;
    const bool none = k.lse[t] == -INFINITY;
    l = none ? 0.f : k.lse[t];
    r = -k.rest[t] * kLog2e;
    // (a target that is none of the vocabulary's: NaN, as its log probability)
    by_p = g == 0.f && h == 0.f ? 0.f : to >= V ? NAN : none ? 0.f : h - g;
  }
  // From a logit, beside the target; 0 is for the caller where by_p is: a token without a gradient
  // gives none, its logits NaN or not.
  __device__ __forceinline__ float other(float logit) const {
    return by_p * __builtin_amdgcn_exp2f(fmaf(logit - l, kLog2e, r));
  }
};
// What rounding to 16 bits leaves of it (scaled by `by`).  A token's target has most of its dl, so
// the products add this back, and both are off by 1.0 to 1.1 times what rounding them once is;
// without it by 1.4, and by up to 2.4 with a few tokens, whose roundings do not average.
template <int KIND>
__device__ __forceinline__ float target_rest(const Tokens& k, int t, float by) {
  const float h = k.dlse ? k.dlse[t] * by : 0.f;
  const float d = at_target(k.logprob[t], k.lse[t], k.dlp[t] * by, h);
  const float rest = d - from16<KIND>(to16<KIND>(d));
  return fabsf(rest) < INFINITY ? rest : 0.f;
}

// dl [T][ld] of rows v0 .. v0 + n of w (ld a multiple of 8; columns n .. n rounded up to 8 are zeros).
// Bound as the forward pass: 4096 tokens, 32768 x 4096 805 to 830 us, 1.32 to 1.37 PFLOP/s.
template <int KIND, int SP, int SQ, int WI, int WJ, int BI, int BJ>
__global__ __launch_bounds__(64 * WI * WJ) JARQ_WAVES(2) void linlog_dl_kernel(
    const void* __restrict__ X, const void* __restrict__ W, int T, int D, int V, int v0, int n,
    int ld, Tokens k, const float* __restrict__ scale, uint16_t* __restrict__ dl, int ni, int nj) {
  constexpr int TI = 16 * WI * BI, TJ = 16 * WJ * BJ, NW = WI * WJ;
  typedef PairContig<TI, NW> LP;
  typedef PairContig<TJ, NW> LQ;
  JARQ_SLOTS(SP, SQ, LP::kBytes, LQ::kBytes);
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wi = wave / WJ, wj = wave % WJ;
  int ti, tj;
  xcd_tile(blockIdx.x, ni, nj, ti, tj);
  const int c0 = ti * TI, t0 = tj * TJ;
  LP lp;
  LQ lq;
  lp.init((const char*)W + (size_t)v0 * 2 * D, 2 * (size_t)D, c0, n, 2 * D, wave, lane);
  lq.init(X, 2 * (size_t)D, t0, T, 2 * D, wave, lane);
  f32x4 acc[BI][BJ] = {};
  mma_pairs<SP, SQ, BI, BJ>(lp, lq, 0, (2 * D + kChunk - 1) / kChunk, lane, wi * 16 * BI,
                            wj * 16 * BJ, pslots, qslots,
                            [&](const u32x4& p, const u32x4& q, int a, int b)
                                __attribute__((always_inline)) {
                                  acc[a][b] = Mma<KIND>::mul(p, q, acc[a][b]);
                                });
  const float by = scale ? scale[0] : 1.f;
  const int cw = c0 + wi * 16 * BI + 4 * (lane >> 4);   // this lane's first column of dl
#pragma unroll
  for (int b = 0; b < BJ; ++b) {
    const int t = min(t0 + wj * 16 * BJ + 16 * b + (lane & 15), T - 1);
    const TokenGrad of(k, t, V, by);
#pragma unroll
    for (int a = 0; a < BI; ++a)
#pragma unroll
      for (int i = 0; i < 4; ++i) acc[a][b][i] = of.other(acc[a][b][i]);
    if (of.by_p == 0.f)
#pragma unroll
      for (int a = 0; a < BI; ++a) acc[a][b] = f32x4{};
    const int64_t at = of.to - v0 - cw;
    if (__any(at >= 0 && at < 16 * BI && at < n - cw)) {
      const float d = at_target(k.logprob[t], k.lse[t], of.g, of.h);
#pragma unroll
      for (int a = 0; a < BI; ++a)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (at == 16 * a + i) acc[a][b][i] = d;
    }
    if (c0 + TI > n)
#pragma unroll
      for (int a = 0; a < BI; ++a)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (cw + 16 * a + i >= n) acc[a][b][i] = 0.f;
  }
  char* const stage = wj == 0 ? pslot0 : wj == 1 ? pslot1 : wj == 2 ? qslot0 : qslot1;
  const int tw = t0 + wj * 16 * BJ;
  store_tile16<KIND, WI, BI, BJ>(acc, stage, wi, lane, [&](int t, int i, const u32x4& w) {
    if (tw + t < T && c0 + i < ld) *(u32x4*)(dl + (size_t)(tw + t) * ld + c0 + i) = w;
  });
}

// The same of few tokens, from the forward pass's sums.  Bound by reading w, as they are: one token,
// 128000 x 4096 217 us behind a gradient of w of the same size (in tiles 229), 8 x 32001 78 (90).
template <int KIND, int IB, int JB>
__global__ __launch_bounds__(512) void linlog_few_dl_kernel(
    const void* __restrict__ X, const void* __restrict__ W, int T, int D, int V, int v0, int n,
    int ld, Tokens k, const float* __restrict__ scale, uint16_t* __restrict__ dl) {
  constexpr int NW = 8;
  __shared__ __attribute__((aligned(16))) float red[NW * IB * JB * 256];
  const int c0 = blockIdx.x * (16 * JB);
  few_logits<KIND, IB, JB>(X, (const char*)W + (size_t)v0 * 2 * D, T, D, n, c0, red);
  const float by = scale ? scale[0] : 1.f;
  for (int e = threadIdx.x; e < IB * JB * 256; e += 512) {
    const int j = e & (16 * JB - 1), t = e / (16 * JB), c = c0 + j;
    if (t >= T) continue;
    const TokenGrad of(k, t, V, by);
    const float x = skinny_sum<NW, JB * IB>(red, JB * (t >> 4) + (j >> 4), t & 15, j & 15);
    float d = of.by_p == 0.f ? 0.f : of.other(x);
    if (of.to - v0 == c) d = at_target(k.logprob[t], k.lse[t], of.g, of.h);
    if (c < ld) dl[(size_t)t * ld + c] = to16<KIND>(c < n ? d : 0.f);
  }
}

// ---- backward: dx += dl w of a piece ----
// Rows v0 .. v0 + n of w.  part [splits][T][D] fp32: the sums so far of the share blockIdx.y of each
// piece's rows; the last piece's go to dX where there is one share.  Bound by the matrix cores: 4096
// tokens, 32768 x 4096 750 to 770 us, 1.45 PFLOP/s; with four by two wavefronts of 64 x 128 each, which
// take a fifth less of LDS, as long.
template <int KIND, int SP, int SQ, int WI, int WJ, int BI, int BJ>
__global__ __launch_bounds__(64 * WI * WJ) JARQ_WAVES(2) void linlog_dx_kernel(
    const void* __restrict__ dl, const void* __restrict__ W, int T, int D, int V, int v0, int n,
    int ld, int each, Tokens k, float* __restrict__ part, const float* __restrict__ scale,
    uint16_t* __restrict__ dX, int ni, int nj) {
  constexpr int TI = 16 * WI * BI, TJ = 16 * WJ * BJ, NW = WI * WJ;
  typedef PairStrided<TI, NW> LP;
  typedef PairContig<TJ, NW> LQ;
  JARQ_SLOTS(SP, SQ, LP::kBytes, LQ::kBytes);
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wi = wave / WJ, wj = wave % WJ;
  int ti, tj;
  xcd_tile(blockIdx.x, ni, nj, ti, tj);
  const int d0 = ti * TI, t0 = tj * TJ;
  LP lp;
  LQ lq;
  lp.init((const char*)W + (size_t)v0 * 2 * D, 2 * (size_t)D, d0, D, n, wave, lane);
  lq.init(dl, 2 * (size_t)ld, t0, T, 2 * ((n + 7) & ~7), wave, lane);
  f32x4 acc[BI][BJ] = {};
  const int nk = (2 * n + kChunk - 1) / kChunk;
  const int q0 = blockIdx.y * each, q1 = min(q0 + each, nk);
  if (q0 < q1)   // (a short last piece has no rows for the last shares)
    mma_pairs<SP, SQ, BI, BJ>(lp, lq, q0, q1, lane, wi * 16 * BI, wj * 16 * BJ, pslots, qslots,
                              [&](const u32x4& p, const u32x4& q, int a, int b)
                                  __attribute__((always_inline)) {
                                    acc[a][b] = Mma<KIND>::mul(p, q, acc[a][b]);
                                  });
  if (v0 + n == V && blockIdx.y == 0) {   // with the last piece, what the targets' roundings left
    float rest[BJ];
    int64_t v[BJ];
#pragma unroll
    for (int b = 0; b < BJ; ++b) {
      const int t = t0 + wj * 16 * BJ + 16 * b + (lane & 15);
      v[b] = t < T ? k.targets[t] : -1;
      if (v[b] >= V) v[b] = -1;
      rest[b] = v[b] >= 0 ? target_rest<KIND>(k, t, scale ? scale[0] : 1.f) : 0.f;
    }
#pragma unroll
    for (int a = 0; a < BI; ++a) {
      const int d = d0 + wi * 16 * BI + 16 * a + 4 * (lane >> 4);
#pragma unroll
      for (int b = 0; b < BJ; ++b) {
        u32x2 w{};
        if (v[b] >= 0 && d < D) w = *(const u32x2*)((const uint16_t*)W + (size_t)v[b] * D + d);
#pragma unroll
        for (int i = 0; i < 4; ++i)
          acc[a][b][i] = fmaf(rest[b], from16<KIND>((uint16_t)(w[i / 2] >> (16 * (i % 2)))),
                              acc[a][b][i]);
      }
    }
  }
  if (part) {   // uniform
#pragma unroll
    for (int b = 0; b < BJ; ++b) {
      const int t = t0 + wj * 16 * BJ + 16 * b + (lane & 15);
#pragma unroll
      for (int a = 0; a < BI; ++a) {
        const int d = d0 + wi * 16 * BI + 16 * a + 4 * (lane >> 4);
        if (t < T && d < D) {
          f32x4* const at = (f32x4*)(part + ((size_t)blockIdx.y * T + t) * D + d);
          if (v0 > 0) acc[a][b] += *at;
          if (!dX) *at = acc[a][b];
        }
      }
    }
    if (!dX) return;
  }
  const float by = scale ? scale[1] : 1.f;
#pragma unroll
  for (int a = 0; a < BI; ++a)
#pragma unroll
    for (int b = 0; b < BJ; ++b) acc[a][b] *= by;
  char* const stage = wj == 0 ? pslot0 : wj == 1 ? pslot1 : wj == 2 ? qslot0 : qslot1;
  const int tw = t0 + wj * 16 * BJ;
  store_tile16<KIND, WI, BI, BJ>(acc, stage, wi, lane, [&](int t, int i, const u32x4& w) {
    if (tw + t < T && d0 + i < D) *(u32x4*)(dX + (size_t)(tw + t) * D + d0 + i) = w;
  });
}

// The shares' sums in their order, rounded once.
template <int KIND>
__global__ __launch_bounds__(256) void linlog_dx_sum_kernel(const float* __restrict__ part,
                                                            int splits, size_t n,
                                                            const float* __restrict__ scale,
                                                            uint16_t* __restrict__ dX) {
  const float by = scale ? scale[1] : 1.f;
  for (size_t e = 4 * ((size_t)blockIdx.x * 256 + threadIdx.x); e < n;
       e += 4 * (size_t)gridDim.x * 256) {
    f32x4 s = *(const f32x4*)(part + e);
    for (int k = 1; k < splits; ++k) s += *(const f32x4*)(part + k * n + e);
    s *= by;
    *(u32x2*)(dX + e) = u32x2{pack16<KIND>(s[0], s[1]), pack16<KIND>(s[2], s[3])};
  }
}

// ---- backward: dw = dl^T x of a piece ----
// Bound by the matrix cores and the transposing reads of LDS, which take twice as long as plain ones:
// 4096 tokens, 32768 x 4096 840 to 870 us, 1.28 PFLOP/s.  With x transposed beforehand, so that plain
// reads do for eight fragments of twelve, 1 % less.
template <int KIND, int SP, int SQ, int WI, int WJ, int BI, int BJ>
__global__ __launch_bounds__(64 * WI * WJ) JARQ_WAVES(2) void linlog_dw_kernel(
    const void* __restrict__ dl, const void* __restrict__ X, int T, int D, int v0, int n, int ld,
    Tokens k, const float* __restrict__ scale, uint16_t* __restrict__ dW, int ni, int nj) {
  constexpr int TI = 16 * WI * BI, TJ = 16 * WJ * BJ, NW = WI * WJ;
  typedef PairStrided<TI, NW> LP;
  typedef PairStrided<TJ, NW> LQ;
  JARQ_SLOTS(SP, SQ, LP::kBytes, LQ::kBytes);
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wi = wave / WJ, wj = wave % WJ;
  int ti, tj;
  xcd_tile(blockIdx.x, ni, nj, ti, tj);
  const int d0 = ti * TI, c0 = tj * TJ;
  LP lp;
  LQ lq;
  lp.init(X, 2 * (size_t)D, d0, D, T, wave, lane);
  lq.init(dl, 2 * (size_t)ld, c0, (n + 7) & ~7, T, wave, lane);
  const int64_t ahead = k.targets[min(lane, T - 1)];
  f32x4 acc[BI][BJ] = {};
  mma_pairs<SP, SQ, BI, BJ>(lp, lq, 0, (2 * T + kChunk - 1) / kChunk, lane, wi * 16 * BI,
                            wj * 16 * BJ, pslots, qslots,
                            [&](const u32x4& p, const u32x4& q, int a, int b)
                                __attribute__((always_inline)) {
                                  acc[a][b] = Mma<KIND>::mul(p, q, acc[a][b]);
                                });
  // What the roundings of dl at this tile's targets left, as further products: 64 tokens at a time,
  // their rows of x and a row each that has its token's rest (in 16 bits) at its target and zeros.
  // Bound by latency: 2.5 us a tile with a target or two, 5.5 for each 64 (611 tokens, 50257 x 1000
  // 80 -> 95 us; 4096 tokens, 32768 x 4096 690 -> 730).  Looked up before the products above, the
  // targets take registers from them (twice the cost).
  static_assert(SP == 3 && LP::kBytes % 2048 == 0, "the list of tokens has a slot of its own");
  constexpr int kListed = LP::kBytes / 8, IT = kListed / (64 * NW), PC = TI / 8, QC = TJ / 8;
  static_assert(IT * 64 * NW == kListed && PC % NW == 0 && QC % NW == 0, "shares of a wave");
  uint32_t* const list = (uint32_t*)pslot2;               // a token's place and its row of w in the tile
  int* const counts = (int*)(pslot2 + 4 * kListed);
  const typename LP::template Lane<BI> pl(wi * 16 * BI, lane);
  const typename LQ::template Lane<BJ> ql(wj * 16 * BJ, lane);
  // (up to 64 tokens a wave knows by itself whether the tile has any, without a wait)
  const int end = T > 64 || __any(ahead - v0 - c0 >= 0 && ahead - v0 - c0 < min(TJ, n - c0)) ? T : 0;
  for (int t0 = 0; t0 < end; t0 += kListed) {
    if (t0 > 0) __syncthreads();   // (the last list is read)
    int at[IT], mine;
#pragma unroll
    for (int i = 0; i < IT; ++i) {
      const int t = t0 + 64 * (wave * IT + i) + lane;
      const int64_t v = k.targets[min(t, T - 1)] - v0 - c0;   // (no branch: all loads at once)
      at[i] = t < T && v >= 0 && v < min(TJ, n - c0) ? (int)v : -1;
    }
    int begin[NW], listed;
    for (bool all = true;; all = false) {
      mine = 0;
#pragma unroll
      for (int i = 0; i < IT; ++i) {   // each wave's from a place of its own on
        const uint64_t found = __ballot(at[i] >= 0);
        if (at[i] >= 0)
          list[64 * IT * wave + mine + __popcll(found & (((uint64_t)1 << lane) - 1))] =
              (uint32_t)(64 * (wave * IT + i) + lane) << 8 | (uint32_t)at[i];
        mine += __popcll(found);
      }
      if (lane == 0) counts[wave] = mine;
      __syncthreads();
      listed = 0;
#pragma unroll
      for (int w = 0; w < NW; ++w) {
        begin[w] = listed;
        listed += counts[w];
      }
      if (!all || listed <= 64) break;   // uniform
      // many: masked tokens may share a target, and those without a gradient have no rest
#pragma unroll
      for (int i = 0; i < IT; ++i) {
        const int t = min(t0 + 64 * (wave * IT + i) + lane, T - 1);
        if (k.dlp[t] == 0.f && (!k.dlse || k.dlse[t] == 0.f)) at[i] = -1;
      }
      __syncthreads();   // (the counts are read)
    }
    auto entry = [&](int e) __attribute__((always_inline)) {
      int place = e;
#pragma unroll
      for (int w = 1; w < NW; ++w) place = e >= begin[w] ? 64 * IT * w + e - begin[w] : place;
      return list[place];
    };
    for (int first = 0; first < listed; first += 64) {
      const int rows = min(listed - first, 64), halves = rows > 32 ? 2 : 1;
      u32x4 w[PC / NW];
#pragma unroll
      for (int i = 0; i < PC / NW; ++i) {   // (no branch here either; what is past the last row is not kept)
        const int e = threadIdx.x + 64 * NW * i, r = e / PC, d = d0 + 8 * LP::piece(r, e % PC);
        const int t = t0 + (int)(entry(first + min(r, rows - 1)) >> 8);
        w[i] = *(const u32x4*)((const uint16_t*)X + (size_t)t * D + min(d, D - 8));
      }
      float rest = 0.f;
      uint32_t one = 0;
      if ((int)threadIdx.x < rows) {
        one = entry(first + threadIdx.x);
        rest = target_rest<KIND>(k, t0 + (int)(one >> 8), scale ? scale[0] : 1.f);
      }
#pragma unroll
      for (int i = 0; i < QC / NW; ++i) *(u32x4*)(qslot0 + 16 * (threadIdx.x + 64 * NW * i)) = u32x4{};
#pragma unroll
      for (int i = 0; i < PC / NW; ++i) {
        const int e = threadIdx.x + 64 * NW * i;
        *(u32x4*)(pslot0 + 16 * e) = e / PC < rows ? w[i] : u32x4{};
      }
      __syncthreads();
      if ((int)threadIdx.x < rows) {
        const int r = threadIdx.x, v = (int)(one & 255);
        *(uint16_t*)(qslot0 + 2 * (r * TJ + 8 * LQ::piece(r, v / 8) + v % 8)) = to16<KIND>(rest);
      }
      __syncthreads();
      for (int half = 0; half < halves; ++half) {
        u32x4 q[BJ];
#pragma unroll
        for (int b = 0; b < BJ; ++b) q[b] = ql.frag(qslot0, half, b);
#pragma unroll
        for (int a = 0; a < BI; ++a) {
          const u32x4 p = pl.frag(pslot0, half, a);
#pragma unroll
          for (int b = 0; b < BJ; ++b) acc[a][b] = Mma<KIND>::mul(p, q[b], acc[a][b]);
        }
      }
      __syncthreads();
    }
  }
  const float by = scale ? scale[1] : 1.f;
#pragma unroll
  for (int a = 0; a < BI; ++a)
#pragma unroll
    for (int b = 0; b < BJ; ++b) acc[a][b] *= by;
  char* const stage = wj == 0 ? pslot0 : wj == 1 ? pslot1 : wj == 2 ? qslot0 : qslot1;
  const int cw = c0 + wj * 16 * BJ;
  store_tile16<KIND, WI, BI, BJ>(acc, stage, wi, lane, [&](int r, int i, const u32x4& w) {
    if (cw + r < n && d0 + i < D) *(u32x4*)(dW + (size_t)(cw + r) * D + d0 + i) = w;
  });
}

__global__ __launch_bounds__(256) void linlog_zero_kernel(u32x4* out, size_t n) {
  for (size_t e = (size_t)blockIdx.x * 256 + threadIdx.x; e < n; e += (size_t)gridDim.x * 256)
    out[e] = u32x4{};
}

namespace {

constexpr int kTokensAtOnce = 16384;   // of the forward pass: bounds its parts

// Tiles of l = x w^T by rows of w and tokens, the ones that cost the least.  In us with tiles of 256 x
// 256 (rows x tokens), 128 x 128, 128 x 64 and 64 x 64 (the rule is 1.8 % off the best over 84 sizes):
//   d 1000   200 x  5003     25  12   9  10     611 x 50257   83  78 111 135
//   d 4096   200 x 17000     75  49  61  58    2047 x 50257  656 730 1054 1302
constexpr int kWide[4] = {256, 128, 128, 64}, kTall[4] = {256, 128, 64, 64};
int logit_tiles(int T, int D, int n) {
  constexpr TileTime time[4] = {{9.6, 0.54, 4.7, 0.72},
                                {5.4, 0.225, 1.3, 0.225},
                                {3.5, 0.18, 0.6, 0.17},
                                {3.7, 0.137, 0.5, 0.10}};
  const int nk = (2 * D + kChunk - 1) / kChunk;
  int best = 0;
  double least = 0.0;
  for (int k = 0; k < 4; ++k) {
    const long long tiles = (long long)((n + kWide[k] - 1) / kWide[k]) * ((T + kTall[k] - 1) / kTall[k]);
    const double cost = tile_cost(tiles, nk, time[k]);
    if (k == 0 || cost < least) {
      best = k;
      least = cost;
    }
  }
  return best;
}
// Rows of w a work-group where fragments come straight from memory, 0: tiles.  In us with 16
// rows, 32, and in tiles, the weights from memory (several copies in turn):
//    d 4096    1 token  x 16000 28 34 40      x 128000 172 197 176
//              8 tokens x  5003 19 17 36      x  32001  59  61  64     x 128000 223 212 180
//             24        x  5003 28 21 36      x  16000  54  46  42     x  32001 102  85  65
//    d  512    4        x 16000 14 14 14      x  32001  19  14  14     x 128000  56  41  33
// The rule looks at tokens and vocabulary alone: 3 % off the best over 175 sizes in the mean, up to
// 17 % from 4096 channels on, and up to 1.7 times with few channels and a large vocabulary (the last
// row).  With the weights in the last cache tiles gain up to a third.
int few_rows(int T, int V) {
  if (T > 32) return 0;
  if (T <= 4 || V <= 4096) return 16;
  return V <= (T <= 16 ? 32768 : 8192) ? 32 : 0;
}
// Parts a token of n that the forward pass takes at once, of T.
int forward_parts(int T, int n, int D, int V) {
  if (const int rows = few_rows(T, V)) return (V + rows - 1) / rows;
  const int k = logit_tiles(n, D, V);
  return (V + kWide[k] - 1) / kWide[k];
}

// Rows of w a piece: 256 MiB of dl (at least 1024 rows).  Its stride, up to 64 values longer, adds 128
// bytes a token: 272 MiB at 2^17 tokens.
int piece_rows(int T, int V) {
  const int64_t most = std::max<int64_t>(1024, ((int64_t)1 << 27) / std::max(T, 1) / 1024 * 1024);
  return (int)std::min<int64_t>(most, V);
}

// Tiles of dw by channels and rows of w: 256 x 256, 128 x 128, 128 x 64.  d 1000, 200 tokens x 5003
// 12, 8.9, 9.5 us; 611 x 50257 83, 77, 103; d 4096, 611 x 17000 104, 96, 128.
int dw_tiles(int T, int D, int n) {
  constexpr int wide[3] = {256, 128, 128}, tall[3] = {256, 128, 64};
  constexpr TileTime time[3] = {{7.2, 0.62, 7.6, 0.71}, {4.2, 0.254, 1.8, 0.2}, {3.2, 0.195, 1.2, 0.14}};
  const int nk = (2 * T + kChunk - 1) / kChunk;
  int best = 0;
  double least = 0.0;
  for (int k = 0; k < 3; ++k) {
    const long long tiles = (long long)((D + wide[k] - 1) / wide[k]) * ((n + tall[k] - 1) / tall[k]);
    const double cost = tile_cost(tiles, nk, time[k]);
    if (k == 0 || cost < least) {
      best = k;
      least = cost;
    }
  }
  return best;
}

// Tiles and shares of dx, the ones that cost the least; each further share adds its sums' way through
// memory and the launch that joins them.  dl and dx in us by tiles (channels x tokens) / shares:
//    8 x 32001, d 4096       128 x 64 / 8   97     128 x 128 / 8  99    256 x 256 / 16 111
//    200 x 5003, d 1000      128 x 64 / 8   28     128 x 128 / 8  31    256 x 256 /  8  43
//    611 x 50257, d 1000     128 x 128 / 6 187     256 x 256 / 12 185   128 x  64 /  6 205
//    2047 x 32001, d 4096    256 x 256 / 2 833     / 4 860   / 3 899    128 x 128 /  1 932
// 1.7 % off the best of ten sizes in the mean; the most, 6 %, at 611 x 17000, d 4096 (191, 180).
struct DxPlan {
  int kind;   // tiles of 256 x 256 (channels x tokens), 128 x 128, 128 x 64
  int ni, nj, splits, each;
};
DxPlan dx_plan(int T, int D, int rows) {
  const int nk = (2 * rows + kChunk - 1) / kChunk;
  constexpr int wide[3] = {256, 128, 128}, tall[3] = {256, 128, 64};
  constexpr TileTime time[3] = {
      {8.0, 0.62, 8.0, 0.62}, {4.0, 0.26, 4.0, 0.26}, {3.0, 0.19, 3.0, 0.19}};
  DxPlan best{};
  double least = 0.0;
  for (int kind = 0; kind < 3; ++kind) {
    const int ni = (D + wide[kind] - 1) / wide[kind], nj = (T + tall[kind] - 1) / tall[kind];
    for (int parts = 1; parts <= 32; ++parts) {
      const int each = ((nk + parts - 1) / parts + 3) / 4 * 4;   // whole pairs of chunks, two and two
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
// Values a row of dl: an odd number of cache lines (rows a power of two apart share a channel).
int dl_stride(int rows) { return ((rows + 63) / 64 | 1) * 64; }

}  // namespace

size_t linear_logprobs_workspace_bytes(int T, int D, int V) {
  const int most = std::min(T, kTokensAtOnce);
  // (a shorter last share of the tokens may take smaller tiles)
  size_t parts = (size_t)forward_parts(T, most, D, V) * most;
  if (const int last = T % kTokensAtOnce; T > kTokensAtOnce && last)
    parts = std::max(parts, (size_t)forward_parts(T, last, D, V) * last);
  return pad256(4 * (size_t)most) + 8 * parts;
}

template <int KIND, int SP, int SQ, int WI, int WJ, int BI, int BJ>
static void linlog_tiles(hipStream_t st, int T, int D, int V, const void* X, const void* W,
                         const int64_t* targets, float* logit, float2* part) {
  const int ni = (V + 16 * WI * BI - 1) / (16 * WI * BI);
  const int nj = (T + 16 * WJ * BJ - 1) / (16 * WJ * BJ);
  hipLaunchKernelGGL((linlog_tile_kernel<KIND, SP, SQ, WI, WJ, BI, BJ>), dim3((unsigned)(ni * nj)),
                     dim3(64 * WI * WJ), 0, st, X, W, T, D, V, targets, logit, part, ni, nj);
}

template <int KIND>
static hipError_t launch_linlog_kind(hipStream_t st, int T, int D, int V, const void* X,
                                     const void* W, const int64_t* targets, float* logprob,
                                     float* lse, float* rest, char* ws) {
  float* logit = (float*)ws;
  float2* part = (float2*)(ws + pad256(4 * (size_t)std::min(T, kTokensAtOnce)));
  for (int t0 = 0; t0 < T; t0 += kTokensAtOnce) {
    const int n = std::min(T - t0, kTokensAtOnce);
    const void* x = (const char*)X + (size_t)t0 * 2 * D;
    const int64_t* to = targets + t0;
    const int parts = forward_parts(T, n, D, V);
    if (const int rows = few_rows(T, V)) {   // (not a last share alone: the backward pass's rule)
#define JARQ_LINLOG_FEW(IB, JB)                                                                 \
  hipLaunchKernelGGL((linlog_skinny_kernel<KIND, IB, JB>), dim3(parts), dim3(512), 0, st, x, W, \
                     n, D, V, to, logit, part)
      if (n <= 16 && rows == 16) JARQ_LINLOG_FEW(1, 1);
      else if (n <= 16) JARQ_LINLOG_FEW(1, 2);
      else if (rows == 16) JARQ_LINLOG_FEW(2, 1);
      else JARQ_LINLOG_FEW(2, 2);
#undef JARQ_LINLOG_FEW
    } else {
      switch (logit_tiles(n, D, V)) {
        case 0: linlog_tiles<KIND, 3, 2, 2, 4, 8, 4>(st, n, D, V, x, W, to, logit, part); break;
        case 1: linlog_tiles<KIND, 3, 2, 2, 2, 4, 4>(st, n, D, V, x, W, to, logit, part); break;
        case 2: linlog_tiles<KIND, 3, 2, 2, 2, 4, 2>(st, n, D, V, x, W, to, logit, part); break;
        default: linlog_tiles<KIND, 3, 3, 1, 2, 4, 2>(st, n, D, V, x, W, to, logit, part);
      }
    }
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    int tw = 1;
    while (tw < 16 && tw < n) tw *= 2;
    hipLaunchKernelGGL(linlog_join_kernel, dim3((n + tw - 1) / tw), dim3(256), 0, st, part, parts,
                       n, V, tw, to, logit, logprob + t0, lse + t0, rest + t0);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }
  return hipSuccess;
}

hipError_t launch_linear_logprobs(hipStream_t st, int dtype, int T, int D, int V, const void* X,
                                  const void* W, const int64_t* targets, float* logprob,
                                  float* lse, float* rest, char* ws) {
  return dtype == kBF16
             ? launch_linlog_kind<kBF16>(st, T, D, V, X, W, targets, logprob, lse, rest, ws)
             : launch_linlog_kind<kF16>(st, T, D, V, X, W, targets, logprob, lse, rest, ws);
}

size_t linear_logprobs_backward_workspace_bytes(int T, int D, int V) {
  const int rows = piece_rows(T, V);
  const DxPlan p = dx_plan(T, D, rows);
  size_t n = 256 + pad256(2 * (size_t)T * dl_stride(rows));
  if (p.splits > 1 || rows < V) n += 4 * (size_t)p.splits * T * D;
  return n;
}

template <int KIND, int SP, int SQ, int WI, int WJ, int BI, int BJ>
static void linlog_dl(hipStream_t st, int T, int D, int V, int v0, int n, int ld, const void* X,
                      const void* W, const Tokens& k, const float* scale, uint16_t* dl) {
  const int ni = (n + 16 * WI * BI - 1) / (16 * WI * BI);
  const int nj = (T + 16 * WJ * BJ - 1) / (16 * WJ * BJ);
  hipLaunchKernelGGL((linlog_dl_kernel<KIND, SP, SQ, WI, WJ, BI, BJ>), dim3((unsigned)(ni * nj)),
                     dim3(64 * WI * WJ), 0, st, X, W, T, D, V, v0, n, ld, k, scale, dl, ni,
                     nj);
}

template <int KIND>
static hipError_t launch_linlog_backward_kind(hipStream_t st, int T, int D, int V, const void* X,
                                              const void* W, const int64_t* targets,
                                              const float* logprob, const float* lse,
                                              const float* rest, const float* dlp,
                                              const float* dlse, void* dX, void* dW, char* ws) {
  if (T == 0) {
    if (!dW) return hipSuccess;
    hipLaunchKernelGGL(linlog_zero_kernel, dim3(1024), dim3(256), 0, st, (u32x4*)dW,
                       (size_t)V * D / 8);
    return hipGetLastError();
  }
  if (!dX && !dW) return hipSuccess;
  const int rows = piece_rows(T, V), ld = dl_stride(rows);
  const DxPlan p = dx_plan(T, D, rows);
  float* scale = KIND == kF16 ? (float*)ws : nullptr;   // bf16 has fp32's range
  uint16_t* dl = (uint16_t*)(ws + 256);
  const Tokens tokens{targets, logprob, lse, rest, dlp, dlse};
  float* part = p.splits > 1 || rows < V ? (float*)(ws + 256 + pad256(2 * (size_t)T * ld)) : nullptr;
  if (scale) {
    hipLaunchKernelGGL(linlog_scale_kernel, dim3(1), dim3(1024), 0, st, targets, dlp, dlse, T,
                       scale);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  for (int v0 = 0; v0 < V; v0 += rows) {
    const int n = std::min(rows, V - v0);
#define JARQ_LINLOG_DL(...) \
  linlog_dl<KIND, __VA_ARGS__>(st, T, D, V, v0, n, ld, X, W, tokens, scale, dl)
#define JARQ_LINLOG_FEW(IB, JB)                                                              \
  hipLaunchKernelGGL((linlog_few_dl_kernel<KIND, IB, JB>), dim3((n + few - 1) / few), dim3(512), 0, \
                     st, X, W, T, D, V, v0, n, ld, tokens, scale, dl)
    if (const int few = few_rows(T, V)) {   // the forward pass's rule
      if (T <= 16 && few == 16) JARQ_LINLOG_FEW(1, 1);
      else if (T <= 16) JARQ_LINLOG_FEW(1, 2);
      else if (few == 16) JARQ_LINLOG_FEW(2, 1);
      else JARQ_LINLOG_FEW(2, 2);
    } else {
      switch (logit_tiles(T, D, n)) {
        case 0: JARQ_LINLOG_DL(3, 2, 2, 4, 8, 4); break;
        case 1: JARQ_LINLOG_DL(3, 2, 2, 2, 4, 4); break;
        case 2: JARQ_LINLOG_DL(3, 2, 2, 2, 4, 2); break;
        default: JARQ_LINLOG_DL(3, 3, 1, 2, 4, 2);
      }
    }
#undef JARQ_LINLOG_FEW
#undef JARQ_LINLOG_DL
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    if (dX) {
      const dim3 grid((unsigned)(p.ni * p.nj), (unsigned)p.splits);
      const bool last = v0 + n == V;
      uint16_t* out = p.splits == 1 && last ? (uint16_t*)dX : nullptr;
      if (p.kind == 0)
        hipLaunchKernelGGL((linlog_dx_kernel<KIND, 3, 2, 2, 4, 8, 4>), grid, dim3(512), 0, st, dl,
                           W, T, D, V, v0, n, ld, p.each, tokens, part, scale, out, p.ni, p.nj);
      else if (p.kind == 1)
        hipLaunchKernelGGL((linlog_dx_kernel<KIND, 3, 2, 2, 2, 4, 4>), grid, dim3(256), 0, st, dl,
                           W, T, D, V, v0, n, ld, p.each, tokens, part, scale, out, p.ni, p.nj);
      else
        hipLaunchKernelGGL((linlog_dx_kernel<KIND, 3, 2, 2, 2, 4, 2>), grid, dim3(256), 0, st, dl,
                           W, T, D, V, v0, n, ld, p.each, tokens, part, scale, out, p.ni, p.nj);
      if ((e = hipGetLastError()) != hipSuccess) return e;
      if (last && p.splits > 1) {
        const size_t all = (size_t)T * D, b = (all / 4 + 255) / 256;
        hipLaunchKernelGGL((linlog_dx_sum_kernel<KIND>), dim3((unsigned)std::min<size_t>(b, 4096)),
                           dim3(256), 0, st, part, p.splits, all, scale, (uint16_t*)dX);
        if ((e = hipGetLastError()) != hipSuccess) return e;
      }
    }
    if (dW) {
      uint16_t* out = (uint16_t*)dW + (size_t)v0 * D;
      const int k = dw_tiles(T, D, n), wide = k == 0 ? 256 : 128, tall = k == 0 ? 256 : k == 1 ? 128 : 64;
      const int ni = (D + wide - 1) / wide, nj = (n + tall - 1) / tall;
      const dim3 grid((unsigned)(ni * nj));
      if (k == 0)
        hipLaunchKernelGGL((linlog_dw_kernel<KIND, 3, 2, 2, 4, 8, 4>), grid, dim3(512), 0, st, dl,
                           X, T, D, v0, n, ld, tokens, scale, out, ni, nj);
      else if (k == 1)
        hipLaunchKernelGGL((linlog_dw_kernel<KIND, 3, 2, 2, 2, 4, 4>), grid, dim3(256), 0, st, dl,
                           X, T, D, v0, n, ld, tokens, scale, out, ni, nj);
      else
        hipLaunchKernelGGL((linlog_dw_kernel<KIND, 3, 2, 2, 2, 4, 2>), grid, dim3(256), 0, st, dl,
                           X, T, D, v0, n, ld, tokens, scale, out, ni, nj);
      if ((e = hipGetLastError()) != hipSuccess) return e;
    }
  }
  return hipSuccess;
}

hipError_t launch_linear_logprobs_backward(hipStream_t st, int dtype, int T, int D, int V,
                                           const void* X, const void* W, const int64_t* targets,
                                           const float* logprob, const float* lse,
                                           const float* rest, const float* dlp,
                                           const float* dlse, void* dX, void* dW, char* ws) {
  return dtype == kBF16 ? launch_linlog_backward_kind<kBF16>(st, T, D, V, X, W, targets, logprob,
                                                             lse, rest, dlp, dlse, dX, dW, ws)
                        : launch_linlog_backward_kind<kF16>(st, T, D, V, X, W, targets, logprob,
                                                            lse, rest, dlp, dlse, dX, dW, ws);
}

}  // namespace jarq
