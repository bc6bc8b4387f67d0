// Linear layers in 8-bit integers.
//
// quant_rows_kernel: a row's values on a symmetric grid of its own, scale = amax /
// 127, q = rint(x (127 / amax)), all in fp32.
//
// The product: y[t][n] = sx_t sum_g sw[n][g] sum_{k in g} xq[t][k] wq[n][k], the
// integer sums exact in int32 on v_mfma_i32_16x16x64_i8, a group's sum converted
// and added in fp32.  Tokens are the P rows and channels the Q rows, so that a lane
// holds one channel and needs one group scale.
#include <type_traits>

#include "skinny.h"

namespace jarq {

namespace {

constexpr uint32_t kInfBits = 0x7f800000u;
constexpr uint32_t kTinyBits = 0x0d800000u;   // 2^-100

// |x| as ordered bits: NaN above infinity above every finite value
__device__ __forceinline__ uint32_t abs_bits(float x) { return __float_as_uint(x) & 0x7fffffffu; }

// A row's scale and multiplier.  Rows under 2^-100 are zeros (their multiplier
// would overflow); a row with an infinity or a NaN has a NaN scale and zeros, so that
// what is computed from it is NaN.
__device__ __forceinline__ void row_scale(uint32_t amax_bits, float& scale, float& mul) {
  const float amax = __uint_as_float(amax_bits);
  mul = 0.f;
  if (amax_bits >= kInfBits) {
    scale = __uint_as_float(0x7fc00000u);
  } else if (amax_bits < kTinyBits) {
    scale = 0.f;
  } else {
    scale = amax / 127.f;
    mul = 127.f / amax;
  }
}
__device__ __forceinline__ uint32_t quant(float x, float mul) {
  // a zero multiplier gives 0 for any x
  return mul == 0.f ? 0u : (uint32_t)(int)rintf(x * mul) & 0xffu;
}

__device__ __forceinline__ u32x2 quant8(const float (&x)[8], float mul) {
  uint32_t lo = 0, hi = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    lo |= quant(x[i], mul) << (8 * i);
    hi |= quant(x[4 + i], mul) << (8 * i);
  }
  return u32x2{lo, hi};
}

// Eight values from element 8 v of a row, as they are stored.
template <int DT> struct Piece { u32x4 w[DT == 0 ? 2 : 1]; };
template <int DT>
__device__ __forceinline__ Piece<DT> load_piece(const void* row, int v) {
  Piece<DT> p;
#pragma unroll
  for (int i = 0; i < (DT == 0 ? 2 : 1); ++i)
    p.w[i] = *((const u32x4*)row + (DT == 0 ? 2 : 1) * v + i);
  return p;
}
template <int DT>
__device__ __forceinline__ void unpack8(const Piece<DT>& p, float (&x)[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (DT == 0) {
      x[i] = __uint_as_float(p.w[0][i]);
      x[4 + i] = __uint_as_float(p.w[DT == 0 ? 1 : 0][i]);
    } else {
      x[2 * i] = from16<DT>((uint16_t)p.w[0][i]);
      x[2 * i + 1] = from16<DT>((uint16_t)(p.w[0][i] >> 16));
    }
  }
}

}  // namespace

// A work-group a row; K a multiple of 16.  A row of up to 16384 values stays in registers
// between its maximum and its integers: 8192 rows of 14336 in bf16 57 us, read
// twice 88 (352 MB: 69 at the rate of a copy).
template <int DT>
__global__ __launch_bounds__(256) void quant_rows_kernel(const void* __restrict__ X, int K,
                                                         int8_t* __restrict__ Q,
                                                         float* __restrict__ scale) {
  constexpr int R = 8;   // pieces of eight values a thread holds
  __shared__ uint32_t red[4];
  const int tid = threadIdx.x;
  const size_t r = blockIdx.x;
  const char* row = (const char*)X + r * K * (DT == 0 ? 4 : 2);
  const int nv = K / 8;
  Piece<DT> p[R];
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < R; ++i)
    p[i] = tid + 256 * i < nv ? load_piece<DT>(row, tid + 256 * i) : Piece<DT>{};
  auto most = [&](const Piece<DT>& w) __attribute__((always_inline)) {
    float x[8];
    unpack8<DT>(w, x);
#pragma unroll
    for (int i = 0; i < 8; ++i) m = max(m, abs_bits(x[i]));
  };
#pragma unroll
  for (int i = 0; i < R; ++i) most(p[i]);
  for (int v = tid + 256 * R; v < nv; v += 256) most(load_piece<DT>(row, v));
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) m = max(m, (uint32_t)__shfl_xor((int)m, off));
  if ((tid & 63) == 0) red[tid >> 6] = m;
  __syncthreads();
  m = max(max(red[0], red[1]), max(red[2], red[3]));
  float s, mul;
  row_scale(m, s, mul);
  auto put = [&](int v, const Piece<DT>& w) __attribute__((always_inline)) {
    float x[8];
    unpack8<DT>(w, x);
    *(u32x2*)(Q + r * K + 8 * (size_t)v) = quant8(x, mul);
  };
#pragma unroll
  for (int i = 0; i < R; ++i)
    if (tid + 256 * i < nv) put(tid + 256 * i, p[i]);
  for (int v = tid + 256 * R; v < nv; v += 256) put(v, load_piece<DT>(row, v));
  if (tid == 0) scale[r] = s;
}

hipError_t launch_quant_rows(hipStream_t st, int dtype, const void* X, int rows, int K, int8_t* Q,
                             float* scale) {
  const dim3 g(rows), b(256);
  if (dtype == 0) hipLaunchKernelGGL(quant_rows_kernel<0>, g, b, 0, st, X, K, Q, scale);
  else if (dtype == 1) hipLaunchKernelGGL(quant_rows_kernel<1>, g, b, 0, st, X, K, Q, scale);
  else hipLaunchKernelGGL(quant_rows_kernel<2>, g, b, 0, st, X, K, Q, scale);
  return hipGetLastError();
}

// ---- codes minus zero points as int8 ----
// Sixteen codes a thread (within a group); bad is set by a value outside int8.  Bound by
// memory: 14336 x 4096 19 us, 6 TB/s (in part from the last-level cache).
__global__ __launch_bounds__(256) void codes_i8_kernel(const uint8_t* __restrict__ codes,
                                                       const int32_t* __restrict__ zeros,
                                                       long long n16, int g,
                                                       int8_t* __restrict__ out,
                                                       int32_t* __restrict__ bad) {
  const long long e = (long long)blockIdx.x * 256 + threadIdx.x;
  if (e >= n16) return;
  const u32x4 q = *((const u32x4*)codes + e);
  // (held where q - z cannot overflow; beyond that it is out of range anyway)
  const int z = max(-1024, min(1024, zeros[16 * e / g]));
  u32x4 o;
  bool out_of_range = false;
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    uint32_t p = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int c = (int)((q[w] >> (8 * i)) & 0xffu) - z;
      out_of_range |= c < -128 || c > 127;
      p |= ((uint32_t)c & 0xffu) << (8 * i);
    }
    o[w] = p;
  }
  *((u32x4*)out + e) = o;
  if (out_of_range) *bad = 1;
}
__global__ void clear_flag_kernel(int32_t* flag) { *flag = 0; }

hipError_t launch_codes_i8(hipStream_t st, const uint8_t* codes, const int32_t* zeros, int rows,
                           int cols, int g, int8_t* out, int32_t* bad) {
  hipLaunchKernelGGL(clear_flag_kernel, dim3(1), dim3(1), 0, st, bad);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const long long n16 = (long long)rows * cols / 16;
  hipLaunchKernelGGL(codes_i8_kernel, dim3((unsigned)((n16 + 255) / 256)), dim3(256), 0, st, codes,
                     zeros, n16, g, out, bad);
  return hipGetLastError();
}

// ---- products ----
namespace {

__device__ __forceinline__ void store_y(void* Y, int dtype, size_t at, float y) {   // dtype uniform
  if (dtype == 0) ((float*)Y)[at] = y;
  else if (dtype == 1) ((uint16_t*)Y)[at] = to16<kF16>(y);
  else ((uint16_t*)Y)[at] = to16<kBF16>(y);
}

}  // namespace

// Many tokens.  GROUP 0: one scale a channel, int32 sums over all of k, bound by the
// matrix cores at the clock that the card's power allows (8192 x 14336 -> 4096 375 to 400 us,
// 2.4 POP/s and more).  Otherwise a group's int32 sums go to fp32: converting one and adding
// it takes two vector instructions, eight to a matrix instruction of half their time, beside
// LDS reads of as much (2048 x 11008 -> 4096, groups of 64, 163 to 178 us, 1.0 to 1.1 POP/s).
template <int GROUP, int S, int WI, int WJ, int BI, int BJ>
__global__ __launch_bounds__(64 * WI * WJ) JARQ_WAVES(GROUP && WI * WJ == 8 ? 4 : 2) void i8_tile_kernel(
    const int8_t* __restrict__ Xq, const float* __restrict__ sx, const int8_t* __restrict__ Wq,
    const float* __restrict__ sw, int T, int N, int K, int dtype, void* __restrict__ Y, int ni,
    int nj) {
  constexpr int TI = 16 * WI * BI, TJ = 16 * WJ * BJ, NW = WI * WJ;
  typedef KContig<TI, NW, kOne> LP;
  typedef KContig<TJ, NW, kOne> LQ;
  constexpr int STAGE = LP::kBytes + LQ::kBytes;
  JARQ_STAGES(S, STAGE);
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wi = wave / WJ, wj = wave % WJ;
  int ti, tj;
  xcd_tile(blockIdx.x, ni, nj, ti, tj);
  const int t0 = ti * TI, n0 = tj * TJ;
  LP lp;
  LQ lq;
  lp.init(Xq, Xq, K, t0, T, K, wave, lane);
  lq.init(Wq, Wq, K, n0, N, K, wave, lane);
  const int nk = (K + kChunk - 1) / kChunk, prow = wi * 16 * BI, qrow = wj * 16 * BJ;
  f32x4 y[GROUP ? BI : 1][GROUP ? BJ : 1] = {};
  i32x4 acc[BI][BJ] = {};
  const int G = GROUP ? K / GROUP : 1;
  const float* srow[BJ];
#pragma unroll
  for (int b = 0; b < BJ; ++b)
    srow[b] = sw + (size_t)min(n0 + qrow + 16 * b + (lane & 15), N - 1) * G;
  if constexpr (GROUP == 0) {
    mma_loop<S, BI, BJ>(lp, lq, 0, nk, lane, prow, qrow, stages, [](int) {},
                        [&](const u32x4& p, const u32x4& q, int a, int b, int)
                            __attribute__((always_inline)) {
                              acc[a][b] = Mma<kI8>::mul(p, q, acc[a][b]);
                            });
  } else {
    constexpr int GR = S * kChunk / GROUP;   // groups a round
    constexpr int GL = GR < 4 ? 1 : GR / 4;  // loads for them
    // the scales a round ahead of their use, as they come from memory; past the last
    // group 0
    float s[GR][BJ] = {};
    u32x4 ahead[GL][BJ];
    float before = 0.f, before0 = 0.f;   // the last block's, of the round before
    const Buffer scales = buffer_at(sw + (size_t)n0 * G, (size_t)(N - n0) * G * 4);
    uint32_t sat[BJ];
#pragma unroll
    for (int b = 0; b < BJ; ++b)
      sat[b] = (uint32_t)min(qrow + 16 * b + (lane & 15), N - 1 - n0) * (uint32_t)(4 * G);
    auto fetch = [&](int g0) __attribute__((always_inline)) {
#pragma unroll
      for (int b = 0; b < BJ; ++b)
#pragma unroll
        for (int l = 0; l < GL; ++l) {
          // (all of the offset in the part that is compared with the buffer's end)
          const int at = (int)sat[b] + 16 * l + 4 * g0;
          if constexpr (GR == 2) {
            const u32x2 w =
                __builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(scales, at, 0, 0));
            ahead[l][b] = u32x4{w[0], w[1], 0u, 0u};
          } else {
            ahead[l][b] =
                __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(scales, at, 0, 0));
          }
        }
    };
    fetch(0);
    // (here already: behind the tiles' loads every round would wait for all of those)
#pragma unroll
    for (int b = 0; b < BJ; ++b)
#pragma unroll
      for (int l = 0; l < GL; ++l) asm volatile("" : "+v"(ahead[l][b]));
    auto scale = [&](int a, int b, const i32x4& c, float sc) __attribute__((always_inline)) {
#pragma unroll
      for (int v = 0; v < 4; ++v) y[a][b][v] = fmaf((float)c[v], sc, y[a][b][v]);
    };
    const bool low = lane < 32;
    mma_loop<S, BI, BJ>(
        lp, lq, 0, nk, lane, prow, qrow, stages,
        [&](int q) __attribute__((always_inline)) {
          before = s[GR - 1][BJ - 1];
          before0 = GROUP == 32 ? s[GR - 2][BJ - 1] : 0.f;
#pragma unroll
          for (int g = 0; g < GR; ++g)
#pragma unroll
            for (int b = 0; b < BJ; ++b)
              s[g][b] = q / S * GR + g < G ? __uint_as_float(ahead[g / 4][b][g % 4]) : 0.f;
          fetch((q / S + 1) * GR);
        },
        [&](const u32x4& p, const u32x4& q, int a, int b, int i) __attribute__((always_inline)) {
          // the sums of the block before go to fp32 while the matrix cores form this one's
          const int at = a * BJ + b, pa = at ? (at - 1) / BJ : BI - 1, pb = at ? (at - 1) % BJ : BJ - 1;
          if constexpr (GROUP == 32) {
            // a chunk's 64 k are two groups: lanes 0-31 hold the first, 32-63 the second
            const u32x4 none = {};
            const i32x4 c0 = Mma<kI8>::mul(low ? p : none, q, i32x4{});
            const i32x4 c1 = Mma<kI8>::mul(low ? none : p, q, i32x4{});
            scale(pa, pb, acc[0][0], at ? s[2 * i][pb] : i ? s[2 * i - 2][pb] : before0);
            scale(pa, pb, acc[0][1], at ? s[2 * i + 1][pb] : i ? s[2 * i - 1][pb] : before);
            acc[0][0] = c0;
            acc[0][1] = c1;
          } else {
            constexpr int PER = GROUP / kChunk;   // chunks a group
            acc[a][b] = Mma<kI8>::mul(p, q, i % PER == 0 ? i32x4{} : acc[a][b]);
            if (at != 0 && i % PER == PER - 1) scale(pa, pb, acc[pa][pb], s[i / PER][pb]);
            if (at == 0 && i % PER == 0)
              scale(pa, pb, acc[pa][pb], i ? s[i / PER - 1][pb] : before);
          }
        });
    if constexpr (GROUP == 32) scale(BI - 1, BJ - 1, acc[0][0], s[GR - 2][BJ - 1]);
    scale(BI - 1, BJ - 1, GROUP == 32 ? acc[0][1] : acc[BI - 1][BJ - 1], s[GR - 1][BJ - 1]);
  }
  // Out through LDS as fp32, 32 tokens x 16 BJ channels of a wave at a time.
  constexpr int CH = 16 * BJ;
  constexpr int PER = STAGE / (32 * CH * 4);   // waves a stage serves
  static_assert(PER >= 1 && PER * 4 >= NW, "stage");
  float* const mine = (float*)(wave / PER == 0 ? stage0 : wave / PER == 1 ? stage1
                               : wave / PER == 2 ? stage2 : stage3) + wave % PER * 32 * CH;
  const int nw = n0 + qrow;
  // every token's scale before the first store: loaded row by row they cost their latency
  // each time (1993 x 128 -> 6966 in fp32: 33 us, now 27)
  float scale_of[BI][4];
#pragma unroll
  for (int a = 0; a < BI; ++a)
#pragma unroll
    for (int v = 0; v < 4; ++v)
      scale_of[a][v] = sx[min(t0 + prow + 16 * a + 4 * (lane >> 4) + v, T - 1)];
  // four values at a time where every row starts at their boundary and none ends inside four
  const bool wide = (uintptr_t)Y % (dtype == 0 ? 16 : 8) == 0 && N % 4 == 0;
#pragma unroll
  for (int aa = 0; aa < BI; aa += 2) {
#pragma unroll
    for (int a = aa; a < aa + 2; ++a)
#pragma unroll
      for (int b = 0; b < BJ; ++b)
#pragma unroll
        for (int v = 0; v < 4; ++v)
          mine[(16 * (a - aa) + 4 * (lane >> 4) + v) * CH + 16 * b + (lane & 15)] =
              (GROUP ? y[GROUP ? a : 0][GROUP ? b : 0][v] : (float)acc[a][b][v] * srow[b][0]) *
              scale_of[a][v];
    asm volatile("" ::: "memory");   // one wave: its LDS accesses complete in order
    const int tw = t0 + prow + 16 * aa;
    if (wide) {
#pragma unroll 1
      for (int p = lane; p < 32 * CH / 4; p += 64) {
        const int t = tw + p / (CH / 4), n = nw + 4 * (p % (CH / 4));
        if (t < T && n < N) {
          const f32x4 o = *(const f32x4*)(mine + 4 * p);
          const size_t e = (size_t)t * N + n;
          if (dtype == 0) *(f32x4*)((float*)Y + e) = o;
          else if (dtype == kF16)
            *(u32x2*)((uint16_t*)Y + e) = u32x2{pack16<kF16>(o[0], o[1]), pack16<kF16>(o[2], o[3])};
          else
            *(u32x2*)((uint16_t*)Y + e) =
                u32x2{pack16<kBF16>(o[0], o[1]), pack16<kBF16>(o[2], o[3])};
        }
      }
    } else {
      // a row (CH 64) or two (CH 32) at a time
      const int n = nw + lane % CH;
#pragma unroll 4
      for (int r = lane / CH; r < 32; r += 64 / CH)
        if (tw + r < T && n < N)
          store_y(Y, dtype, (size_t)(tw + r) * N + n, mine[r * CH + lane % CH]);
    }
    asm volatile("" ::: "memory");
  }
}

// Step `st` (64 k) of a wave's 16 x 16 block: GROUP 0 sums on; otherwise the group's
// integer sum is complete after its last step and goes to fp32 with its scale.
template <int GROUP, class Sum4>
__device__ __forceinline__ void i8_step(int st, const u32x4& fp, const u32x4& fq, bool low,
                                        const float* s, i32x4& acc, Sum4& sum) {
  if constexpr (GROUP == 0) {
    sum = Mma<kI8>::mul(fp, fq, sum);
  } else if constexpr (GROUP == 32) {
    // a step's 64 k are two groups: lanes 0-31 hold the first, 32-63 the second
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const u32x4 part = (h == 0) == low ? fp : u32x4{};
      const i32x4 c = Mma<kI8>::mul(part, fq, i32x4{});
#pragma unroll
      for (int v = 0; v < 4; ++v) sum[v] = fmaf((float)c[v], s[2 * st + h], sum[v]);
    }
  } else {
    constexpr int SG = GROUP / 64;   // steps a group
    acc = Mma<kI8>::mul(fp, fq, st % SG == 0 ? i32x4{} : acc);
    if (st % SG == SG - 1) {
#pragma unroll
      for (int v = 0; v < 4; ++v) sum[v] = fmaf((float)acc[v], s[st / SG], sum[v]);
    }
  }
}

// Few tokens: 16 JB channels x up to 16 IB tokens (blockIdx.y) a work-group, k dealt to
// its wavefronts.  Bound by a short launch's latency and the weights: four tokens, 4096 ->
// 4096 8.7 us with their quantization, 64 tokens 11.
template <int GROUP, int IB, int JB, int U>
__global__ __launch_bounds__(512) void i8_skinny_kernel(
    const int8_t* __restrict__ Xq, const float* __restrict__ sx, const int8_t* __restrict__ Wq,
    const float* __restrict__ sw, int T, int N, int K, int dtype, void* __restrict__ Y) {
  constexpr int NW = 8;
  constexpr int GU = GROUP ? 64 * U / GROUP : 1;   // groups a unit
  static_assert(GROUP == 0 || GU >= 1, "unit");
  typedef typename std::conditional<GROUP == 0, int32_t, float>::type Sum;
  typedef Sum Sum4 __attribute__((ext_vector_type(4)));
  __shared__ __attribute__((aligned(16))) Sum red[NW * IB * JB * 256];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n0 = blockIdx.x * 16 * JB, t0 = blockIdx.y * 16 * IB;
  const int row = lane & 15;
  const int G = GROUP ? K / GROUP : 1;
  const char *p[IB], *q[JB];
  const float* srow[JB];
#pragma unroll
  for (int a = 0; a < IB; ++a)
    p[a] = (const char*)Xq + (size_t)min(t0 + 16 * a + row, T - 1) * K;
#pragma unroll
  for (int b = 0; b < JB; ++b) {
    const int n = min(n0 + 16 * b + row, N - 1);
    q[b] = (const char*)Wq + (size_t)n * K;
    srow[b] = sw + (size_t)n * G;
  }
  float s[2][JB][GU];
  Sum4 sum[IB][JB] = {};
  i32x4 acc[IB][JB];
  const bool low = lane < 32;
  skinny_loop<IB, JB, U, NW>(
      p, q, K, wave, lane,
      [&](int u, int set) __attribute__((always_inline)) {
        if constexpr (GROUP != 0) {
#pragma unroll
          for (int b = 0; b < JB; ++b)
#pragma unroll
            for (int g = 0; g < GU; ++g)
              s[set][b][g] = u * GU + g < G ? srow[b][u * GU + g] : 0.f;
        }
      },
      [&](int st, int set, const u32x4(&fp)[IB], const u32x4(&fq)[JB])
          __attribute__((always_inline)) {
#pragma unroll
        for (int a = 0; a < IB; ++a)
#pragma unroll
          for (int b = 0; b < JB; ++b)
            i8_step<GROUP>(st, fp[a], fq[b], low, s[set][b], acc[a][b], sum[a][b]);
      });
#pragma unroll
  for (int a = 0; a < IB; ++a)
#pragma unroll
    for (int b = 0; b < JB; ++b)
      *(Sum4*)(red + ((wave * IB + a) * JB + b) * 256 + 4 * lane) = sum[a][b];
  __syncthreads();
  for (int e = threadIdx.x; e < IB * JB * 256; e += 512) {
    const int j = e % (16 * JB), i = e / (16 * JB) % 16, a = e / (256 * JB);
    const int t = t0 + 16 * a + i, c = n0 + j;
    if (t < T && c < N) {
      float y = (float)skinny_sum<NW, IB * JB>(red, a * JB + j / 16, i, j % 16);
      if (GROUP == 0) y *= sw[c];
      store_y(Y, dtype, (size_t)t * N + c, y * sx[t]);
    }
  }
}

// One or two tokens, quantized by every work-group for itself: one launch instead of two.
// The weights' first fragments are on their way while the tokens go to LDS as integers.
// 4096 -> 4096, weights from memory, launches back to back: one token 7.8 us (in two
// launches 8.2), two 8.7 (8.6), four 10.5 (8.7); a launch takes the host 3 us more.
constexpr int kFusedTokens = 2, kFusedBytes = 48 << 10;   // at most, tokens and bytes of them
template <int DT, int GROUP>
__global__ __launch_bounds__(512) void i8_fused_kernel(const void* __restrict__ X,
                                                       const int8_t* __restrict__ Wq,
                                                       const float* __restrict__ sw, int T, int N,
                                                       int K, void* __restrict__ Y) {
  constexpr int NW = 8, U = 4;
  constexpr int GU = GROUP ? 64 * U / GROUP : 1;
  typedef typename std::conditional<GROUP == 0, int32_t, float>::type Sum;
  typedef Sum Sum4 __attribute__((ext_vector_type(4)));
  extern __shared__ __attribute__((aligned(16))) char xq[];   // [T][K], 64 U bytes behind them
  __shared__ __attribute__((aligned(16))) Sum red[NW * 256];
  __shared__ uint32_t amax[kFusedTokens][NW];
  __shared__ float sx[kFusedTokens];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n0 = blockIdx.x * 16, row = lane & 15, at = 16 * (lane >> 4);
  const int n = min(n0 + row, N - 1);
  const int G = GROUP ? K / GROUP : 1;
  const char* q = (const char*)Wq + (size_t)n * K;
  const float* srow = sw + (size_t)n * G;
  const int units = (K + 64 * U - 1) / (64 * U);
  u32x4 fq[2][U];
  float s[2][GU];
  auto load = [&](int u, int set) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const int k = u * 64 * U + 64 * i + at;
      fq[set][i] = k < K ? *(const u32x4*)(q + k) : u32x4{};
    }
    if constexpr (GROUP != 0) {
#pragma unroll
      for (int g = 0; g < GU; ++g) s[set][g] = u * GU + g < G ? srow[u * GU + g] : 0.f;
    }
  };
  if (wave < units) load(wave, 0);
  const size_t es = DT == 0 ? 4 : 2;
  for (int t = 0; t < T; ++t) {
    uint32_t m = 0;
    for (int v = tid; v < K / 8; v += 512) {
      float x[8];
      unpack8<DT>(load_piece<DT>((const char*)X + (size_t)t * K * es, v), x);
#pragma unroll
      for (int i = 0; i < 8; ++i) m = max(m, abs_bits(x[i]));
    }
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) m = max(m, (uint32_t)__shfl_xor((int)m, off));
    if (lane == 0) amax[t][wave] = m;
  }
  __syncthreads();
  for (int t = 0; t < T; ++t) {
    uint32_t m = 0;
#pragma unroll
    for (int w = 0; w < NW; ++w) m = max(m, amax[t][w]);
    float scale, mul;
    row_scale(m, scale, mul);
    for (int v = tid; v < K / 8; v += 512) {
      float x[8];
      unpack8<DT>(load_piece<DT>((const char*)X + (size_t)t * K * es, v), x);
      *(u32x2*)(xq + t * K + 8 * v) = quant8(x, mul);
    }
    if (tid == t) sx[t] = scale;
  }
  __syncthreads();
  const char* p = xq + min(row, T - 1) * K + at;
  Sum4 sum = {};
  i32x4 acc;
  const bool low = lane < 32;
  auto mul = [&](int u, int set) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < U; ++i) {
      // (past k the weights are zeros)
      const u32x4 fp = *(const u32x4*)(p + u * 64 * U + 64 * i);
      i8_step<GROUP>(i, fp, fq[set][i], low, s[set], acc, sum);
    }
  };
  for (int u = wave; u < units; u += 2 * NW) {
    if (u + NW < units) load(u + NW, 1);
    mul(u, 0);
    if (u + NW < units) {
      if (u + 2 * NW < units) load(u + 2 * NW, 0);
      mul(u + NW, 1);
    }
  }
  *(Sum4*)(red + wave * 256 + 4 * lane) = sum;
  __syncthreads();
  if (tid < 256) {
    const int j = tid & 15, t = tid >> 4, c = n0 + j;
    if (t < T && c < N) {
      float y = (float)skinny_sum<NW, 1>(red, 0, t, j);
      if (GROUP == 0) y *= sw[c];
      store_y(Y, DT, (size_t)t * N + c, y * sx[t]);
    }
  }
}

template <int GROUP, int IB, int JB, int U>
static hipError_t launch_i8_skinny(hipStream_t st, int dtype, int T, int N, int K,
                                   const int8_t* Xq, const float* sx, const int8_t* Wq,
                                   const float* sw, void* Y) {
  const dim3 grid((N + 16 * JB - 1) / (16 * JB), (T + 16 * IB - 1) / (16 * IB));
  hipLaunchKernelGGL((i8_skinny_kernel<GROUP, IB, JB, U>), grid, dim3(512), 0, st, Xq, sx, Wq, sw,
                     T, N, K, dtype, Y);
  return hipGetLastError();
}
template <int GROUP, int S, int WI, int WJ, int BI, int BJ>
static hipError_t launch_i8_tiles(hipStream_t st, int dtype, int T, int N, int K, const int8_t* Xq,
                                  const float* sx, const int8_t* Wq, const float* sw, void* Y) {
  const int ni = (T + 16 * WI * BI - 1) / (16 * WI * BI);
  const int nj = (N + 16 * WJ * BJ - 1) / (16 * WJ * BJ);
  hipLaunchKernelGGL((i8_tile_kernel<GROUP, S, WI, WJ, BI, BJ>), dim3((unsigned)(ni * nj)),
                     dim3(64 * WI * WJ), 0, st, Xq, sx, Wq, sw, T, N, K, dtype, Y, ni, nj);
  return hipGetLastError();
}

// Up to 32 tokens, and up to 64 for layers of up to 8192 channels, fragments straight from
// memory; channels in blocks of 16 where wider ones are too few for the chip.  k = 4096:
// 64 tokens -> 4096 with 16, 32 channels a work-group 13, 11 us, tiles 14; 64 -> 1000 (groups
// of 32) 10, 18, 31; 37 -> 11008 (groups of 128) 29, 27 and 21.  Beyond, the tiles that
// tile_cost makes the cheapest, or fragments from memory again for a narrow layer (whose
// wavefronts cut k in eight).  k = 4096 -> 1000, 4096 and 11008 channels, in us with tiles of
// 256 x 256, 128 x 128 (tokens x channels), 128 x 64, 64 x 64, 64 x 32 and fragments:
//    128 tokens   43 19 14 11 10 10   43 21 16 12 10  31   44  22  18  20  21   78
//    512          46 21 16 12 10 31   46 22 18 21 29 114   51  40  46  52  65  301
//   2048          47 22 18 20 29 114  52 49 61 68 90 447  109 121 163 169 218 1198
// and groups of 64:
//    128              31 26 18 16 13       32 26 18 16  45        33  28  28  26  117
//    512              32 26 18 16 45       33 29 28 40 169        57  60  75  86  450
//   2048              33 29 28 39 167      66 84 97 118 669      178 212 254 293 1792
// Four stages against eight: 128 x 64 never slower, k = 256 -> 11008, 512 tokens 9.0 us and 17
// (three work-groups fit a CU, not one); 64 x 64 4.3 and 5.0 at k = 256, 13.6 and 12.8 at 4096.
// Groups at 128 x 128: eight wavefronts, since converting their sums takes the vector units
// twice as long as the matrix cores (3000 tokens, k = 2048 -> 1000, groups of 64: 20 us, four
// wavefronts 26).
template <int GROUP>
static hipError_t launch_i8_group(hipStream_t st, int dtype, int T, int N, int K, const int8_t* Xq,
                                  const float* sx, const int8_t* Wq, const float* sw, void* Y) {
  auto tiles = [&](int t, int n) { return (long long)((T + t - 1) / t) * ((N + n - 1) / n); };
  if (T <= 16 || (T <= 64 && N <= 2048))
    return launch_i8_skinny<GROUP, 1, 1, 4>(st, dtype, T, N, K, Xq, sx, Wq, sw, Y);
  if (T <= 32) return launch_i8_skinny<GROUP, 2, 1, 4>(st, dtype, T, N, K, Xq, sx, Wq, sw, Y);
  if (T <= 64 && N <= 8192)
    return launch_i8_skinny<GROUP, 2, 2, 2>(st, dtype, T, N, K, Xq, sx, Wq, sw, Y);
  const int nk = (K + kChunk - 1) / kChunk;
  constexpr TileTime plain[5] = {{7.0, 0.31, 2.5, 0.27},
                                 {4.7, 0.21, 1.1, 0.21},
                                 {3.6, 0.145, 0.6, 0.125},
                                 {3.5, 0.108, 0.5, 0.085},
                                 {2.4, 0.06, 0.25, 0.053}};
  constexpr TileTime grouped[5] = {{6.0, 0.53, 1.2, 0.37},
                                   {3.9, 0.39, 0.8, 0.30},
                                   {3.3, 0.25, 1.0, 0.165},
                                   {3.1, 0.205, 0.7, 0.105},
                                   {2.2, 0.085, 0.4, 0.083}};
  const TileTime* t = GROUP ? grouped : plain;
  const double cost[6] = {
      tile_cost(tiles(128, 128), nk, t[0]), tile_cost(tiles(128, 64), nk, t[1]),
      tile_cost(tiles(64, 64), nk, t[2]),   tile_cost(tiles(64, 32), nk, t[3]),
      tile_cost(tiles(16, 16), nk, t[4]),
      GROUP ? 1e30 : tile_cost(tiles(256, 256), nk, {15.0, 0.65, 15.0, 0.65})};
  switch ((int)(std::min_element(cost, cost + 6) - cost)) {
    case 0:
      return launch_i8_tiles<GROUP, 4, 2, GROUP ? 4 : 2, 4, GROUP ? 2 : 4>(st, dtype, T, N, K, Xq,
                                                                          sx, Wq, sw, Y);
    case 1:
      return launch_i8_tiles<GROUP, 4, 2, 2, 4, 2>(st, dtype, T, N, K, Xq, sx, Wq, sw, Y);
    case 2:
      if (nk <= 32)
        return launch_i8_tiles<GROUP, 4, 2, 2, 2, 2>(st, dtype, T, N, K, Xq, sx, Wq, sw, Y);
      return launch_i8_tiles<GROUP, 8, 2, 2, 2, 2>(st, dtype, T, N, K, Xq, sx, Wq, sw, Y);
    case 3:
      return launch_i8_tiles<GROUP, 8, 2, 1, 2, 2>(st, dtype, T, N, K, Xq, sx, Wq, sw, Y);
    case 4: return launch_i8_skinny<GROUP, 1, 1, 4>(st, dtype, T, N, K, Xq, sx, Wq, sw, Y);
    default:
      if constexpr (GROUP == 0)
        return launch_i8_tiles<0, 4, 2, 4, 8, 4>(st, dtype, T, N, K, Xq, sx, Wq, sw, Y);
      return hipErrorInvalidValue;
  }
}

hipError_t launch_matmul_i8(hipStream_t st, int dtype, int T, int N, int K, int group,
                            const int8_t* Xq, const float* sx, const int8_t* Wq, const float* sw,
                            void* Y) {
  switch (group) {
    case 0: return launch_i8_group<0>(st, dtype, T, N, K, Xq, sx, Wq, sw, Y);
    case 32: return launch_i8_group<32>(st, dtype, T, N, K, Xq, sx, Wq, sw, Y);
    case 64: return launch_i8_group<64>(st, dtype, T, N, K, Xq, sx, Wq, sw, Y);
    case 128: return launch_i8_group<128>(st, dtype, T, N, K, Xq, sx, Wq, sw, Y);
    default: return hipErrorInvalidValue;
  }
}

template <int DT>
static hipError_t launch_i8_fused(hipStream_t st, int T, int N, int K, int group, const void* X,
                                  const int8_t* Wq, const float* sw, void* Y) {
  const dim3 grid((N + 15) / 16), block(512);
  const size_t lds = (size_t)T * K + 256;
  if (group == 0)
    hipLaunchKernelGGL((i8_fused_kernel<DT, 0>), grid, block, lds, st, X, Wq, sw, T, N, K, Y);
  else if (group == 32)
    hipLaunchKernelGGL((i8_fused_kernel<DT, 32>), grid, block, lds, st, X, Wq, sw, T, N, K, Y);
  else if (group == 64)
    hipLaunchKernelGGL((i8_fused_kernel<DT, 64>), grid, block, lds, st, X, Wq, sw, T, N, K, Y);
  else
    hipLaunchKernelGGL((i8_fused_kernel<DT, 128>), grid, block, lds, st, X, Wq, sw, T, N, K, Y);
  return hipGetLastError();
}

hipError_t launch_linear_i8(hipStream_t st, int dtype, int T, int N, int K, int group,
                            const void* X, const int8_t* Wq, const float* sw, void* Y, int8_t* Xq,
                            float* sx) {
  if (T <= kFusedTokens && T * K <= kFusedBytes) {
    if (dtype == 0) return launch_i8_fused<0>(st, T, N, K, group, X, Wq, sw, Y);
    if (dtype == kF16) return launch_i8_fused<kF16>(st, T, N, K, group, X, Wq, sw, Y);
    return launch_i8_fused<kBF16>(st, T, N, K, group, X, Wq, sw, Y);
  }
  const hipError_t e = launch_quant_rows(st, dtype, X, T, K, Xq, sx);
  if (e != hipSuccess) return e;
  return launch_matmul_i8(st, dtype, T, N, K, group, Xq, sx, Wq, sw, Y);
}

}  // namespace jarq
