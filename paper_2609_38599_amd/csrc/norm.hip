// The root-mean-square norm of rows with the residual's addition, its result on 8 bits,
// and its backward pass.
//
// h = x + residual, rounded to the tokens' type (what the next residual addition and the
// backward pass read), r = 1 / sqrt(mean h^2 + eps), y = (h r) gain, rounded once.
// On 8 bits: w = h gain in fp32, a = max |w|, q = rint(w (127 / a)), scale = (a / 127) r.  r > 0
// scales a whole row, so the integers do not depend on it, nor on the order of its sum.
// Backward, u = dy gain: dx = r (u - h r^2 mean(u h)) + dh, dgain = sum_t dy (h r).
//
// Sums over a row are in fp64: squares of what fp32 or bf16 hold pass fp32's range (rows
// beyond 1.8e19 would come out as zeros), and the matrix-free kernels here are bound by
// memory, not by their arithmetic.
#include "mma_tile.h"

namespace jarq {

namespace {

// Eight values from element 8 v of a row at any element's alignment, as they are stored.
typedef u32x4 AnyVec __attribute__((aligned(2)));
template <int DT> struct Elem { typedef uint16_t T; };
template <> struct Elem<0> { typedef float T; };
template <int DT> struct Eight { u32x4 w[DT == 0 ? 2 : 1]; };

// Values past the row's end are 0.
template <int DT>
__device__ __forceinline__ Eight<DT> load8(const void* row, int v, int cols) {
  Eight<DT> p{};
  if (8 * v + 8 <= cols) {
#pragma unroll
    for (int i = 0; i < (DT == 0 ? 2 : 1); ++i)
      p.w[i] = *(const AnyVec*)((const typename Elem<DT>::T*)row + 8 * v + 4 * i);
  } else if (8 * v < cols) {
#pragma unroll
    for (int i = 0; i < 7; ++i) {
      if (8 * v + i >= cols) break;
      if constexpr (DT == 0)
        p.w[i / 4][i % 4] = ((const uint32_t*)row)[8 * v + i];
      else
        p.w[0][i / 2] |= (uint32_t)((const uint16_t*)row)[8 * v + i] << (16 * (i % 2));
    }
  }
  return p;
}
template <int DT>
__device__ __forceinline__ void store8(void* row, int v, int cols, const Eight<DT>& p) {
  if (8 * v + 8 <= cols) {
#pragma unroll
    for (int i = 0; i < (DT == 0 ? 2 : 1); ++i)
      *(AnyVec*)((typename Elem<DT>::T*)row + 8 * v + 4 * i) = p.w[i];
  } else if (8 * v < cols) {
#pragma unroll
    for (int i = 0; i < 7; ++i) {
      if (8 * v + i >= cols) break;
      if constexpr (DT == 0)
        ((uint32_t*)row)[8 * v + i] = p.w[i / 4][i % 4];
      else
        ((uint16_t*)row)[8 * v + i] = (uint16_t)(p.w[0][i / 2] >> (16 * (i % 2)));
    }
  }
}
template <int DT>
__device__ __forceinline__ void values(const Eight<DT>& p, float (&x)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    if constexpr (DT == 0) x[i] = __uint_as_float(p.w[i / 4][i % 4]);
    else x[i] = from16<DT>((uint16_t)(p.w[0][i / 2] >> (16 * (i % 2))));
  }
}
template <int DT>
__device__ __forceinline__ Eight<DT> rounded(const float (&x)[8]) {
  Eight<DT> p;
#pragma unroll
  for (int i = 0; i < (DT == 0 ? 8 : 4); ++i) {
    if constexpr (DT == 0) p.w[i / 4][i % 4] = __float_as_uint(x[i]);
    else p.w[0][i] = pack16<DT>(x[2 * i], x[2 * i + 1]);
  }
  return p;
}

__device__ __forceinline__ double wave_sum(double s) {
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) s += __shfl_xor(s, off);
  return s;
}
// |x| as ordered bits: NaN above infinity above every finite value
__device__ __forceinline__ uint32_t abs_bits(float x) { return __float_as_uint(x) & 0x7fffffffu; }
constexpr uint32_t kInfBits = 0x7f800000u;
constexpr uint32_t kTinyBits = 0x0d800000u;   // 2^-100

// A row's scale and multiplier on 8 bits from its largest |w| (as jarq_quant_rows_i8).
__device__ __forceinline__ void scale_of(uint32_t amax_bits, float r, float& scale, float& mul) {
  const float amax = __uint_as_float(amax_bits);
  mul = 0.f;
  if (amax_bits >= kInfBits) {
    scale = __uint_as_float(0x7fc00000u);
  } else if (amax_bits < kTinyBits) {
    scale = 0.f;
  } else {
    scale = amax / 127.f * r;
    mul = 127.f / amax;
  }
}
__device__ __forceinline__ u32x2 eight_i8(const float (&w)[8], float mul) {
  u32x2 q{};
  if (mul != 0.f)
#pragma unroll
    for (int i = 0; i < 8; ++i)
      q[i / 4] |= ((uint32_t)(int)rintf(w[i] * mul) & 0xffu) << (8 * (i % 4));
  return q;
}

__device__ __forceinline__ float inverse_rms(double squares, int cols, float eps) {
  return (float)(1.0 / sqrt(squares / cols + (double)eps));
}

}  // namespace

// ---- forward ----
// NW wavefronts a row, which stays in registers (R pieces of eight values a lane) between
// its sum and its outputs; what is beyond 512 NW R columns is read again, from H where there
// is a residual (H may be X or the residual: each lane reads an element before it writes it).
// Bound by memory: 8192 x 4096 in bf16 with a residual 47 to 49 us, 5.6 TB/s; 4096 x 4096 on 8 bits
// 23.5 us, 5.0 TB/s.  A row of 4096 by four wavefronts: one row's loads are all in flight at once and
// eight rows share a unit; up to 1024 columns a wavefront has a row to itself and needs no barrier.
template <int DT, bool GAIN32, bool I8, int NW, int R>
__global__ __launch_bounds__(256) void norm_kernel(const void* X, const void* residual,
                                                   const void* __restrict__ gain, float eps, int T,
                                                   int cols, void* H, void* Y, float* scale) {
  constexpr int GT = GAIN32 ? 0 : DT, LANES = 64 * NW, E = DT == 0 ? 4 : 2;
  __shared__ double red[4];
  __shared__ uint32_t redm[4];
  const int lane = NW == 1 ? threadIdx.x & 63 : threadIdx.x;
  const int t = NW == 1 ? blockIdx.x * 4 + (threadIdx.x >> 6) : blockIdx.x;
  if (t >= T) return;   // (only where a wave has a row for itself: no barrier behind it)
  const size_t at = (size_t)t * cols * E;
  const char* const x = (const char*)X + at;
  const char* const res = residual ? (const char*)residual + at : nullptr;
  char* const h = residual ? (char*)H + at : nullptr;
  const int nv = (cols + 7) / 8;
  double ss = 0.0;
  uint32_t most = 0;
  Eight<DT> keep[R];
  // the sum's piece v, with what it adds to the row's statistics
  auto take = [&](const Eight<DT>& a, const Eight<DT>& b, int v) __attribute__((always_inline)) {
    Eight<DT> p = a;
    float f[8];
    values<DT>(a, f);
    if (res) {
      float g[8];
      values<DT>(b, g);
#pragma unroll
      for (int i = 0; i < 8; ++i) f[i] += g[i];
      p = rounded<DT>(f);
      values<DT>(p, f);
      store8<DT>(h, v, cols, p);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) ss = fma((double)f[i], (double)f[i], ss);
    if constexpr (I8) {
      float g[8];
      values<GT>(load8<GT>(gain, v, cols), g);
#pragma unroll
      for (int i = 0; i < 8; ++i) most = max(most, abs_bits(f[i] * g[i]));
    }
    return p;
  };
  {
    Eight<DT> b[R];
#pragma unroll
    for (int i = 0; i < R; ++i) {
      keep[i] = load8<DT>(x, lane + LANES * i, cols);
      if (res) b[i] = load8<DT>(res, lane + LANES * i, cols);
    }
#pragma unroll
    for (int i = 0; i < R; ++i)
      if (LANES * i < nv) keep[i] = take(keep[i], b[i], lane + LANES * i);
  }
  for (int v = lane + LANES * R; v < nv; v += LANES)
    take(load8<DT>(x, v, cols), res ? load8<DT>(res, v, cols) : Eight<DT>{}, v);
  ss = wave_sum(ss);
  if constexpr (I8)
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) most = max(most, (uint32_t)__shfl_xor((int)most, off));
  if constexpr (NW > 1) {
    if ((lane & 63) == 0) {
      red[lane >> 6] = ss;
      if constexpr (I8) redm[lane >> 6] = most;
    }
    __syncthreads();
    ss = (red[0] + red[1]) + (red[2] + red[3]);
    if constexpr (I8) most = max(max(redm[0], redm[1]), max(redm[2], redm[3]));
  }
  const float r = inverse_rms(ss, cols, eps);
  float sc = 0.f, mul = 0.f;
  if constexpr (I8) {
    scale_of(most, r, sc, mul);
    if (lane == 0) scale[t] = sc;
  }
  auto put = [&](const Eight<DT>& p, int v) __attribute__((always_inline)) {
    float f[8], g[8];
    values<DT>(p, f);
    values<GT>(load8<GT>(gain, v, cols), g);
    if constexpr (I8) {
#pragma unroll
      for (int i = 0; i < 8; ++i) f[i] *= g[i];
      *(u32x2*)((char*)Y + (size_t)t * cols + 8 * (size_t)v) = eight_i8(f, mul);   // cols % 16 = 0
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) f[i] = f[i] * r * g[i];
      store8<DT>((char*)Y + at, v, cols, rounded<DT>(f));
    }
  };
#pragma unroll
  for (int i = 0; i < R; ++i)
    if (lane + LANES * i < nv) put(keep[i], lane + LANES * i);
  for (int v = lane + LANES * R; v < nv; v += LANES) put(load8<DT>(res ? h : x, v, cols), v);
}

template <int DT, bool GAIN32, bool I8>
static hipError_t launch_norm_of(hipStream_t st, const void* X, const void* residual,
                                 const void* gain, float eps, int T, int cols, void* H, void* Y,
                                 float* scale) {
  const dim3 four((T + 3) / 4), one(T), b(256);
#define JARQ_NORM(GRID, NW, R)                                                                  \
  hipLaunchKernelGGL((norm_kernel<DT, GAIN32, I8, NW, R>), GRID, b, 0, st, X, residual, gain,   \
                     eps, T, cols, H, Y, scale)
  if (cols <= 512) JARQ_NORM(four, 1, 1);
  else if (cols <= 1024) JARQ_NORM(four, 1, 2);
  else if (cols <= 2048) JARQ_NORM(one, 4, 1);
  else if (cols <= 4096) JARQ_NORM(one, 4, 2);
  else if (cols <= 8192) JARQ_NORM(one, 4, 4);
  else JARQ_NORM(one, 4, 8);
#undef JARQ_NORM
  return hipGetLastError();
}

template <bool I8>
static hipError_t launch_norm_form(hipStream_t st, int dtype, int gain_dtype, const void* X,
                                   const void* residual, const void* gain, float eps, int T,
                                   int cols, void* H, void* Y, float* scale) {
  const bool g32 = gain_dtype == 0;
  if (dtype == 0)
    return launch_norm_of<0, true, I8>(st, X, residual, gain, eps, T, cols, H, Y, scale);
  if (dtype == kF16)
    return g32 ? launch_norm_of<kF16, true, I8>(st, X, residual, gain, eps, T, cols, H, Y, scale)
               : launch_norm_of<kF16, false, I8>(st, X, residual, gain, eps, T, cols, H, Y, scale);
  return g32 ? launch_norm_of<kBF16, true, I8>(st, X, residual, gain, eps, T, cols, H, Y, scale)
             : launch_norm_of<kBF16, false, I8>(st, X, residual, gain, eps, T, cols, H, Y, scale);
}

hipError_t launch_rms_norm(hipStream_t st, int dtype, int gain_dtype, const void* X,
                           const void* residual, const void* gain, float eps, int T, int cols,
                           void* H, void* Y) {
  return launch_norm_form<false>(st, dtype, gain_dtype, X, residual, gain, eps, T, cols, H, Y,
                                 nullptr);
}
hipError_t launch_rms_norm_i8(hipStream_t st, int dtype, int gain_dtype, const void* X,
                              const void* residual, const void* gain, float eps, int T, int cols,
                              void* H, int8_t* Q, float* scale) {
  return launch_norm_form<true>(st, dtype, gain_dtype, X, residual, gain, eps, T, cols, H, Q,
                                scale);
}

// ---- backward ----
// As forward, for rows w, w + step, ... (a row's NW wavefronts work together, 4 / NW rows of
// a work-group side by side); a lane's columns are the same in every row, so that it adds
// dgain up in registers.  part [work-groups][cols]: their sums.  Bound by memory: 8192 x 4096 in bf16
// with dH 51 to 55 us, 5 TB/s (one wavefront a row 73, two 57: more registers each, fewer rows
// in flight).
template <int DT, bool GAIN32, int NW, int R>
__global__ __launch_bounds__(NW > 4 ? 64 * NW : 256) void norm_grad_kernel(
    const void* __restrict__ H, const void* __restrict__ gain, const void* dY, const void* dH,
    float eps, int T, int cols, void* dX, float* __restrict__ part) {
  constexpr int GT = GAIN32 ? 0 : DT, LANES = 64 * NW, E = DT == 0 ? 4 : 2;
  constexpr int TEAMS = NW < 4 ? 4 / NW : 1;
  __shared__ double red[2][2 * NW];
  __shared__ float sums[TEAMS > 1 ? (TEAMS - 1) * 512 * R : 1];
  const int lane = threadIdx.x % LANES, team = threadIdx.x / LANES;
  float acc[R][8] = {};
  int odd = 0;
  for (int t = blockIdx.x * TEAMS + team; t < T; t += gridDim.x * TEAMS) {
    const size_t at = (size_t)t * cols * E;
    Eight<DT> ph[R], py[R], pd[R];
#pragma unroll
    for (int i = 0; i < R; ++i) {
      const int v = lane + LANES * i;
      ph[i] = load8<DT>((const char*)H + at, v, cols);
      py[i] = load8<DT>((const char*)dY + at, v, cols);
      if (dX && dH) pd[i] = load8<DT>((const char*)dH + at, v, cols);
    }
    double ss = 0.0, su = 0.0;
#pragma unroll
    for (int i = 0; i < R; ++i) {
      float h[8], y[8], g[8];
      values<DT>(ph[i], h);
      values<DT>(py[i], y);
      values<GT>(load8<GT>(gain, lane + LANES * i, cols), g);
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        ss = fma((double)h[k], (double)h[k], ss);
        su = fma((double)(y[k] * g[k]), (double)h[k], su);
      }
    }
    ss = wave_sum(ss);
    su = wave_sum(su);
    if constexpr (NW > 1) {   // two sets of slots: a row's are written while the last one's are read
      if ((lane & 63) == 0) {
        red[odd][lane >> 6] = ss;
        red[odd][NW + (lane >> 6)] = su;
      }
      __syncthreads();
      ss = su = 0.0;
#pragma unroll
      for (int w = 0; w < NW; ++w) {
        ss += red[odd][w];
        su += red[odd][NW + w];
      }
      odd ^= 1;
    }
    const float r = inverse_rms(ss, cols, eps);
    const float c = (float)(su / cols / (ss / cols + (double)eps));
#pragma unroll
    for (int i = 0; i < R; ++i) {
      const int v = lane + LANES * i;
      float h[8], y[8], g[8];
      values<DT>(ph[i], h);
      values<DT>(py[i], y);
      if (dX) {
        values<GT>(load8<GT>(gain, v, cols), g);
        float d[8] = {}, x[8];
        if (dH) values<DT>(pd[i], d);
#pragma unroll
        for (int k = 0; k < 8; ++k) x[k] = fmaf(r, fmaf(-h[k], c, y[k] * g[k]), d[k]);
        store8<DT>((char*)dX + at, v, cols, rounded<DT>(x));
      }
#pragma unroll
      for (int k = 0; k < 8; ++k) acc[i][k] = fmaf(y[k], h[k] * r, acc[i][k]);
    }
  }
  if (!part) return;   // uniform
  if constexpr (TEAMS > 1) {   // the teams' sums in their order
    if (team > 0)
#pragma unroll
      for (int i = 0; i < R; ++i)
#pragma unroll
        for (int k = 0; k < 8; ++k)
          sums[((team - 1) * R + i) * 512 + 64 * k + lane] = acc[i][k];
    __syncthreads();
    if (team > 0) return;
#pragma unroll
    for (int i = 0; i < R; ++i)
#pragma unroll
      for (int k = 0; k < 8; ++k)
#pragma unroll
        for (int m = 0; m < TEAMS - 1; ++m)
          acc[i][k] += sums[(m * R + i) * 512 + 64 * k + lane];
  }
#pragma unroll
  for (int i = 0; i < R; ++i)
    store8<0>(part + (size_t)blockIdx.x * cols, lane + LANES * i, cols, rounded<0>(acc[i]));
}

// dgain from the work-groups' sums, in a fixed order: 64 columns, sixteen shares of the parts.  Bound
// by latency: 1024 parts of 4096 columns (17 MB) 5 us, one load at a time 10.
template <int GT>
__global__ __launch_bounds__(1024) void norm_gain_kernel(const float* __restrict__ part, int parts,
                                                        int cols, void* dgain) {
  __shared__ float red[16][65];
  const int j = threadIdx.x & 63, s = threadIdx.x >> 6;
  const int c = blockIdx.x * 64 + j;
  float sum = 0.f;
  if (c < cols) {
    int p = s;
    for (; p + 112 < parts; p += 128) {
      float x[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = part[(size_t)(p + 16 * i) * cols + c];
#pragma unroll
      for (int i = 0; i < 8; ++i) sum += x[i];
    }
    for (; p < parts; p += 16) sum += part[(size_t)p * cols + c];
  }
  red[s][j] = sum;
  __syncthreads();
  if (s == 0 && c < cols) {
#pragma unroll
    for (int i = 1; i < 16; ++i) sum += red[i][j];
    if constexpr (GT == 0) ((float*)dgain)[c] = sum;
    else ((uint16_t*)dgain)[c] = to16<GT>(sum);
  }
}

// Rows that pass the registers: read twice, dgain apart from each row's r.
template <int DT, bool GAIN32>
__global__ __launch_bounds__(256) void norm_grad_long_kernel(
    const void* __restrict__ H, const void* __restrict__ gain, const void* dY, const void* dH,
    float eps, int cols, void* dX, float* __restrict__ rs) {
  constexpr int GT = GAIN32 ? 0 : DT, E = DT == 0 ? 4 : 2;
  __shared__ double red[8];
  const int lane = threadIdx.x;
  const size_t at = (size_t)blockIdx.x * cols * E;
  const int nv = (cols + 7) / 8;
  double ss = 0.0, su = 0.0;
  for (int v = lane; v < nv; v += 256) {
    float h[8], y[8], g[8];
    values<DT>(load8<DT>((const char*)H + at, v, cols), h);
    values<DT>(load8<DT>((const char*)dY + at, v, cols), y);
    values<GT>(load8<GT>(gain, v, cols), g);
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      ss = fma((double)h[k], (double)h[k], ss);
      su = fma((double)(y[k] * g[k]), (double)h[k], su);
    }
  }
  ss = wave_sum(ss);
  su = wave_sum(su);
  if ((lane & 63) == 0) {
    red[lane >> 6] = ss;
    red[4 + (lane >> 6)] = su;
  }
  __syncthreads();
  ss = (red[0] + red[1]) + (red[2] + red[3]);
  su = (red[4] + red[5]) + (red[6] + red[7]);
  const float r = inverse_rms(ss, cols, eps);
  const float c = (float)(su / cols / (ss / cols + (double)eps));
  if (lane == 0 && rs) rs[blockIdx.x] = r;
  if (!dX) return;
  for (int v = lane; v < nv; v += 256) {
    float h[8], y[8], g[8], d[8] = {}, x[8];
    values<DT>(load8<DT>((const char*)H + at, v, cols), h);
    values<DT>(load8<DT>((const char*)dY + at, v, cols), y);
    values<GT>(load8<GT>(gain, v, cols), g);
    if (dH) values<DT>(load8<DT>((const char*)dH + at, v, cols), d);
#pragma unroll
    for (int k = 0; k < 8; ++k) x[k] = fmaf(r, fmaf(-h[k], c, y[k] * g[k]), d[k]);
    store8<DT>((char*)dX + at, v, cols, rounded<DT>(x));
  }
}
// part of rows blockIdx.y, blockIdx.y + gridDim.y, ...
template <int DT>
__global__ __launch_bounds__(256) void norm_gain_long_kernel(const void* __restrict__ H,
                                                             const void* __restrict__ dY,
                                                             const float* __restrict__ rs, int T,
                                                             int cols, float* __restrict__ part) {
  constexpr int E = DT == 0 ? 4 : 2;
  const int v = blockIdx.x * 256 + threadIdx.x;
  if (8 * v >= cols) return;
  float acc[8] = {};
  for (int t = blockIdx.y; t < T; t += gridDim.y) {
    const size_t at = (size_t)t * cols * E;
    float h[8], y[8];
    values<DT>(load8<DT>((const char*)H + at, v, cols), h);
    values<DT>(load8<DT>((const char*)dY + at, v, cols), y);
    const float r = rs[t];
#pragma unroll
    for (int k = 0; k < 8; ++k) acc[k] = fmaf(y[k], h[k] * r, acc[k]);
  }
  store8<0>(part + (size_t)blockIdx.y * cols, v, cols, rounded<0>(acc));
}

namespace {

constexpr int kMostCols = 16384;   // of a row in registers

// Work-groups of the backward pass, each with a part of dgain: as many as are on the card at once by
// their registers (8192 x 4096 in bf16: 256, 512, 768, 1024 of them 79, 58, 53, 51 us).
int norm_parts(int T, int cols) {
  const int rows = cols <= 1024 ? 4 : 1;   // at a time
  return std::max(1, std::min(cols <= 4096 ? 1024 : 512, (T + rows - 1) / rows));
}
int norm_long_parts(int T) { return std::max(1, std::min(64, T)); }

size_t pad256(size_t n) { return (n + 255) & ~(size_t)255; }

}  // namespace

size_t rms_norm_workspace_bytes(int T, int cols) {
  if (cols > kMostCols) return pad256(4 * (size_t)T) + 4 * (size_t)norm_long_parts(T) * cols;
  return 4 * (size_t)norm_parts(T, cols) * cols;
}

template <int DT, bool GAIN32>
static hipError_t launch_norm_grad(hipStream_t st, const void* H, const void* gain, const void* dY,
                                   const void* dH, float eps, int T, int cols, void* dX,
                                   void* dgain, char* ws) {
  constexpr int GT = GAIN32 ? 0 : DT;
  int parts = norm_parts(T, cols);
  float* part = dgain ? (float*)ws : nullptr;
  if (cols > kMostCols) {
    float* rs = dgain ? (float*)ws : nullptr;
    // dgain reads dY once more: where dX lies over it, before dX is formed
    const bool over = dgain && dX == dY;
    if (T > 0)
      hipLaunchKernelGGL((norm_grad_long_kernel<DT, GAIN32>), dim3(T), dim3(256), 0, st, H, gain,
                         dY, dH, eps, cols, over ? nullptr : dX, rs);
    if (dgain) {
      parts = norm_long_parts(T);
      part = (float*)(ws + pad256(4 * (size_t)T));
      hipLaunchKernelGGL((norm_gain_long_kernel<DT>), dim3((cols + 2047) / 2048, parts), dim3(256),
                         0, st, H, dY, rs, T, cols, part);
    }
    if (T > 0 && over)
      hipLaunchKernelGGL((norm_grad_long_kernel<DT, GAIN32>), dim3(T), dim3(256), 0, st, H, gain,
                         dY, dH, eps, cols, dX, nullptr);
  } else {
#define JARQ_NORM_GRAD(NW, R)                                                                   \
  hipLaunchKernelGGL((norm_grad_kernel<DT, GAIN32, NW, R>), dim3(parts),                        \
                     dim3(NW > 4 ? 64 * NW : 256), 0, st, H, gain, dY, dH, eps, T, cols, dX,    \
                     part)
    if (cols <= 512) JARQ_NORM_GRAD(1, 1);
    else if (cols <= 1024) JARQ_NORM_GRAD(1, 2);
    else if (cols <= 2048) JARQ_NORM_GRAD(4, 1);
    else if (cols <= 4096) JARQ_NORM_GRAD(4, 2);
    else if (cols <= 8192) JARQ_NORM_GRAD(4, 4);
    else JARQ_NORM_GRAD(8, 4);
#undef JARQ_NORM_GRAD
  }
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || !dgain) return e;
  hipLaunchKernelGGL((norm_gain_kernel<GT>), dim3((cols + 63) / 64), dim3(1024), 0, st, part, parts,
                     cols, dgain);
  return hipGetLastError();
}

hipError_t launch_rms_norm_backward(hipStream_t st, int dtype, int gain_dtype, const void* H,
                                    const void* gain, const void* dY, const void* dH, float eps,
                                    int T, int cols, void* dX, void* dgain, char* ws) {
  const bool g32 = gain_dtype == 0;
  if (dtype == 0)
    return launch_norm_grad<0, true>(st, H, gain, dY, dH, eps, T, cols, dX, dgain, ws);
  if (dtype == kF16)
    return g32 ? launch_norm_grad<kF16, true>(st, H, gain, dY, dH, eps, T, cols, dX, dgain, ws)
               : launch_norm_grad<kF16, false>(st, H, gain, dY, dH, eps, T, cols, dX, dgain, ws);
  return g32 ? launch_norm_grad<kBF16, true>(st, H, gain, dY, dH, eps, T, cols, dX, dgain, ws)
             : launch_norm_grad<kBF16, false>(st, H, gain, dY, dH, eps, T, cols, dX, dgain, ws);
}

}  // namespace jarq
