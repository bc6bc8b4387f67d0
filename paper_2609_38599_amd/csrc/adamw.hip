// A step of AdamW over many tensors at once, the moments in 32 bits or in 8.
//
//     m = b1 m + (1 - b1) g,  v = b2 v + (1 - b2) g^2,
//     p = p (1 - lr wd) - (lr / (1 - b1^t)) m / (sqrt(v) / sqrt(1 - b2^t) + eps),
//
// each product and sum rounded to fp32 by itself, so that what is held in 8 bits is the same
// wherever it is computed.  On 8 bits m and sqrt(v) are e4m3 values times a power of two a
// block of 128, the block's largest in 2^7..2^8.  sqrt(v), not v: half the binades.  A power of
// two, not a quotient: a block's new scale moves none of its values off their grid.  Rounded by
// a dither, not to nearest: a step moves v by a thousandth of itself, e4m3's grid is an
// eighth wide, so that to nearest v would stay where it is until g^2 is a hundred times v;
// with the dither it moves as far as it should on average.  sqrt(v) > 0 stays above 0: beside an
// m that survives its rounding, 0 would make the step m / eps.
#include "mma_tile.h"

namespace jarq {

namespace {

typedef u32x4 AnyVec __attribute__((aligned(2)));   // sixteen bytes at any element

constexpr int kUnit = 2048;     // values a work-group takes at a time, eight a lane
constexpr int kTensors = 64;    // of a launch: one a lane where a work-group looks for its own

struct AdamTensor {
  const void* grad;
  const void* param;
  void* param_out;
  int64_t at, n;   // where its moments begin, its length
};
struct AdamArgs {
  AdamTensor tensor[kTensors];
  uint32_t first[kTensors];   // its first unit; past the last tensor: none
};
struct AdamScalars {
  float b1, c1, b2, c2, eps;
  float rate, root, keep;       // lr / (1 - b1^t), 1 / sqrt(1 - b2^t), 1 - lr wd
  uint32_t key;
  double lr, beta1, beta2, decay;
  uint64_t seed;
  int64_t step;
  const float *lr_at, *grad_mul;
  const int64_t* step_at;
};

// 32 bits of noise from 32.
__host__ __device__ inline uint32_t mix(uint32_t x) {
  x ^= x >> 16;
  x *= 0x9E3779B9u;
  x ^= x >> 15;
  x *= 0xBB67AE85u;
  return x ^ (x >> 16);
}
__host__ __device__ inline uint32_t key_of(uint64_t seed, int64_t step) {
  return mix(mix(mix((uint32_t)seed) + (uint32_t)(seed >> 32)) + (uint32_t)step);
}
// What the step number and the rate fix.
__host__ __device__ inline void set_step(AdamScalars& s, double lr, int64_t step) {
#pragma clang fp contract(off)
  double p1 = 1.0, p2 = 1.0, a = s.beta1, b = s.beta2;
  for (uint64_t t = (uint64_t)step; t != 0; t >>= 1) {
    if (t & 1) {
      p1 *= a;
      p2 *= b;
    }
    a *= a;
    b *= b;
  }
  s.rate = (float)(lr / (1.0 - p1));
  s.root = (float)(1.0 / sqrt(1.0 - p2));
  s.keep = (float)(1.0 - lr * s.decay);
  s.key = key_of(s.seed, step);
}

template <int DT>
__device__ __forceinline__ void load_values(const void* from, int64_t i, int64_t n, float (&x)[8]) {
  if (i + 8 <= n) {
    if constexpr (DT == 0) {
      const u32x4 a = *(const AnyVec*)((const float*)from + i);
      const u32x4 b = *(const AnyVec*)((const float*)from + i + 4);
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        x[k] = __uint_as_float(a[k]);
        x[4 + k] = __uint_as_float(b[k]);
      }
    } else {
      const u32x4 a = *(const AnyVec*)((const uint16_t*)from + i);
#pragma unroll
      for (int k = 0; k < 8; ++k) x[k] = from16<DT>((uint16_t)(a[k / 2] >> (16 * (k % 2))));
    }
  } else {
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      x[k] = 0.f;
      if (i + k < n) {
        if constexpr (DT == 0) x[k] = ((const float*)from)[i + k];
        else x[k] = from16<DT>(((const uint16_t*)from)[i + k]);
      }
    }
  }
}
template <int DT>
__device__ __forceinline__ void store_values(void* to, int64_t i, int64_t n, const float (&x)[8]) {
  if (i + 8 <= n) {
    if constexpr (DT == 0) {
      u32x4 a, b;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        a[k] = __float_as_uint(x[k]);
        b[k] = __float_as_uint(x[4 + k]);
      }
      *(AnyVec*)((float*)to + i) = a;
      *(AnyVec*)((float*)to + i + 4) = b;
    } else {
      u32x4 a;
#pragma unroll
      for (int k = 0; k < 4; ++k) a[k] = pack16<DT>(x[2 * k], x[2 * k + 1]);
      *(AnyVec*)((uint16_t*)to + i) = a;
    }
  } else {
#pragma unroll
    for (int k = 0; k < 8; ++k)
      if (i + k < n) {
        if constexpr (DT == 0) ((float*)to)[i + k] = x[k];
        else ((uint16_t*)to)[i + k] = to16<DT>(x[k]);
      }
  }
}
// Eight values of a state array (padded to whole blocks, 16-byte aligned).
__device__ __forceinline__ void load_state(const float* from, int64_t i, float (&x)[8]) {
  const f32x4 a = *(const f32x4*)(from + i), b = *(const f32x4*)(from + i + 4);
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    x[k] = a[k];
    x[4 + k] = b[k];
  }
}
__device__ __forceinline__ void store_state(float* to, int64_t i, const float (&x)[8]) {
  *(f32x4*)(to + i) = f32x4{x[0], x[1], x[2], x[3]};
  *(f32x4*)(to + i + 4) = f32x4{x[4], x[5], x[6], x[7]};
}

// e4m3 values and their block's power of two.
__device__ __forceinline__ void decode(u32x2 w, uint32_t e, float (&x)[8]) {
  const int by = (int)e - 134;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const auto f = k % 2 ? __builtin_amdgcn_cvt_pk_f32_fp8((int)w[k / 2], true)
                         : __builtin_amdgcn_cvt_pk_f32_fp8((int)w[k / 2], false);
    x[2 * k] = __builtin_ldexpf(f[0], by);
    x[2 * k + 1] = __builtin_ldexpf(f[1], by);
  }
}
// The largest of the sixteen lanes that share a block.
__device__ __forceinline__ uint32_t block_max(uint32_t m) {
  m = max(m, (uint32_t)__builtin_amdgcn_mov_dpp((int)m, 0x128, 0xf, 0xf, true));   // row_ror
  m = max(m, (uint32_t)__builtin_amdgcn_mov_dpp((int)m, 0x124, 0xf, 0xf, true));
  m = max(m, (uint32_t)__builtin_amdgcn_mov_dpp((int)m, 0x122, 0xf, 0xf, true));
  m = max(m, (uint32_t)__builtin_amdgcn_mov_dpp((int)m, 0x121, 0xf, 0xf, true));
  return m;
}
// noise: 16 bits a value, which reach the 16 highest of the 20 that are cut off (a rounding
// up is too rare by 2^-17 of a step).
template <bool POSITIVE>
__device__ __forceinline__ u32x2 encode(const float (&x)[8], const uint32_t (&noise)[8],
                                        uint32_t& e) {
  uint32_t most = 0;
#pragma unroll
  for (int k = 0; k < 8; ++k) most = max(most, __float_as_uint(x[k]) & 0x7fffffffu);
  const uint32_t field = max(block_max(most) >> 23, 1u);
  e = field;
  if (field == 255) return u32x2{0x7f7f7f7fu, 0x7f7f7f7fu};   // NaN: the largest is no number
  u32x2 w{};
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    // (the bits of value 2^-120 in fp32 are e4m3's, 20 places further up)
    const float s = __builtin_ldexpf(fabsf(x[k]), 14 - (int)field);
    uint32_t c = (__float_as_uint(s) + (noise[k] << 4)) >> 20;
    if (POSITIVE) c = max(c, x[k] > 0.f ? 1u : 0u);
    else c |= x[k] < 0.f ? 0x80u : 0u;
    w[k / 4] |= c << (8 * (k % 4));
  }
  return w;
}

// p, m and v of the step; root becomes sqrt(v).
__device__ __forceinline__ void advance(const AdamScalars& s, float g, float& p, float& m,
                                        float& v, float& root) {
#pragma clang fp contract(off)
  m = s.b1 * m + s.c1 * g;
  v = s.b2 * v + (s.c2 * g) * g;
  root = sqrtf(v);   // (the correctly rounded one: the integers hang on it)
  p = s.keep * p - (s.rate * m) * __builtin_amdgcn_rcpf(root * s.root + s.eps);
}

}  // namespace

// dtype of the parameters and gradients; BITS of the moments.  A work-group takes 2048 values, a
// lane eight of each array, all loaded at once; sixteen lanes are a block on 8 bits, whose largest
// comes by four exchanges in a row of lanes.  Bound by memory: 135 M values in bf16, moments in
// 32 bits (28 bytes a value) 686 us, 5.5 TB/s, in 8 (16.03 bytes) 371 to 378 us, 5.8 TB/s; the noise, the
// roundings and a correctly rounded root are hidden behind it.
template <int DT, int BITS>
__global__ __launch_bounds__(256) void adamw_kernel(AdamArgs a, AdamScalars s, jarq_adamw_state in,
                                                    jarq_adamw_state out, int same) {
  const uint32_t unit = blockIdx.x;
  const int k = __builtin_amdgcn_readfirstlane(
      __popcll(__ballot(a.first[threadIdx.x & 63] <= unit)) - 1);
  const int64_t n = a.tensor[k].n;
  const int64_t i = (int64_t)(unit - a.first[k]) * kUnit + 8 * threadIdx.x;   // in its tensor
  const int64_t at = a.tensor[k].at + i;                                      // in the state
  const bool live = i < n;   // (no lane leaves: sixteen share a block)
  const float mul = s.grad_mul ? *s.grad_mul : 1.f;
  bool skip = !(fabsf(mul) < INFINITY);
  if (s.step_at || s.lr_at) {
    const int64_t step = s.step_at ? *s.step_at : s.step;
    set_step(s, s.lr_at ? (double)*s.lr_at : s.lr, step);
    skip |= step < 1;
  }
  if (skip && same) return;   // uniform, as all of the above
  float g[8] = {}, p[8] = {}, m[8] = {}, v[8] = {};
  if (live) {
    load_values<DT>(a.tensor[k].grad, i, n, g);
    if constexpr (DT == 0) load_values<0>(a.tensor[k].param, i, n, p);
    else load_state(in.master, at, p);
    if constexpr (BITS == 32) {
      load_state((const float*)in.m, at, m);
      load_state((const float*)in.v, at, v);
    } else {
      decode(*(const u32x2*)((const char*)in.m + at), in.m_exp[at >> 7], m);
      decode(*(const u32x2*)((const char*)in.v + at), in.v_exp[at >> 7], v);
    }
  }
  if (skip) {
    if (!live) return;
    float q[8];
    load_values<DT>(a.tensor[k].param, i, n, q);
    store_values<DT>(a.tensor[k].param_out, i, n, q);
    if constexpr (DT != 0) store_state(out.master, at, p);
    if constexpr (BITS == 32) {
      store_state((float*)out.m, at, m);
      store_state((float*)out.v, at, v);
    } else {
      *(u32x2*)((char*)out.m + at) = *(const u32x2*)((const char*)in.m + at);
      *(u32x2*)((char*)out.v + at) = *(const u32x2*)((const char*)in.v + at);
      if ((threadIdx.x & 15) == 0) {
        out.m_exp[at >> 7] = in.m_exp[at >> 7];
        out.v_exp[at >> 7] = in.v_exp[at >> 7];
      }
    }
    return;
  }
  float root[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    if (i + j >= n) p[j] = m[j] = v[j] = 0.f;   // the padding has no part in its block's largest
    if constexpr (BITS == 8) v[j] *= v[j];
    advance(s, s.grad_mul ? g[j] * mul : g[j], p[j], m[j], v[j], root[j]);
  }
  u32x2 cm, cv;
  uint32_t em, ev;
  if constexpr (BITS == 8) {
    const uint32_t key = s.key ^ mix((uint32_t)(at >> 32));
    uint32_t low[8], high[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const uint32_t r = mix((uint32_t)at + j + key);
      low[j] = r & 0xffffu;
      high[j] = r >> 16;
    }
    cm = encode<false>(m, low, em);
    cv = encode<true>(root, high, ev);
  }
  if (!live) return;
  store_values<DT>(a.tensor[k].param_out, i, n, p);
  if constexpr (DT != 0) store_state(out.master, at, p);
  if constexpr (BITS == 32) {
    store_state((float*)out.m, at, m);
    store_state((float*)out.v, at, v);
  } else {
    *(u32x2*)((char*)out.m + at) = cm;
    *(u32x2*)((char*)out.v + at) = cv;
    if ((threadIdx.x & 15) == 0) {
      out.m_exp[at >> 7] = (uint8_t)em;
      out.v_exp[at >> 7] = (uint8_t)ev;
    }
  }
}

template <int DT, int BITS>
static hipError_t launch_adamw_of(hipStream_t st, int count, const jarq_adamw_tensor* tensors,
                                  const jarq_adamw_state& in, const jarq_adamw_state& out,
                                  const AdamScalars& s) {
  const int same = in.m == out.m;
  int64_t at = 0;
  AdamArgs a;
  int held = 0;
  int64_t units = 0;
  auto launch = [&]() {
    for (int k = held; k < kTensors; ++k) a.first[k] = 0xffffffffu;
    if (units > 0)
      hipLaunchKernelGGL((adamw_kernel<DT, BITS>), dim3((unsigned)units), dim3(256), 0, st, a, s,
                         in, out, same);
    held = 0;
    units = 0;
    return hipGetLastError();
  };
  for (int k = 0; k < count; ++k) {
    const jarq_adamw_tensor& t = tensors[k];
    if (t.numel == 0) continue;
    const int64_t most = (t.numel + kUnit - 1) / kUnit;
    if (t.grad == nullptr) {   // stays as it is
      at += (t.numel + 127) / 128 * 128;
      continue;
    }
    if (held == kTensors || units + most >= 1 << 24) {   // (fewer than 2^32 threads)
      const hipError_t e = launch();
      if (e != hipSuccess) return e;
    }
    a.tensor[held] = AdamTensor{t.grad, t.param, t.param_out, at, t.numel};
    a.first[held++] = (uint32_t)units;
    units += most;
    at += (t.numel + 127) / 128 * 128;
  }
  return launch();
}

hipError_t launch_adamw(hipStream_t st, int dtype, int bits, int count,
                        const jarq_adamw_tensor* tensors, const jarq_adamw_state& in,
                        const jarq_adamw_state& out, const jarq_adamw_options& o) {
  AdamScalars s{};
  s.b1 = (float)o.beta1;
  s.c1 = (float)(1.0 - o.beta1);
  s.b2 = (float)o.beta2;
  s.c2 = (float)(1.0 - o.beta2);
  s.eps = (float)o.eps;
  s.lr = o.lr;
  s.beta1 = o.beta1;
  s.beta2 = o.beta2;
  s.decay = o.weight_decay;
  s.seed = o.seed;
  s.step = o.step;
  s.lr_at = o.lr_at;
  s.grad_mul = o.grad_mul;
  s.step_at = o.step_at;
  set_step(s, o.lr, o.step);
  if (dtype == 0)
    return bits == 32 ? launch_adamw_of<0, 32>(st, count, tensors, in, out, s)
                      : launch_adamw_of<0, 8>(st, count, tensors, in, out, s);
  if (dtype == kF16)
    return bits == 32 ? launch_adamw_of<kF16, 32>(st, count, tensors, in, out, s)
                      : launch_adamw_of<kF16, 8>(st, count, tensors, in, out, s);
  return bits == 32 ? launch_adamw_of<kBF16, 32>(st, count, tensors, in, out, s)
                    : launch_adamw_of<kBF16, 8>(st, count, tensors, in, out, s);
}

}  // namespace jarq
