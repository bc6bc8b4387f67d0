// Log probabilities of given tokens, entropies and top alternatives of rows of
// logits, and the gradient of the logits.
//
// With m = max x, z = sum exp(x - m): lse = m + log z, log p_v = x_v - lse and
// H = log z - sum exp(x - m) (x - m) / z, all from one pass that keeps (m, z, sum
// exp(x - m) (x - m)) per lane and rescales when m grows.
//
// A row in which any entry is +infinity or NaN gives NaN (and index -1); entries
// of -infinity have probability 0; a row of nothing else has lse = -infinity.
#include <float.h>

#include "mma_tile.h"

namespace jarq {

namespace {

typedef unsigned long long u64;

template <int DT> struct Elem { typedef uint16_t T; static constexpr int kVec = 8; };
template <> struct Elem<0> { typedef float T; static constexpr int kVec = 4; };

template <int DT>
__device__ __forceinline__ float value(typename Elem<DT>::T w) {
  if constexpr (DT == 0) return w;
  else return from16<DT>(w);
}
template <int DT>
__device__ __forceinline__ void unpack(const u32x4& w, float (&x)[Elem<DT>::kVec]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (DT == 0) {
      x[i] = __uint_as_float(w[i]);
    } else {
      x[2 * i] = from16<DT>((uint16_t)w[i]);
      x[2 * i + 1] = from16<DT>((uint16_t)(w[i] >> 16));
    }
  }
}
// fp32 logits: exp to an ulp; 16-bit ones: t log2 e rounded, off by |t| 2^-24
template <int DT>
__device__ __forceinline__ float exp_of(float t) {
  if constexpr (DT == 0) return expf(t);
  else return __expf(t);
}

// The running maximum (at least -FLT_MAX, so that x - m is never -inf + inf), sum
// and weighted sum.
struct Soft {
  float m, z, zt;
};
__device__ __forceinline__ Soft no_entries() { return Soft{-FLT_MAX, 0.f, 0.f}; }
// Keeps exp's argument within range for the weighted sum: exp is 0 there.
constexpr float kLeast = -1000.f;

template <int DT, int N>
__device__ __forceinline__ void add(Soft& s, const float (&x)[N]) {
  float m = s.m;
#pragma unroll
  for (int i = 0; i < N; ++i) m = fmaxf(m, x[i]);
  if (m > s.m) {
    const float t = s.m - m, e = exp_of<DT>(t);
    s.zt = e * (s.zt + s.z * fmaxf(t, kLeast));
    s.z *= e;
    s.m = m;
  }
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const float t = x[i] - m, e = exp_of<DT>(t);
    s.z += e;
    s.zt = fmaf(e, fmaxf(t, kLeast), s.zt);
  }
}
__device__ __forceinline__ void join(Soft& s, const Soft& o) {
  const float m = fmaxf(s.m, o.m);
  const float ta = s.m - m, tb = o.m - m, ea = expf(ta), eb = expf(tb);
  s.zt = ea * (s.zt + s.z * fmaxf(ta, kLeast)) + eb * (o.zt + o.z * fmaxf(tb, kLeast));
  s.z = ea * s.z + eb * o.z;
  s.m = m;
}

// Orders by value, then by the lowest index; -0 counts as 0.
__device__ __forceinline__ u64 top_key(float x, uint32_t index) {
  const uint32_t b = __float_as_uint(x + 0.f);
  const uint32_t o = b & 0x80000000u ? ~b : b | 0x80000000u;
  return ((u64)o << 32) | (0xffffffffu - index);
}
__device__ __forceinline__ float key_value(u64 k) {
  const uint32_t o = (uint32_t)(k >> 32);
  return __uint_as_float(o & 0x80000000u ? o & 0x7fffffffu : ~o);
}
__device__ __forceinline__ uint32_t key_index(u64 k) { return 0xffffffffu - (uint32_t)k; }

__device__ __forceinline__ u64 wave_max(u64 k) {
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) {
    const u64 o = __shfl_xor(k, off);
    k = o > k ? o : k;
  }
  return k;
}

struct RowOut {
  float *logprob, *entropy, *lse, *top_logprob;
  int32_t* top_index;
};

// log p = (x - m) - log z: closer than x - lse where one entry takes nearly all.
__device__ __forceinline__ float log_p(float x, const Soft& s, float lz) {
  return s.z == 0.f ? -INFINITY : (x - s.m) - lz;
}

// One thread: the row's results from its sums, lz = log z.
template <int DT>
__device__ __forceinline__ void finish_row(const Soft& s, const void* row, int64_t target, int V,
                                           size_t t, float lz, const RowOut& o) {
  float lp = 0.f;
  if (target >= V) lp = __uint_as_float(0x7fc00000u);
  else if (target >= 0) lp = log_p(value<DT>(((const typename Elem<DT>::T*)row)[target]), s, lz);
  o.logprob[t] = lp;
  if (o.entropy) o.entropy[t] = s.z == 0.f ? 0.f : lz - s.zt / s.z;
  if (o.lse) o.lse[t] = s.z == 0.f ? -INFINITY : s.m + lz;
}
__device__ __forceinline__ void store_top(const RowOut& o, size_t at, u64 key, const Soft& s,
                                          float lz) {
  const bool bad = s.z != s.z;
  o.top_index[at] = bad ? -1 : (int32_t)key_index(key);
  o.top_logprob[at] = bad ? s.z : log_p(key_value(key), s, lz);
}

}  // namespace

// Work-group `id`: part id % splits (of `each` entries) of row id / splits.  With one
// part it finishes the row; otherwise its sums and top keys go to the workspace.
template <int DT>
__global__ __launch_bounds__(256) void logprob_kernel(const void* __restrict__ logits, size_t ld,
                                                      int V, const int64_t* __restrict__ targets,
                                                      int splits, int each, int top, RowOut out,
                                                      float* __restrict__ psum,
                                                      u64* __restrict__ pkey) {
  typedef typename Elem<DT>::T E;
  constexpr int VE = Elem<DT>::kVec;
  __shared__ Soft red[4];
  __shared__ u64 best[4];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const size_t t = blockIdx.x / (unsigned)splits;
  const int part = blockIdx.x % (unsigned)splits;
  const E* row = (const E*)logits + t * ld;
  const int b = part * each, e = min(V, b + each);
  // scalars up to the first 16-byte boundary, vectors, scalars
  const int head = min(e - b, (int)((16 - (uintptr_t)(row + b) % 16) % 16 / sizeof(E)));
  const int nv = (e - b - head) / VE, rest = b + head + nv * VE;
  const u32x4* vec = (const u32x4*)(row + b + head);
  const int own = tid < head ? b + tid : rest + tid - head;   // this thread's scalar, if any
  const bool has = tid < head || own < e;
  Soft s = no_entries();
  if (has) {
    const float x[1] = {value<DT>(row[own])};
    add<DT>(s, x);
  }
  for (int v = tid; v < nv; v += 256) {
    float x[VE];
    unpack<DT>(vec[v], x);
    add<DT>(s, x);
  }
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) {
    Soft o;
    o.m = __shfl_xor(s.m, off);
    o.z = __shfl_xor(s.z, off);
    o.zt = __shfl_xor(s.zt, off);
    join(s, o);
  }
  if (lane == 0) red[wave] = s;
  __syncthreads();
  s = red[0];
#pragma unroll
  for (int w = 1; w < 4; ++w) join(s, red[w]);
  const float lz = logf(s.z);
  if (splits == 1) {
    if (tid == 0) finish_row<DT>(s, row, targets[t], V, t, lz, out);
  } else if (tid == 0) {
    float* p = psum + 3 * (size_t)blockIdx.x;
    p[0] = s.m;
    p[1] = s.z;
    p[2] = s.zt;
  }
  u64 last = ~0ull;
  for (int k = 0; k < top; ++k) {
    u64 mine = 0;
    auto look = [&](float x, int i) {
      const u64 key = top_key(x, (uint32_t)i);
      if (key < last && key > mine) mine = key;
    };
    if (has) look(value<DT>(row[own]), own);
    for (int v = tid; v < nv; v += 256) {
      float x[VE];
      unpack<DT>(vec[v], x);
#pragma unroll
      for (int i = 0; i < VE; ++i) look(x[i], b + head + v * VE + i);
    }
    mine = wave_max(mine);
    if (lane == 0) best[wave] = mine;
    __syncthreads();
    last = best[0];
#pragma unroll
    for (int w = 1; w < 4; ++w) last = best[w] > last ? best[w] : last;
    __syncthreads();
    if (tid == 0) {
      if (splits == 1) store_top(out, t * top + k, last, s, lz);
      else pkey[(size_t)blockIdx.x * top + k] = last;   // 0 where the part has fewer entries
    }
  }
}

// A work-group a row: its parts' sums in order, the top of their keys.
template <int DT>
__global__ __launch_bounds__(256) void logprob_join_kernel(
    const void* __restrict__ logits, size_t ld, int V, const int64_t* __restrict__ targets,
    int splits, int top, RowOut out, const float* __restrict__ psum,
    const u64* __restrict__ pkey) {
  typedef typename Elem<DT>::T E;
  __shared__ u64 best[4];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const size_t t = blockIdx.x;
  Soft s = no_entries();
  for (int p = 0; p < splits; ++p) {
    const float* q = psum + 3 * (t * splits + p);
    Soft o;
    o.m = q[0];
    o.z = q[1];
    o.zt = q[2];
    join(s, o);
  }
  const float lz = logf(s.z);
  if (tid == 0) finish_row<DT>(s, (const E*)logits + t * ld, targets[t], V, t, lz, out);
  u64 last = ~0ull;
  const u64* keys = pkey + t * splits * top;
  for (int k = 0; k < top; ++k) {
    u64 mine = 0;
    for (int i = tid; i < splits * top; i += 256) {
      const u64 key = keys[i];
      if (key < last && key > mine) mine = key;
    }
    mine = wave_max(mine);
    if (lane == 0) best[wave] = mine;
    __syncthreads();
    last = best[0];
#pragma unroll
    for (int w = 1; w < 4; ++w) last = best[w] > last ? best[w] : last;
    __syncthreads();
    if (tid == 0) store_top(out, t * top + k, last, s, lz);
  }
}

// ---- gradient ----
// d x_v = g (onehot - p) - h p (log p + H), g and h the gradients of the log
// probability and of the entropy.  Work-group `id`: part id % splits of a row.  A
// thread reads each entry before it writes it: dlogits may be the logits.
template <int DT>
__global__ __launch_bounds__(256) void logprob_grad_kernel(
    const void* logits, size_t ld, int V, const int64_t* __restrict__ targets,
    const float* __restrict__ lse_of, const float* __restrict__ entropy,
    const float* __restrict__ dlp, const float* __restrict__ dent, int splits, int each,
    void* dlogits, size_t ldd) {
  typedef typename Elem<DT>::T E;
  constexpr int VE = Elem<DT>::kVec;
  const int tid = threadIdx.x;
  const size_t t = blockIdx.x / (unsigned)splits;
  const int b = (int)(blockIdx.x % (unsigned)splits) * each, e = min(V, b + each);
  const E* row = (const E*)logits + t * ld;
  E* drow = (E*)dlogits + t * ldd;
  const float lse = lse_of[t];
  const int64_t target = targets[t];
  const float g = target < 0 ? 0.f : target >= V ? __uint_as_float(0x7fc00000u) : dlp[t];
  const float h = dent ? dent[t] : 0.f;
  const float ent = dent ? entropy[t] : 0.f;
  const bool empty = lse == -INFINITY;   // nothing but -infinity: no gradient
  auto grad = [&](float x, int64_t v) __attribute__((always_inline)) {
    const float t = x - lse, p = exp_of<DT>(t);
    const float c = p * (g + h * (fmaxf(t, kLeast) + ent));
    return empty ? 0.f : (v == target ? g - c : -c);
  };
  auto word = [](float x) __attribute__((always_inline)) -> E {
    if constexpr (DT == 0) return x;
    else return to16<DT>(x);
  };
  const uintptr_t ax = (uintptr_t)(row + b) % 16, ad = (uintptr_t)(drow + b) % 16;
  if (ax != ad) {   // uniform
    for (int v = b + tid; v < e; v += 256) drow[v] = word(grad(value<DT>(row[v]), v));
    return;
  }
  const int head = min(e - b, (int)((16 - ax) % 16 / sizeof(E)));
  const int nv = (e - b - head) / VE, rest = b + head + nv * VE;
  const int own = tid < head ? b + tid : rest + tid - head;
  if (tid < head || own < e) drow[own] = word(grad(value<DT>(row[own]), own));
  const u32x4* vec = (const u32x4*)(row + b + head);
  u32x4* dvec = (u32x4*)(drow + b + head);
  for (int v = tid; v < nv; v += 256) {
    float x[VE];
    unpack<DT>(vec[v], x);
    const int v0 = b + head + v * VE;
    u32x4 w;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (DT == 0) w[i] = __float_as_uint(grad(x[i], v0 + i));
      else w[i] = pack16<DT>(grad(x[2 * i], v0 + 2 * i), grad(x[2 * i + 1], v0 + 2 * i + 1));
    }
    dvec[v] = w;
  }
}

namespace {

// Parts a row is cut into: few rows alone would leave CUs idle.
struct LogprobPlan {
  int splits, each;
};
LogprobPlan logprob_plan(int T, int V) {
  LogprobPlan p;
  int splits = 512 / T;
  const int most = V / 4096;
  splits = splits < 1 || most < 1 ? 1 : splits > most ? most : splits;
  if (splits > 64) splits = 64;
  p.each = ((V + splits - 1) / splits + 63) / 64 * 64;
  p.splits = (V + p.each - 1) / p.each;
  return p;
}

template <int DT>
hipError_t logprob_kind(hipStream_t st, const void* logits, size_t ld, int T, int V,
                        const int64_t* targets, int top, const RowOut& out, char* ws) {
  const LogprobPlan p = logprob_plan(T, V);
  u64* pkey = (u64*)ws;
  float* psum = (float*)(ws + 8 * (size_t)T * p.splits * top);
  hipLaunchKernelGGL((logprob_kernel<DT>), dim3((unsigned)(T * p.splits)), dim3(256), 0, st,
                     logits, ld, V, targets, p.splits, p.each, top, out, psum, pkey);
  if (p.splits > 1) {
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((logprob_join_kernel<DT>), dim3((unsigned)T), dim3(256), 0, st, logits, ld,
                       V, targets, p.splits, top, out, psum, pkey);
  }
  return hipGetLastError();
}

template <int DT>
hipError_t logprob_grad_kind(hipStream_t st, const void* logits, size_t ld, int T, int V,
                             const int64_t* targets, const float* lse, const float* entropy,
                             const float* dlp, const float* dent, void* dlogits, size_t ldd) {
  const LogprobPlan p = logprob_plan(T, V);
  hipLaunchKernelGGL((logprob_grad_kernel<DT>), dim3((unsigned)(T * p.splits)), dim3(256), 0, st,
                     logits, ld, V, targets, lse, entropy, dlp, dent, p.splits, p.each, dlogits,
                     ldd);
  return hipGetLastError();
}

}  // namespace

size_t logprob_workspace_bytes(int T, int V, int top) {
  const LogprobPlan p = logprob_plan(T, V);
  return p.splits == 1 ? 0 : (size_t)T * p.splits * (8 * (size_t)top + 12);
}

hipError_t launch_token_logprobs(hipStream_t st, int dtype, const void* logits, size_t ld, int T,
                                 int V, const int64_t* targets, int top, float* logprob,
                                 float* entropy, float* lse, int32_t* top_index,
                                 float* top_logprob, char* ws) {
  const RowOut out{logprob, entropy, lse, top_logprob, top_index};
  if (dtype == 0) return logprob_kind<0>(st, logits, ld, T, V, targets, top, out, ws);
  if (dtype == kF16) return logprob_kind<kF16>(st, logits, ld, T, V, targets, top, out, ws);
  return logprob_kind<kBF16>(st, logits, ld, T, V, targets, top, out, ws);
}

hipError_t launch_token_logprobs_backward(hipStream_t st, int dtype, const void* logits, size_t ld,
                                          int T, int V, const int64_t* targets, const float* lse,
                                          const float* entropy, const float* dlp,
                                          const float* dent, void* dlogits, size_t ldd) {
  if (dtype == 0)
    return logprob_grad_kind<0>(st, logits, ld, T, V, targets, lse, entropy, dlp, dent, dlogits,
                                ldd);
  if (dtype == kF16)
    return logprob_grad_kind<kF16>(st, logits, ld, T, V, targets, lse, entropy, dlp, dent, dlogits,
                                   ldd);
  return logprob_grad_kind<kBF16>(st, logits, ld, T, V, targets, lse, entropy, dlp, dent, dlogits,
                                  ldd);
}

}  // namespace jarq
