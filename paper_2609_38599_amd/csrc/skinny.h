// Products with few rows: sum_k P[i][k] Q[j][k] for IB x 16 rows i (tokens) and
// JB x 16 rows j (channels), the k-range dealt to the work-group's wavefronts.
// Bound by reading Q once; a wavefront's fragments go from memory to registers (a
// lane holds 16 bytes of row lane % 16 at 16 (lane / 16) of each 64 bytes of k).
#pragma once

#include "mma_tile.h"

namespace jarq {

// k in units of U steps of 64 bytes; wavefront w takes units w, w + NW, ...  p, q:
// this lane's row pointers.  extra(unit, set) may load more for a unit into set 0 or 1
// of its own; step(s, set, fp, fq) gets the fragments of each step.
template <int IB, int JB, int U, int NW, class Extra, class Step>
__device__ __forceinline__ void skinny_loop(const char* const (&p)[IB], const char* const (&q)[JB],
                                            int kbytes, int wave, int lane, const Extra& extra,
                                            const Step& step) {
  const int at = 16 * (lane >> 4);
  const int units = (kbytes + 64 * U - 1) / (64 * U);
  u32x4 fp[2][U][IB], fq[2][U][JB];
  auto load = [&](int u, int set) __attribute__((always_inline)) {
    const int k0 = u * 64 * U;
    extra(u, set);
    if (k0 + 64 * U <= kbytes) {   // uniform
#pragma unroll
      for (int s = 0; s < U; ++s) {
#pragma unroll
        for (int b = 0; b < JB; ++b) fq[set][s][b] = *(const u32x4*)(q[b] + k0 + 64 * s + at);
#pragma unroll
        for (int a = 0; a < IB; ++a) fp[set][s][a] = *(const u32x4*)(p[a] + k0 + 64 * s + at);
      }
    } else {                       // k past the end is 0
#pragma unroll
      for (int s = 0; s < U; ++s) {
        const int k = k0 + 64 * s + at;
#pragma unroll
        for (int b = 0; b < JB; ++b) fq[set][s][b] = k < kbytes ? *(const u32x4*)(q[b] + k) : u32x4{};
#pragma unroll
        for (int a = 0; a < IB; ++a) fp[set][s][a] = k < kbytes ? *(const u32x4*)(p[a] + k) : u32x4{};
      }
    }
  };
  auto mul = [&](int set) __attribute__((always_inline)) {
#pragma unroll
    for (int s = 0; s < U; ++s) step(s, set, fp[set][s], fq[set][s]);
  };
  if (wave < units) load(wave, 0);
  for (int u = wave; u < units; u += 2 * NW) {
    if (u + NW < units) load(u + NW, 1);
    mul(0);
    if (u + NW < units) {
      if (u + 2 * NW < units) load(u + 2 * NW, 0);
      mul(1);
    }
  }
}

// Sum over the NW wavefronts' parts in LDS (in order) of entry (i, j) of block b:
// a part is [block][lane][4], lane = 16 (i / 4) + j, component i % 4.
template <int NW, int BLOCKS, class T>
__device__ __forceinline__ T skinny_sum(const T* red, int b, int i, int j) {
  const T* at = red + (b * 64 + (i >> 2) * 16 + j) * 4 + (i & 3);
  T s = at[0];
#pragma unroll
  for (int w = 1; w < NW; ++w) s += at[w * BLOCKS * 256];
  return s;
}

}  // namespace jarq
