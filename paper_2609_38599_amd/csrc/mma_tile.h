// Tiles of C[j][i] = sum_k P[i][k] Q[j][k] on the matrix cores, for 16-bit floats
// (fp32 sums) and 8-bit integers (int32 sums).
//
// Both operands pass through LDS in chunks of 128 bytes of k (64 values of 16
// bits, 128 of 8), straight from memory (global_load_lds_dwordx4), one chunk
// ahead.  An operand lies in memory either with k along its rows (KContig) or
// with k down its rows (KStrided, 16 bits only: read out of LDS through the
// transposing read), so no product needs a transposed copy.
//
// 32 x 32 blocks per instruction.  In a result block a lane holds column
// j = lane % 32 and rows i = 8 (v / 4) + 4 (lane / 32) + v % 4, v = 0..15.
#pragma once

#include "bf16x3.h"

namespace jarq {

enum : int { kF16 = 1, kBF16 = 2, kI8 = 3 };   // 1, 2 as JARQ_F16, JARQ_BF16

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef int32_t i32x4 __attribute__((ext_vector_type(4)));
typedef int32_t i32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

template <int KIND> struct Mma;
template <> struct Mma<kBF16> {
  typedef f32x16 Acc;
  typedef f32x4 Acc16;
  static __device__ __forceinline__ Acc mul(const u32x4& a, const u32x4& b, const Acc& c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a),
                                                   __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  }
  static __device__ __forceinline__ Acc16 mul16(const u32x4& a, const u32x4& b, const Acc16& c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a),
                                                   __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  }
};
template <> struct Mma<kF16> {
  typedef f32x16 Acc;
  typedef f32x4 Acc16;
  static __device__ __forceinline__ Acc mul(const u32x4& a, const u32x4& b, const Acc& c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a),
                                                  __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
  }
  static __device__ __forceinline__ Acc16 mul16(const u32x4& a, const u32x4& b, const Acc16& c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a),
                                                  __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
  }
};
template <> struct Mma<kI8> {
  typedef i32x16 Acc;
  typedef i32x4 Acc16;
  static __device__ __forceinline__ Acc mul(const u32x4& a, const u32x4& b, const Acc& c) {
    return __builtin_amdgcn_mfma_i32_32x32x32_i8(__builtin_bit_cast(i32x4, a),
                                                 __builtin_bit_cast(i32x4, b), c, 0, 0, 0);
  }
  static __device__ __forceinline__ Acc16 mul16(const u32x4& a, const u32x4& b, const Acc16& c) {
    return __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(i32x4, a),
                                                 __builtin_bit_cast(i32x4, b), c, 0, 0, 0);
  }
};

// ---- 16-bit values ----
template <int KIND>
__device__ __forceinline__ uint16_t to16(float x) {
  if constexpr (KIND == kBF16) return __builtin_bit_cast(uint16_t, (__bf16)x);
  else return __builtin_bit_cast(uint16_t, (_Float16)x);
}
template <int KIND>
__device__ __forceinline__ float from16(uint16_t w) {
  if constexpr (KIND == kBF16) return __uint_as_float((uint32_t)w << 16);
  else return (float)__builtin_bit_cast(_Float16, w);
}
template <int KIND>
__device__ __forceinline__ uint32_t pack16(float lo, float hi) {
  return (uint32_t)to16<KIND>(lo) | ((uint32_t)to16<KIND>(hi) << 16);
}

constexpr int kChunk = 128;   // bytes of k per chunk and row

// What lanes past an operand's last k read.
static __device__ __attribute__((aligned(16))) const uint32_t kZeros[4] = {0, 0, 0, 0};

__device__ __forceinline__ void load_lds16(const void* from, char* to) {
  __builtin_amdgcn_global_load_lds(from, (__attribute__((address_space(3))) void*)to, 16, 0, 0);
}

// An operand tile of TR rows with k along the rows, staged by NW wavefronts.  A
// row's chunk is 8 pieces of 16 bytes; piece x of row r lies at x ^ (r % 8), so
// that the rows of a fragment read fall in distinct banks.  DUAL: the first
// half of the rows from one matrix, the second half from another.  Rows past
// the last read the last one (their results are not stored); k past the end
// reads zeros.
template <int TR, int NW, bool DUAL>
struct KContig {
  static constexpr int N = TR / 8 / NW;   // load instructions a wave (1 KB = 8 rows each)
  static_assert(N >= 1 && N * 8 * NW == TR && (!DUAL || N % 2 == 0), "tile");
  static constexpr int kBytes = TR * kChunk;
  const char *b0, *b1;
  uint32_t off[DUAL ? N / 2 : N];
  int kbytes, wave, piece;

  // p0, p1: the matrices' first rows; ld: bytes a row; row0 < rows: the tile's
  // first row (of each half); ld <= 2^22 so that offsets in a tile fit 32 bits.
  __device__ __forceinline__ void init(const void* p0, const void* p1, size_t ld, int row0,
                                       int rows, int kb, int w, int lane) {
    b0 = (const char*)p0 + (size_t)row0 * ld;
    b1 = DUAL ? (const char*)p1 + (size_t)row0 * ld : b0;
    kbytes = kb;
    wave = w;
    const int r = lane >> 3;
    piece = 16 * ((lane & 7) ^ r);
#pragma unroll
    for (int n = 0; n < (DUAL ? N / 2 : N); ++n)
      off[n] = (uint32_t)min(8 * (w + NW * n) + r, rows - 1 - row0) * (uint32_t)ld +
               (uint32_t)piece;
  }
  __device__ __forceinline__ void issue(int q, char* stage) const {
    const int k0 = q * kChunk;
    const bool in = k0 + kChunk <= kbytes;   // uniform
#pragma unroll
    for (int n = 0; n < N; ++n) {
      const bool second = DUAL && n >= N / 2;
      const char* at = (second ? b1 : b0) + k0 + off[second ? n - N / 2 : n];
      if (!in && k0 + piece >= kbytes) at = (const char*)kZeros;
      load_lds16(at, stage + 1024 * (wave + NW * n));
    }
  }
  // Fragment of the 32 rows from row0 (a multiple of 32), k-slice ks of 4.
  static __device__ __forceinline__ u32x4 frag(const char* stage, int row0, int ks, int lane) {
    const int x = (((lane >> 5) ^ (lane & 7)) << 4) ^ (ks << 5);
    return *(const u32x4*)(stage + (row0 + (lane & 31)) * kChunk + x);
  }
};

__device__ __forceinline__ s16x4 lds_read_tr16(const char* p) {
  return __builtin_amdgcn_ds_read_tr16_b64_v4i16(
      (__attribute__((address_space(3))) s16x4*)(const __attribute__((address_space(3))) void*)p);
}

// An operand tile of TR columns with k down the rows (16-bit values): a chunk is
// 64 rows of TR values.  64-byte block x of row t lies at x ^ (t % 4): a
// transposing read takes one block of four consecutive rows.  Rows sw.. come
// from a second matrix (sw = rows if there is none).  Columns past the last
// read the last eight; rows past the last read zeros.
template <int TR, int NW>
struct KStrided {
  static constexpr int RB = 2 * TR;             // bytes a row
  static constexpr int CPR = RB / 16;           // pieces a row
  static constexpr int RPP = 64 / CPR;          // rows per load instruction
  static constexpr int N = 64 / RPP / NW;
  static_assert(N >= 1 && N * RPP * NW == 64 && (NW * RPP) % 4 == 0, "tile");
  static constexpr int kBytes = TR * kChunk;
  const char *b0, *b1;
  size_t ld;
  uint32_t off;      // of this lane in the first instruction's rows
  int rows, sw, wave, lt;

  // c0: the tile's first column; cols a multiple of 8; ld bytes a row, at most 2^22.
  __device__ __forceinline__ void init(const void* p0, const void* p1, size_t ld_, int c0,
                                       int cols, int rows_, int sw_, int w, int lane) {
    ld = ld_;
    rows = rows_;
    sw = sw_;
    wave = w;
    lt = RPP * w + lane / CPR;
    const int pc = (lane % CPR) ^ ((lt & 3) << 2);
    const uint32_t col = 2u * (uint32_t)min(c0 + 8 * pc, cols - 8);
    b0 = (const char*)p0;
    b1 = (const char*)p1;
    off = col;
  }
  __device__ __forceinline__ void issue(int q, char* stage) const {
    const int k0 = q * 64;
    const bool one = k0 + 64 <= sw || (k0 >= sw && k0 + 64 <= rows);   // uniform
    if (one) {
      const char* base = k0 < sw ? b0 + (size_t)k0 * ld : b1 + (size_t)(k0 - sw) * ld;
#pragma unroll
      for (int n = 0; n < N; ++n)
        load_lds16(base + ((uint32_t)(lt + NW * RPP * n) * (uint32_t)ld + off),
                   stage + 1024 * (wave + NW * n));
    } else {
#pragma unroll 1
      for (int n = 0; n < N; ++n) {
        const int t = k0 + lt + NW * RPP * n;
        const char* at = t < sw ? b0 + (size_t)t * ld + off
                                : b1 + (size_t)(t - sw) * ld + off;
        if (t >= rows) at = (const char*)kZeros;
        load_lds16(at, stage + 1024 * (wave + NW * n));
      }
    }
  }
  static __device__ __forceinline__ u32x4 frag(const char* stage, int col0, int ks, int lane) {
    const int gi = lane >> 4, pi = lane & 15, t = pi >> 2;
    const char* p = stage + (8 * (gi >> 1) + t + 16 * ks) * RB +
                    (((col0 >> 5) ^ t) << 6) + 32 * (gi & 1) + 8 * (pi & 3);
    const s16x4 w[2] = {lds_read_tr16(p), lds_read_tr16(p + 4 * RB)};
    return __builtin_bit_cast(u32x4, w);
  }
};

// The products of one staged chunk.  A wave's blocks: P rows prow(a), Q rows
// qrow + 32 b.
template <int KIND, int BI, int BJ, class LP, class LQ, class PR>
__device__ __forceinline__ void mma_chunk(const char* cur, int lane, const PR& prow, int qrow,
                                          typename Mma<KIND>::Acc (&acc)[BI][BJ]) {
#pragma unroll
  for (int ks = 0; ks < 4; ++ks) {
    u32x4 fp[BI], fq[BJ];
#pragma unroll
    for (int a = 0; a < BI; ++a) fp[a] = LP::frag(cur, prow(a), ks, lane);
#pragma unroll
    for (int b = 0; b < BJ; ++b) fq[b] = LQ::frag(cur + LP::kBytes, qrow + 32 * b, ks, lane);
#pragma unroll
    for (int a = 0; a < BI; ++a)
#pragma unroll
      for (int b = 0; b < BJ; ++b) acc[a][b] = Mma<KIND>::mul(fp[a], fq[b], acc[a][b]);
  }
}

// The k-loop over chunks q0 <= q < q1 (at least one): compute(stage, q) with chunk q
// staged, the next one's loads in flight.
template <class LP, class LQ, class Compute>
__device__ __forceinline__ void mma_loop(const LP& lp, const LQ& lq, int q0, int q1, char* buf0,
                                         char* buf1, const Compute& compute) {
  auto issue = [&](int q, char* stage) __attribute__((always_inline)) {
    lp.issue(q, stage);
    lq.issue(q, stage + LP::kBytes);
  };
  issue(q0, buf0);
  __syncthreads();
  for (int q = q0; q < q1; q += 2) {
    // a stage was last read before the barrier that precedes its loads; the
    // barrier after a chunk waits for the next one's loads
    if (q + 1 < q1) issue(q + 1, buf1);
    compute(buf0, q);
    __syncthreads();
    if (q + 1 < q1) {
      if (q + 2 < q1) issue(q + 2, buf0);
      compute(buf1, q + 1);
      __syncthreads();
    }
  }
}

// Tile (ti, tj) of work-group `id` in a grid of ni x nj tiles: the work-groups
// that one XCD gets (every eighth) take neighbouring tiles, in strips of eight
// along j, so that what they share stays in that XCD's L2.
__device__ __forceinline__ void xcd_tile(int id, int ni, int nj, int& ti, int& tj) {
  const int total = ni * nj, x = id & 7, at = id >> 3;
  const int each = total >> 3, more = total & 7;   // the first `more` XCDs get one more
  const int t = x * each + min(x, more) + at;
  const int strip = t / (8 * ni), in = t - strip * 8 * ni;
  const int w = min(8, nj - 8 * strip);
  ti = in / w;
  tj = 8 * strip + in - ti * w;
}

}  // namespace jarq
