// Tiles of C[j][i] = sum_k P[i][k] Q[j][k] on the matrix cores, for 16-bit floats
// (fp32 sums) and 8-bit integers (int32 sums).
//
// Both operands pass through LDS in chunks of 64 bytes of k (32 values of 16
// bits, 64 of 8), straight from memory (buffer_load_dwordx4 .. lds), three chunks
// ahead.  An operand lies in memory either with k along its rows (KContig) or
// with k down its rows (KStrided, 16 bits only: read out of LDS through the
// transposing read), so no product needs a transposed copy.
//
// 16 x 16 blocks per instruction, 64 bytes of k each (v_mfma_f32_16x16x32_bf16 and the
// like; 32 x 32 blocks take 5 % longer, at the clock that the card's power then allows).
// A lane's operand is 16 bytes of row lane % 16, at 16 (lane / 16); in a result block
// it holds column j = lane % 16 and rows i = 4 (lane / 16) + v, v = 0..3.
#pragma once

#include <algorithm>

#include "bf16x3.h"

namespace jarq {

enum : int { kF16 = 1, kBF16 = 2, kI8 = 3 };   // 1, 2 as JARQ_F16, JARQ_BF16

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef int32_t i32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

template <int KIND> struct Mma;
template <> struct Mma<kBF16> {
  typedef f32x4 Acc;
  static __device__ __forceinline__ Acc mul(const u32x4& a, const u32x4& b, const Acc& c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a),
                                                   __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  }
};
template <> struct Mma<kF16> {
  typedef f32x4 Acc;
  static __device__ __forceinline__ Acc mul(const u32x4& a, const u32x4& b, const Acc& c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a),
                                                  __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
  }
};
template <> struct Mma<kI8> {
  typedef i32x4 Acc;
  static __device__ __forceinline__ Acc mul(const u32x4& a, const u32x4& b, const Acc& c) {
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

constexpr int kChunk = 64;   // bytes of k per chunk and row

// A buffer of memory from `from` (uniform) on; loads at offsets of kNowhere return 0.
typedef __amdgpu_buffer_rsrc_t Buffer;
constexpr uint32_t kNowhere = 0x80000000u;
__device__ __forceinline__ Buffer buffer_at(const void* from, size_t bytes) {
  const uint32_t n = bytes < 0x7fffffffu ? (uint32_t)bytes : 0x7fffffffu;
  return __builtin_amdgcn_make_buffer_rsrc((void*)from, 0, (int)n, 0x00020000);
}
// 16 bytes a lane from `at` + base into LDS, lane after lane.  (A load by buffer, not
// by address: the compiler takes one by address for a possible LDS access and then
// waits for every LDS read in flight at the next use of any.)
__device__ __forceinline__ void load_lds16(Buffer from, uint32_t at, uint32_t base, char* to) {
  __builtin_amdgcn_raw_ptr_buffer_load_lds(from, (__attribute__((address_space(3))) void*)to, 16,
                                           (int)at, (int)base, 0, 0);
}

// An operand tile of TR rows with k along the rows, staged by NW wavefronts.  A
// row's chunk is CPR pieces of 16 bytes; the pieces of a row are permuted by the row
// so that 16 rows' same piece, which a fragment read takes at a time, fall in
// distinct banks (64 banks of 4 bytes).  Rows past the last read the last one (their
// results are not stored); k past the end reads zeros.
// kOne: one matrix.  kRowHalves: the first half of the rows from one matrix, the
// second half from another.  kTwoSpans: k runs through one matrix's columns, then
// through another's (each in chunks of its own).
enum Sources { kOne, kRowHalves, kTwoSpans };
template <int TR, int NW, Sources SRC>
struct KContig {
  static constexpr int CPR = kChunk / 16;      // pieces a row
  static constexpr int RPI = 64 / CPR;         // rows per load instruction (1 KB)
  static constexpr int N = TR / RPI / NW;      // load instructions a wave
  static constexpr bool HALVES = SRC == kRowHalves;
  static constexpr int NO = HALVES ? N / 2 : N;
  static_assert(N >= 1 && N * RPI * NW == TR && (!HALVES || N % 2 == 0), "tile");
  static constexpr int kBytes = TR * kChunk;
  Buffer b0, b1;
  uint32_t off[NO];
  int kbytes, wave, piece;

  static __device__ __forceinline__ int swz(int row) { return (row >> 2) & 3; }
  // p0, p1: the matrices' first rows; ld: bytes a row; kb: bytes of k (of a span);
  // row0 < rows: the tile's first row (of each half); ld <= 2^22 so that offsets in a
  // tile fit 32 bits.
  __device__ __forceinline__ void init(const void* p0, const void* p1, size_t ld, int row0,
                                       int rows, int kb, int w, int lane) {
    const size_t skip = (size_t)row0 * ld, bytes = (size_t)(rows - row0 - 1) * ld + kb;
    b0 = buffer_at((const char*)p0 + skip, bytes);
    b1 = SRC == kOne ? b0 : buffer_at((const char*)p1 + skip, bytes);
    kbytes = kb;
    wave = w;
    const int r = RPI * w + lane / CPR;
    piece = 16 * ((lane % CPR) ^ swz(r));
#pragma unroll
    for (int n = 0; n < NO; ++n)
      off[n] = (uint32_t)min(RPI * NW * n + r, rows - 1 - row0) * (uint32_t)ld + (uint32_t)piece;
  }
  // A chunk's start in its span, past every span where it is not `live`.
  struct Chunk {
    int k0;
    bool second;
  };
  __device__ __forceinline__ Chunk chunk(int q, bool live) const {
    const int span = (kbytes + kChunk - 1) / kChunk;
    const bool second = SRC == kTwoSpans && q >= span;
    return {live ? (second ? q - span : q) * kChunk : kbytes, second};
  }
  // Load instruction n of a chunk.
  __device__ __forceinline__ void issue(const Chunk& c, int n, char* stage) const {
    const bool from1 = HALVES ? n >= N / 2 : c.second;
    load_lds16(from1 ? b1 : b0, c.k0 + piece < kbytes ? off[HALVES && from1 ? n - N / 2 : n] : kNowhere,
               (uint32_t)c.k0, stage + 1024 * (wave + NW * n));
  }
  // This lane's place in a stage for a wave whose B blocks of 16 rows start at row0 (in
  // each half, where there are two).
  template <int B>
  struct Lane {
    uint32_t o;
    __device__ __forceinline__ Lane(int row0, int lane) {
      o = (uint32_t)(row0 + (lane & 15)) * kChunk +
          ((uint32_t)((lane >> 4) ^ swz(lane & 15)) << 4);
    }
    // Fragment of block a.
    __device__ __forceinline__ u32x4 frag(const char* stage, int a) const {
      const int row = HALVES && a >= B / 2 ? TR / 2 + 16 * (a - B / 2) : 16 * a;
      return *(const u32x4*)(stage + o + row * kChunk);
    }
  };
};

__device__ __forceinline__ s16x4 lds_read_tr16(const char* p) {
  return __builtin_amdgcn_ds_read_tr16_b64_v4i16(
      (__attribute__((address_space(3))) s16x4*)(const __attribute__((address_space(3))) void*)p);
}

// An operand tile of TR columns with k down the rows (16-bit values): a chunk is
// kRows rows of TR values.  64-byte block x of row t lies at x ^ swz(t), its 32-byte
// halves exchanged in every other eight rows: the transposing reads of half a wave take 32
// bytes of four consecutive rows and of the four rows eight further down.  Columns past the last
// read the last eight; rows past the last read zeros.  kTwoSpans: k runs down one
// matrix, then down another.
template <int TR, int NW, Sources SRC>
struct KStrided {
  static_assert(SRC != kRowHalves, "sources");
  static constexpr int kRows = kChunk / 2;
  static constexpr int RB = 2 * TR;             // bytes a row
  static constexpr int CPR = RB / 16;           // pieces a row
  static constexpr int RPI = 64 / CPR;          // rows per load instruction
  static constexpr int N = kRows / RPI / NW;
  static_assert(N >= 1 && N * RPI * NW == kRows && (NW * RPI) % 16 == 0, "tile");
  static_assert(TR >= 64, "a row has two 64-byte blocks at least");
  static constexpr int kBytes = TR * kChunk;
  static __device__ __forceinline__ int swz(int t) { return TR >= 128 ? t & 3 : (t >> 1) & 1; }
  const char *b0, *b1;
  size_t ld;
  uint32_t off[N];
  int rows, wave, lt;

  // c0: the tile's first column; cols a multiple of 8; ld bytes a row, at most 2^22;
  // rows_ of a span.
  __device__ __forceinline__ void init(const void* p0, const void* p1, size_t ld_, int c0,
                                       int cols, int rows_, int w, int lane) {
    ld = ld_;
    rows = rows_;
    wave = w;
    lt = RPI * w + lane / CPR;
    const int pc = (lane % CPR) ^ (swz(lt) << 2) ^ ((lt >> 2) & 2);
    b0 = (const char*)p0;
    b1 = (const char*)p1;
#pragma unroll
    for (int n = 0; n < N; ++n)
      off[n] = (uint32_t)(lt + NW * RPI * n) * (uint32_t)ld + 2u * (uint32_t)min(c0 + 8 * pc, cols - 8);
  }
  struct Chunk {
    Buffer from;
    int left;   // rows from its first one on
  };
  __device__ __forceinline__ Chunk chunk(int q, bool live) const {
    const int span = (rows + kRows - 1) / kRows;
    const bool second = SRC == kTwoSpans && q >= span;
    const int k0 = (second ? q - span : q) * kRows;
    return {buffer_at((second ? b1 : b0) + (live ? (size_t)k0 * ld : 0), 0x7fffffff),
            live ? rows - k0 : 0};
  }
  __device__ __forceinline__ void issue(const Chunk& c, int n, char* stage) const {
    load_lds16(c.from, lt + NW * RPI * n < c.left ? off[n] : kNowhere, 0,
               stage + 1024 * (wave + NW * n));
  }
  template <int B>
  struct Lane {
    uint32_t o[B];
    __device__ __forceinline__ Lane(int col0, int lane) {
      const int gi = lane >> 4, pi = lane & 15, t = pi >> 2;
#pragma unroll
      for (int a = 0; a < B; ++a) {
        const int c = (col0 >> 4) + a;   // of 16 columns
        o[a] = (uint32_t)((8 * gi + t) * RB + (((c >> 1) ^ swz(t)) << 6) +
                          (((c ^ gi) & 1) << 5) + 8 * (pi & 3));
      }
    }
    __device__ __forceinline__ u32x4 frag(const char* stage, int a) const {
      const char* p = stage + o[a];
      const s16x4 w[2] = {lds_read_tr16(p), lds_read_tr16(p + 4 * RB)};
      return __builtin_bit_cast(u32x4, w);
    }
  };
};

// Waits until at most n of this wave's loads are outstanding and its LDS accesses
// are done, then for the work-group's other waves.
template <int n>
__device__ __forceinline__ void wait_barrier() {
  __builtin_amdgcn_sched_barrier(0);
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt((n & 15) | (7 << 4) | ((n >> 4) << 14));
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
  __builtin_amdgcn_sched_barrier(0);
}

// At least n waves on a SIMD.  With two a wave has no more than 256 registers, and the
// compiler leaves the sums where the vector units reach them (37 tokens, 4096 -> 11008 in 8
// bits, groups of 128: 18.2 us, 19.5 without; 611 x 1000 -> 2752 forward and backward 60.1 and
// 61.6; the large tiles the same).
#define JARQ_WAVES(n) __attribute__((amdgpu_waves_per_eu(n)))

// The S stages of a work-group, `bytes` each: arrays of their own, so that the
// compiler can tell which of them a load in flight writes.
#define JARQ_STAGES(S, bytes)                                                     \
  __shared__ __attribute__((aligned(1024))) char stage0[bytes], stage1[bytes],    \
      stage2[bytes], stage3[bytes];                                               \
  __shared__ __attribute__((aligned(16))) char stage4[S > 4 ? (bytes) : 16],      \
      stage5[S > 4 ? (bytes) : 16], stage6[S > 4 ? (bytes) : 16],                 \
      stage7[S > 4 ? (bytes) : 16];                                               \
  char* const stages[8] = {stage0, stage1, stage2, stage3, stage4, stage5, stage6, stage7}

// The k-loop over chunks q0 <= q < q1 (at least one) with S stages: while a chunk is
// multiplied, the loads of the S - 1 behind it are in flight, and fragments are read half
// a chunk's products ahead.  The loop runs in whole rounds of the stages (chunks past the
// last are zeros).  A wave's BI blocks of P start at row prow of the tile, its BJ of Q
// at qrow.  round(q) comes before each round (loads of its own make the next wait stricter,
// never laxer); mul(p, q, a, b, i) gets the fragments of P block a and Q block b of chunk i of
// the round.
//
// 4096 x 4096 -> 2 x 14336 channels, 256-wide tiles, compared with each other (780 us with
// the code as it is): two stages of twice the chunk 812 us, four 800; the loads in a row at the
// start of a chunk 860; by address instead of by buffer (every LDS read then waits for all
// others) 905.  Bound by the matrix cores at
// the clock that the card's power allows (1.4 to 1.7 GHz here).
template <int S, int BI, int BJ, class LP, class LQ, class Round, class Mul>
__device__ __forceinline__ void mma_loop(const LP& lp, const LQ& lq, int q0, int q1, int lane,
                                         int prow, int qrow, char* const (&stages)[8],
                                         const Round& round, const Mul& mul) {
  // the products in two halves of P blocks; what is read during the first is the
  // second half's, during the second the next chunk's Q and first half
  constexpr int L = LP::N + LQ::N, H = BI / 2, M = H * BJ, R = BJ + H;
  static_assert(S % 2 == 0 && BI % 2 == 0 && (S - 2) * L < 64, "stages, blocks, loads in flight");
  u32x4 fp[BI], fq[2][BJ];
  const typename LP::template Lane<BI> pl(prow, lane);
  const typename LQ::template Lane<BJ> ql(qrow, lane);
  // read r of a chunk's Q and first half
  auto read = [&](const char* from, int set, int r) __attribute__((always_inline)) {
    if (r < BJ) fq[set][r] = ql.frag(from + LP::kBytes, r);
    else fp[r - BJ] = pl.frag(from, r - BJ);
  };
  auto issue = [&](int l, const typename LP::Chunk& cp, const typename LQ::Chunk& cq, char* stage)
      __attribute__((always_inline)) {
    if (l < LP::N) lp.issue(cp, l, stage);
    else lq.issue(cq, l - LP::N, stage + LP::kBytes);
  };
  auto chunk = [&](int q, int i) __attribute__((always_inline)) {
    char *const cur = stages[i], *const next = stages[(i + 1) % S];
    char* const far = stages[(i + S - 1) % S];
    const typename LP::Chunk cp = lp.chunk(q + i + S - 1, q + i + S - 1 < q1);
    const typename LQ::Chunk cq = lq.chunk(q + i + S - 1, q + i + S - 1 < q1);
    // reads and loads one at a time among the products: in a row they would hold up
    // the wave
#pragma unroll
    for (int m = 0; m < M; ++m) {
      mul(fp[m / BJ], fq[i & 1][m % BJ], m / BJ, m % BJ, i);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int o = m * (H + L) / M; o < (m + 1) * (H + L) / M; ++o) {
        if (o < H) fp[H + o] = pl.frag(cur, H + o);
        else issue(o - H, cp, cq, far);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
    // the loads of the next chunk are in (those behind it may not be), and no wave
    // reads this chunk's stage any more
    wait_barrier<(S - 2) * L>();
#pragma unroll
    for (int m = 0; m < M; ++m) {
      mul(fp[H + m / BJ], fq[i & 1][m % BJ], H + m / BJ, m % BJ, i);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int o = m * (R + R / 2) / M; o < (m + 1) * (R + R / 2) / M; ++o)
        if (o < R) read(next, (i + 1) & 1, o);
      __builtin_amdgcn_sched_barrier(0);
    }
  };
#pragma unroll
  for (int i = 0; i < S - 1; ++i) {
    const typename LP::Chunk cp = lp.chunk(q0 + i, q0 + i < q1);
    const typename LQ::Chunk cq = lq.chunk(q0 + i, q0 + i < q1);
#pragma unroll
    for (int l = 0; l < L; ++l) issue(l, cp, cq, stages[i]);
  }
  wait_barrier<(S - 2) * L>();
#pragma unroll
  for (int r = 0; r < R; ++r) read(stages[0], 0, r);
  for (int q = q0; q < q1; q += S) {
    round(q);
#pragma unroll
    for (int i = 0; i < S; ++i) chunk(q, i);
  }
  wait_barrier<0>();
}

// Rows of RB bytes in LDS on their way to memory: piece c (16 bytes) of row r.
template <int RB>
__device__ __forceinline__ char* out_piece(char* buf, int r, int c) {
  return buf + r * RB + ((c ^ (r & (RB / 16 - 1))) << 4);
}

// A launch's time in us by its tiles: `begin` and `chunk` a chunk for the first work-group
// on a CU, `more` and `more_chunk` a chunk for each further one (beside the others as far as
// they fit).  The launchers' figures are of launches of one to eight work-groups a CU.
struct TileTime {
  double begin, chunk, more, more_chunk;
};
inline double tile_cost(long long groups, int chunks, const TileTime& t) {
  const double further = (double)((groups + 255) / 256 - 1);
  return t.begin + chunks * t.chunk + further * (t.more + chunks * t.more_chunk);
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
