// The tile loop of mma_tile.h on pairs of chunks: an operand with k along its rows is loaded in
// whole cache lines (128 bytes of a row, two chunks, at a time).
//
// A load instruction of 64-byte pieces takes twice the requests of the L1 and L2 caches, and those,
// not the matrix cores, set the pace of 256 x 256 tiles: 4096 tokens x 65536 channels, k 4096, on
// zeros (at the full clock) 0.66 us a chunk, 0.50 in whole lines, 0.44 with no loads at all (the
// products' own time); on random data, where power sets the clock, 0.74 and 0.66.
//
// Each operand has a ring of slots of a pair each.  A pair's slot is free behind the barrier
// in the middle of its second chunk: Q's next pair for it is loaded in that chunk's second half, P's
// in the first half of the next chunk.
#pragma once

#include <utility>

#include "mma_tile.h"

namespace jarq {

// An operand tile of TR rows of one matrix with k along the rows, staged by NW wavefronts: eight
// rows x 128 bytes a load instruction.  The eight pieces of a row are permuted by the row so
// that the sixteen lanes that LDS serves at a time (lanes 0..3, 12..15 and 20..27 of a fragment
// read, and the like) fall in distinct banks.  Rows past the last read the last one; k past the end
// reads zeros.
template <int TR, int NW>
struct PairContig {
  static constexpr int N = TR / 8 / NW;     // load instructions a wave and pair
  static_assert(N >= 1 && N * 8 * NW == TR, "tile");
  static constexpr int kBytes = TR * 128;   // a slot
  Buffer from;
  uint32_t off[N];
  int kbytes, wave, piece;

  // As KContig::init.
  __device__ __forceinline__ void init(const void* p, size_t ld, int row0, int rows, int kb, int w,
                                       int lane) {
    from = buffer_at((const char*)p + (size_t)row0 * ld, (size_t)(rows - row0 - 1) * ld + kb);
    kbytes = kb;
    wave = w;
    piece = 16 * ((lane & 7) ^ ((lane >> 3) & 6));
#pragma unroll
    for (int n = 0; n < N; ++n)
      off[n] = (uint32_t)min(8 * (w + NW * n) + (lane >> 3), rows - 1 - row0) * (uint32_t)ld +
               (uint32_t)piece;
  }
  // A pair's first byte of k, past the end where it is not `live`.
  struct Pair {
    int k0;
  };
  __device__ __forceinline__ Pair pair(int q, bool live) const {
    return {live ? q * kChunk : kbytes};
  }
  __device__ __forceinline__ void issue(const Pair& c, int n, char* slot) const {
    load_lds16(from, c.k0 + piece < kbytes ? off[n] : kNowhere, (uint32_t)c.k0,
               slot + 1024 * (wave + NW * n));
  }
  // This lane's place in a slot for a wave whose blocks of 16 rows start at row0.
  template <int B>
  struct Lane {
    uint32_t o;
    __device__ __forceinline__ Lane(int row0, int lane) {
      const int row = row0 + (lane & 15);
      o = (uint32_t)(row * 128 + 16 * ((lane >> 4) ^ (row & 6)));
    }
    // Fragment of block a of a pair's chunk `half`.
    __device__ __forceinline__ u32x4 frag(const char* slot, int half, int a) const {
      return *(const u32x4*)(slot + (o ^ (64u * half)) + 2048 * a);
    }
  };
};

// An operand tile of TR columns with k down the rows: a pair is 64 rows, which lie as KStrided's.
template <int TR, int NW>
struct PairStrided {
  typedef KStrided<TR, NW, kOne> One;
  static constexpr int N = 64 / One::RPI / NW;
  static_assert(N >= 1 && N * One::RPI * NW == 64, "tile");
  static constexpr int kBytes = TR * 128;
  const char* base;
  size_t ld;
  uint32_t off[N];
  int rows, wave, lt;

  // Which piece (eight columns) of row t of a pair lies in place x of the row; the other way round
  // the same.
  static __device__ __forceinline__ int piece(int t, int x) {
    return x ^ (One::swz(t) << 2) ^ ((t >> 2) & 2);
  }
  // As KStrided::init.
  __device__ __forceinline__ void init(const void* p, size_t ld_, int c0, int cols, int rows_,
                                       int w, int lane) {
    base = (const char*)p;
    ld = ld_;
    rows = rows_;
    wave = w;
    lt = One::RPI * w + lane / One::CPR;
#pragma unroll
    for (int n = 0; n < N; ++n) {
      const int t = lt + NW * One::RPI * n;
      off[n] = (uint32_t)t * (uint32_t)ld +
               2u * (uint32_t)min(c0 + 8 * piece(t, lane % One::CPR), cols - 8);
    }
  }
  struct Pair {
    Buffer from;
    int left;
  };
  __device__ __forceinline__ Pair pair(int q, bool live) const {
    const int k0 = q * One::kRows;
    return {buffer_at(base + (live ? (size_t)k0 * ld : 0), 0x7fffffff), live ? rows - k0 : 0};
  }
  __device__ __forceinline__ void issue(const Pair& c, int n, char* slot) const {
    load_lds16(c.from, lt + NW * One::RPI * n < c.left ? off[n] : kNowhere, 0,
               slot + 1024 * (wave + NW * n));
  }
  template <int B>
  struct Lane {
    typename One::template Lane<B> one;
    __device__ __forceinline__ Lane(int col0, int lane) : one(col0, lane) {}
    __device__ __forceinline__ u32x4 frag(const char* slot, int half, int a) const {
      return one.frag(slot + half * (TR * kChunk), a);
    }
  };
};

// The slots of a work-group, arrays of their own (see JARQ_STAGES): SP of P, SQ of Q.
#define JARQ_SLOTS(SP, SQ, pbytes, qbytes)                                                     \
  __shared__ __attribute__((aligned(1024))) char pslot0[pbytes], pslot1[pbytes],               \
      qslot0[qbytes], qslot1[qbytes], pslot2[SP > 2 ? (pbytes) : 1], qslot2[SQ > 2 ? (qbytes) : 1]; \
  char* const pslots[3] = {pslot0, pslot1, pslot2};                                            \
  char* const qslots[3] = {qslot0, qslot1, qslot2}

// Chunks q0 <= q < q1 (at least one; q0 even, q1 even or the end of k).  SP is SQ or SQ + 1.
template <int SP, int SQ, int BI, int BJ, class LP, class LQ, class Mul>
struct PairLoop {
  static constexpr int H = BI / 2, M = H * BJ, R = BJ + H;
  static constexpr int U = SP == SQ ? SP : SP * SQ;   // pairs a round
  static_assert((SP == SQ || SP == SQ + 1) && SQ >= 2 && SP <= 3 && BI % 2 == 0, "slots, blocks");
  // loads behind the last that the next pair takes
  static constexpr int kBehind = SP == SQ ? (SP - 2) * (LP::N + LQ::N)
                                          : (SQ - 1) * LP::N + (SQ - 2) * LQ::N;
  static constexpr int kAtFirst = SP == SQ ? (SP - 2) * (LP::N + LQ::N) + LQ::N
                                           : (SQ - 1) * (LP::N + LQ::N);
  const LP& lp;
  const LQ& lq;
  const Mul& mul;
  char* const (&ps)[3];
  char* const (&qs)[3];
  const typename LP::template Lane<BI> pl;
  const typename LQ::template Lane<BJ> ql;
  int q, q1;
  u32x4 fp[BI], fq[2][BJ];

  // read r of a chunk's Q and first half of P
  __device__ __forceinline__ void read(const char* p, const char* qq, int half, int r) {
    if (r < BJ) fq[half][r] = ql.frag(qq, half, r);
    else fp[r - BJ] = pl.frag(p, half, r - BJ);
  }
  // One chunk: `half` of the pair in slots J % SP, J % SQ.
  template <int J, int half>
  __device__ __forceinline__ void chunk() {
    const char *const p = ps[J % SP], *const pn = ps[(J + half) % SP];
    const char* const qn = qs[(J + half) % SQ];
    constexpr int NP = half == 0 ? LP::N : 0, NQ = half == 1 ? LQ::N : 0;
    const typename LP::Pair cp = lp.pair(q + 2 * SP - 2, half == 0 && q + 2 * SP - 2 < q1);
    // reads and loads one at a time among the products: in a row they would hold up the wave
#pragma unroll
    for (int m = 0; m < M; ++m) {
      mul(fp[m / BJ], fq[half][m % BJ], m / BJ, m % BJ);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int o = m * (H + NP) / M; o < (m + 1) * (H + NP) / M; ++o) {
        if (o < H) fp[H + o] = pl.frag(p, half, H + o);
        else lp.issue(cp, o - H, ps[(J + SP - 1) % SP]);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
    // the next pair's loads are in, and no wave reads this one's slots any more
    if constexpr (half == 1) wait_barrier<kBehind>();
    const typename LQ::Pair cq = lq.pair(q + 2 * SQ - 1, half == 1 && q + 2 * SQ - 1 < q1);
#pragma unroll
    for (int m = 0; m < M; ++m) {
      mul(fp[H + m / BJ], fq[half][m % BJ], H + m / BJ, m % BJ);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int o = m * (R + R / 2 + NQ) / M; o < (m + 1) * (R + R / 2 + NQ) / M; ++o) {
        if (o < NQ) lq.issue(cq, o, qs[J % SQ]);
        else if (o - NQ < R) read(pn, qn, half ^ 1, o - NQ);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
    ++q;
  }
  template <int J>
  __device__ __forceinline__ bool pair() {
    chunk<J, 0>();
    chunk<J, 1>();
    return q < q1;
  }
  template <int... J>
  __device__ __forceinline__ void rounds(std::integer_sequence<int, J...>) {
    while ((pair<J>() && ...)) {
    }
  }
  __device__ __forceinline__ void run(int q0) {
    q = q0;
#pragma unroll
    for (int k = 0; k < SQ; ++k) {
      const typename LP::Pair cp = lp.pair(q0 + 2 * k, q0 + 2 * k < q1);
      const typename LQ::Pair cq = lq.pair(q0 + 2 * k, q0 + 2 * k < q1);
      if (SP > SQ)
#pragma unroll
        for (int n = 0; n < LP::N; ++n) lp.issue(cp, n, ps[k]);
#pragma unroll
      for (int n = 0; n < LQ::N; ++n) lq.issue(cq, n, qs[k]);
      if (SP == SQ && k < SP - 1)
#pragma unroll
        for (int n = 0; n < LP::N; ++n) lp.issue(cp, n, ps[k]);
    }
    wait_barrier<kAtFirst>();
#pragma unroll
    for (int r = 0; r < R; ++r) read(ps[0], qs[0], 0, r);
    rounds(std::make_integer_sequence<int, U>{});
    wait_barrier<0>();
  }
};
// mul(p, q, a, b) gets the fragments of P block a and Q block b of each chunk; a wave's BI
// blocks of P start at row prow of the tile, its BJ of Q at qrow.
template <int SP, int SQ, int BI, int BJ, class LP, class LQ, class Mul>
__device__ __forceinline__ void mma_pairs(const LP& lp, const LQ& lq, int q0, int q1, int lane,
                                          int prow, int qrow, char* const (&ps)[3],
                                          char* const (&qs)[3], const Mul& mul) {
  PairLoop<SP, SQ, BI, BJ, LP, LQ, Mul> loop{lp, lq, mul, ps, qs, {prow, lane}, {qrow, lane}, 0, q1, {}, {}};
  loop.run(q0);
}

}  // namespace jarq
