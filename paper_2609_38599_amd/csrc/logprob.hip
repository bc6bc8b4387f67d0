// Log probabilities of given tokens, entropies and top alternatives of rows of
// logits, and the gradient of the logits.
//
// With m = max x, z = sum exp(x - m): lse = m + log z, log p_v = x_v - lse and
// H = log z - sum exp(x - m) (x - m) / z, all from one pass that keeps m per wavefront and
// (z - 1, sum exp(x - m) (x - m)) per lane and rescales when m grows.  (z - 1, the sum beside the
// maximum's own 1: where one entry takes nearly all, z would round away what the others
// take, which is the log probability of that entry.)
//
// A row in which any entry is +infinity or NaN gives NaN (and index -1); entries
// of -infinity have probability 0; a row of nothing else has lse = -infinity.
#include <float.h>

#include "mma_tile.h"

namespace jarq {

namespace {

typedef unsigned long long u64;

// Any: sixteen bytes at any element.
template <int DT> struct Elem {
  typedef uint16_t T;
  static constexpr int kVec = 8;
  typedef u32x4 Any __attribute__((aligned(2)));
};
template <> struct Elem<0> {
  typedef float T;
  static constexpr int kVec = 4;
  typedef u32x4 Any __attribute__((aligned(4)));
};

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

template <int DT>
__device__ __forceinline__ u32x4 minus_inf() {
  const uint32_t w = DT == 0 ? 0xff800000u : DT == kF16 ? 0xfc00fc00u : 0xff80ff80u;
  return u32x4{w, w, w, w};
}

// The running maximum (at least -FLT_MAX, so that x - m is never -inf + inf), the sum
// beside the maximum's own 1 (-1: no entry above -infinity) and the weighted sum.
struct Soft {
  float m, more, zt;
  __device__ __forceinline__ bool none() const { return more == -1.f; }
  __device__ __forceinline__ bool broken() const { return more != more; }
};
__device__ __forceinline__ Soft no_entries() { return Soft{-FLT_MAX, -1.f, 0.f}; }
// Keeps exp's argument within range for the weighted sum: exp is 0 there.
constexpr float kLeast = -1000.f;

__device__ __forceinline__ float first_lane(float x) {
  return __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(x)));
}
// A lane's sums under its wave's running maximum.  One entry of the maximum's value, of lane
// `holder` (-1: none yet), is in no sum.  (A maximum a lane would grow in nearly every round
// of some lane, and each time all would rescale.)
struct LaneSums {
  float m, more, zt;
  int holder;
};
__device__ __forceinline__ LaneSums no_sums() { return LaneSums{-FLT_MAX, 0.f, 0.f, -1}; }

// Adds entries; returns the lane's largest.  Every lane of the wave calls it.
template <int DT, int N>
__device__ __forceinline__ float add(LaneSums& s, const float (&entries)[N], int lane) {
  float x[N], most = entries[0];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    x[i] = entries[i];
    most = fmaxf(most, x[i]);
  }
  if (__ballot(most > s.m) != 0) {   // uniform
    float m = fmaxf(most, s.m);
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) m = fmaxf(m, __shfl_xor(m, off));
    m = first_lane(m);
    const float t = s.m - m, e = exp_of<DT>(t), z = s.more + (lane == s.holder ? 1.f : 0.f);
    s.zt = e * (s.zt + z * fmaxf(t, kLeast));
    s.more = e * z;
    s.m = m;
    // (+infinity stays in the sum: it gives a NaN)
    s.holder = m == INFINITY ? -1 : (int)__builtin_ctzll(__ballot(most == m));
    bool out = lane != s.holder;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const bool own = !out && x[i] == m;
      out |= own;
      x[i] = own ? -INFINITY : x[i];
    }
  }
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const float t = x[i] - s.m, e = exp_of<DT>(t);
    s.more += e;
    s.zt = fmaf(e, fmaxf(t, kLeast), s.zt);
  }
  return most;
}
// The wave's sums, in every lane.
__device__ __forceinline__ Soft sums_of(const LaneSums& s) {
  float more = s.more, zt = s.zt;
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) {
    more += __shfl_xor(more, off);
    zt += __shfl_xor(zt, off);
  }
  return Soft{s.m, s.holder < 0 ? more - 1.f : more, zt};
}
__device__ __forceinline__ void join(Soft& s, const Soft& o) {
  const bool first = s.m >= o.m;
  const Soft a = first ? s : o, b = first ? o : s;   // the larger maximum's, the other's
  const float t = b.m - a.m, e = expf(t), z = 1.f + b.more;
  s.m = a.m;
  s.more = fmaf(e, z, a.more);
  s.zt = a.zt + e * (b.zt + z * fmaxf(t, kLeast));
}

__device__ __forceinline__ void join_wave(Soft& s) {
#pragma unroll 1   // (short code: a work-group reads it anew)
  for (int off = 32; off >= 1; off >>= 1) {
    Soft o;
    o.m = __shfl_xor(s.m, off);
    o.more = __shfl_xor(s.more, off);
    o.zt = __shfl_xor(s.zt, off);
    join(s, o);
  }
}
// log sum exp, rounded, and what the rounding left: t = (x - lse) - rest is log p to an ulp
// or two of itself (x - lse alone would be off by an ulp of lse).
__device__ __forceinline__ void lse_parts(const Soft& s, float lz, float& lse, float& rest) {
  lse = s.none() ? -INFINITY : s.m + lz;
  const float d = lse - s.m;
  rest = s.none() ? 0.f : (s.m - (lse - d)) + (lz - d);
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
__device__ __forceinline__ uint32_t ordered(float x) { return (uint32_t)(top_key(x, 0) >> 32); }
constexpr uint32_t kOrderedMinusInf = 0x007fffffu;

// Entries of a wave (R a lane, n in all, 64 to a register) that are at least `t` > 0.
template <int R>
__device__ __forceinline__ int count_from(const uint32_t (&v)[R], int n, uint32_t t) {
  int c = 0;
#pragma unroll
  for (int r = 0; r < R; ++r)
    if (64 * r < n) c += __popcll(__ballot(v[r] >= t));   // uniform
  return c;
}
// The largest value, of `bits` leading bits and zeros behind, that at least k of a
// wave's entries reach; 0 if there are fewer.
template <int R>
__device__ __forceinline__ uint32_t reached_by(const uint32_t (&v)[R], int n, int k, int bits) {
  uint32_t t = 0;
#pragma unroll 1
  for (int b = 31; b >= 32 - bits; --b)
    if (count_from<R>(v, n, t | (1u << b)) >= k) t |= 1u << b;
  return t;
}

// A wave's candidates for the top k: keys in LDS, cut back to the k largest when
// more than kKeep are there.  A lane's entries are offered four at a time.
constexpr int kKeep = 128;
struct TopList {
  static constexpr int kCap = kKeep + 64 * 4;   // and eight zeros behind the last key
  u64* keys;          // of this wave
  uint32_t* slots;    // one a wave: a value that ceil(k / 4) of its entries reach
  int n, k, wave;
  u64 kth;            // the k-th largest key when the list was last cut
  float bound;        // a value that k entries of the row reach

  __device__ __forceinline__ void init(u64* keys_, uint32_t* slots_, int k_, int w) {
    keys = keys_;
    slots = slots_;
    k = k_;
    wave = w;
    n = 0;
    kth = 0;
    bound = -INFINITY;
  }
  // From the lanes' largest entries so far: the four waves' slots together name a
  // value that k entries of the row reach.  Every wave of the work-group calls it.
  __device__ __forceinline__ void raise(float lane_max, int lane) {
    const uint32_t v[1] = {ordered(lane_max)};
    // 16 bits: lower than the value by less than a bf16 step
    const uint32_t mine = max(reached_by<1>(v, 64, (k + 3) / 4, 16), kOrderedMinusInf);
    if (lane == 0) slots[wave] = mine;
    __syncthreads();
    const uint32_t least = min(min(slots[0], slots[1]), min(slots[2], slots[3]));
    bound = fmaxf(bound, key_value((u64)least << 32));
    __syncthreads();   // (before the next one's slots)
  }
  // Entries at the row's end, of the lanes that have one: kept without a look.
  __device__ __forceinline__ void keep(bool has, float x, int i, int lane) {
    const u64 mask = __ballot(has);
    if (has) keys[__popcll(mask & ((1ull << lane) - 1))] = top_key(x, (uint32_t)i);
    n = __popcll(mask);
  }
  // x: this lane's entries from index i0 on; lanes that are not `in` have none.
  __device__ __forceinline__ void offer(const float (&x)[4], bool in, int i0, int lane) {
    if (__ballot(in && fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])) >= bound) == 0) return;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const bool may = in && x[i] >= bound;
      if (__ballot(may) == 0) continue;
      const u64 key = top_key(x[i], (uint32_t)(i0 + i));
      const bool hit = may && key > kth;
      const u64 mask = __ballot(hit);
      if (hit) keys[n + __popcll(mask & ((1ull << lane) - 1))] = key;
      n += __popcll(mask);
    }
  }
  // Drops the keys that the bound has passed.
  __device__ __forceinline__ void sift(int lane) {
    asm volatile("" ::: "memory");   // one wave: its LDS accesses complete in order
    const uint32_t least = ordered(bound);
    int m = 0;
#pragma unroll 1
    for (int r = 0; r < n; r += 64) {
      const u64 key = r + lane < n ? keys[r + lane] : 0;
      const bool keep = key != 0 && (uint32_t)(key >> 32) >= least;
      const u64 mask = __ballot(keep);
      if (keep) keys[m + __popcll(mask & ((1ull << lane) - 1))] = key;
      m += __popcll(mask);
    }
    asm volatile("" ::: "memory");
    n = m;
  }
  __device__ __forceinline__ void cut(int lane) {
    constexpr int R = kCap / 64;
    if (n <= k) return;
    asm volatile("" ::: "memory");   // one wave: its LDS accesses complete in order
    uint32_t hi[R], lo[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const int at = 64 * r + lane;
      const u64 key = at < n ? keys[at] : 0;
      hi[r] = (uint32_t)(key >> 32);
      lo[r] = (uint32_t)key;
    }
    const uint32_t v = reached_by<R>(hi, n, k, 32);
    // among the entries of value v, those of the lowest indices
    int above = 0;
#pragma unroll
    for (int r = 0; r < R; ++r) {
      above += __popcll(__ballot(hi[r] > v));
      if (hi[r] != v) lo[r] = hi[r] > v ? 0xffffffffu : 0u;
    }
    const uint32_t l = reached_by<R>(lo, n, k, 32);
    int m = 0;
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const bool keep = hi[r] > v || (hi[r] == v && lo[r] >= l);
      const u64 mask = __ballot(keep);
      // (a key above v is found again from its LDS place)
      const u64 key = keep ? keys[64 * r + lane] : 0;
      if (keep) keys[m + __popcll(mask & ((1ull << lane) - 1))] = key;
      m += __popcll(mask);
    }
    asm volatile("" ::: "memory");
    n = m;
    kth = ((u64)v << 32) | l;
    bound = fmaxf(bound, key_value((u64)v << 32));
  }
};

struct RowOut {
  float *logprob, *entropy, *lse, *rest, *top_logprob;
  int32_t* top_index;
};

// log p = (x - m) - log z: closer than x - lse where one entry takes nearly all.
__device__ __forceinline__ float log_p(float x, const Soft& s, float lz) {
  return s.none() ? -INFINITY : (x - s.m) - lz;
}

// One thread: the row's results from its sums, lz = log z.
template <int DT>
__device__ __forceinline__ void finish_row(const Soft& s, const void* row, int64_t target, int V,
                                           size_t t, float lz, const RowOut& o) {
  float lp = 0.f;
  if (target >= V) lp = __uint_as_float(0x7fc00000u);
  else if (target >= 0) lp = log_p(value<DT>(((const typename Elem<DT>::T*)row)[target]), s, lz);
  o.logprob[t] = lp;
  if (o.entropy) o.entropy[t] = s.none() ? 0.f : lz - s.zt / (1.f + s.more);
  float lse, rest;
  lse_parts(s, lz, lse, rest);
  if (o.lse) o.lse[t] = lse;
  if (o.rest) o.rest[t] = rest;
}
__device__ __forceinline__ void store_top(const RowOut& o, size_t at, u64 key, const Soft& s,
                                          float lz) {
  const bool bad = s.broken();
  o.top_index[at] = bad ? -1 : (int32_t)key_index(key);
  o.top_logprob[at] = bad ? s.more : log_p(key_value(key), s, lz);
}

}  // namespace

// Work-group `id`: part id % splits (of `each` entries) of row id / splits.  With one
// part it finishes the row; otherwise its sums and top keys go to the workspace.  Bound by
// reading the logits (4096 x 128000 in bf16, no top: 230 us, 4.6 TB/s), with a top by the
// issue of its candidates' votes (2047 x 32001 in fp32: 53 us without, top 20 66 us).
// Eight waves a SIMD, which keeps the registers at 64: with 70 the top 5 of 2047 x 50257 in
// fp16 take 73 us, 69 so.
template <int DT, bool TOP>
__global__ __launch_bounds__(256) JARQ_WAVES(8) void logprob_kernel(
    const void* __restrict__ logits, size_t ld, int V, const int64_t* __restrict__ targets,
    int splits, int each, int top, RowOut out, float* __restrict__ psum,
    u64* __restrict__ pkey) {
  typedef typename Elem<DT>::T E;
  constexpr int VE = Elem<DT>::kVec;
  __shared__ Soft red[4];
  __shared__ __attribute__((aligned(16))) u64 keys[TOP ? 4 * (TopList::kCap + 8) : 1];
  __shared__ uint32_t slots[4];
  __shared__ int counts[4];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const size_t t = blockIdx.x / (unsigned)splits;
  const int part = blockIdx.x % (unsigned)splits;
  const E* row = (const E*)logits + t * ld;
  const int b = part * each, e = min(V, b + each);
  // Vectors from the part's first entry on, wherever that lies, then scalars: what a lane sums
  // goes by the entries' indices alone, so a row's results do not depend on its address.
  // (rows of 32001 in fp32, most off 16 bytes, and from a 16-byte boundary on: the same time)
  const int nv = (e - b) / VE;
  const typename Elem<DT>::Any* vec = (const typename Elem<DT>::Any*)(row + b);
  const int own = b + nv * VE + tid;   // this thread's scalar, if any
  const bool has = own < e;
  LaneSums sums = no_sums();
  TopList list;
  const float edge = has ? value<DT>(row[own]) : -INFINITY;
  float lane_max = edge;
  if constexpr (TOP) {
    list.init(keys + wave * (TopList::kCap + 8), slots, top, wave);
    if (tid < 4) slots[tid] = kOrderedMinusInf;
    __syncthreads();
    list.keep(has, edge, own, lane);
  }
  // U vectors a lane in flight (every lane of a wave stays in the loop, for the list's
  // votes; lanes past the end take -infinity, which adds nothing)
  constexpr int U = 4;
  int round = 0;
  for (int v0 = 64 * wave; v0 - 64 * wave < nv; v0 += 256 * U, ++round) {   // uniform
    u32x4 w[U];
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const int v = v0 + 256 * i + lane;
      w[i] = v < nv ? vec[v] : minus_inf<DT>();
    }
    float most = -INFINITY;
#pragma unroll
    for (int i = 0; i < U; ++i) {
      float x[VE];
      unpack<DT>(w[i], x);
      most = fmaxf(most, add<DT>(sums, x, lane));
    }
    lane_max = fmaxf(lane_max, most);
    if constexpr (TOP) {
      // rounds 0, 2, 6, 14, ..: twice as many entries are in each time
      if (((round + 1) & (round + 2)) == 0) list.raise(lane_max, lane);
      if (__ballot(most >= list.bound) == 0) continue;
      constexpr int Q = U * VE / 4;   // offers
#pragma unroll 1
      for (int i = 0; i < Q; ++i) {
        const int v = v0 + 256 * (i * 4 / VE) + lane;
        float x[VE];
        unpack<DT>(w[0], x);
        const float y[4] = {x[0], x[1], x[2], x[3]};
        list.offer(y, v < nv, b + v * VE + i * 4 % VE, lane);
        // (the others move up: a register array takes no index)
        if constexpr (VE == 4) {
          w[0] = w[1];
          w[1] = w[2];
          w[2] = w[3];
        } else {
#pragma unroll
          for (int j = 0; j < U; ++j) {
            const u32x4 next = j + 1 < U ? w[j + 1] : w[j];
            w[j] = u32x4{w[j][2], w[j][3], next[0], next[1]};
          }
        }
        if (list.n > kKeep) list.cut(lane);
      }
    }
  }
  {
    const float x[1] = {edge};
    add<DT>(sums, x, lane);
  }
  if constexpr (TOP) list.raise(lane_max, lane);
  Soft s = sums_of(sums);
  if (lane == 0) red[wave] = s;
  if constexpr (TOP) {
    list.sift(lane);
    if (list.n > 64) list.cut(lane);
    if (lane < 8) list.keys[list.n + lane] = 0;
    if (lane == 0) counts[wave] = list.n;
  }
  __syncthreads();
  s = red[0];
#pragma unroll
  for (int w = 1; w < 4; ++w) join(s, red[w]);
  const float lz = log1pf(s.more);
  if (splits == 1) {
    if (tid == 0) finish_row<DT>(s, row, targets[t], V, t, lz, out);
  } else if (tid == 0) {
    float* p = psum + 3 * (size_t)blockIdx.x;
    p[0] = s.m;
    p[1] = s.more;
    p[2] = s.zt;
  }
  if constexpr (TOP) {
    // a key's place is the number of larger ones in the four lists
    const u64 mine = lane < list.n ? list.keys[lane] : 0;
    int place = 0, total = 0;
    for (int w = 0; w < 4; ++w) {
      const int m = counts[w];
      total += m;
      // (eight at a time, zeros behind the last)
      for (int i = 0; i < m; i += 8) {
#pragma unroll
        for (int j = 0; j < 8; ++j) place += keys[w * (TopList::kCap + 8) + i + j] > mine;
      }
    }
    const bool bad = s.broken();
    if (splits == 1) {
      if (bad) {
        if (tid < top) store_top(out, t * top + tid, 0, s, lz);
      } else if (lane < list.n && place < top) {
        store_top(out, t * top + place, mine, s, lz);
      }
    } else {
      u64* to = pkey + (size_t)blockIdx.x * top;
      if (lane < list.n && place < top) to[place] = mine;
      if (tid >= total && tid < top) to[tid] = 0;   // a part of fewer entries
    }
  }
}

// A work-group a row: its parts' sums (at most 64 parts, joined in a fixed order) and the
// top of their keys (at most 256).  Bound by its chain's latency: 1 x 128000, 31 parts, top 8
// 6 us.
template <int DT>
__global__ __launch_bounds__(256) void logprob_join_kernel(
    const void* __restrict__ logits, size_t ld, int V, const int64_t* __restrict__ targets,
    int splits, int top, RowOut out, const float* __restrict__ psum,
    const u64* __restrict__ pkey) {
  typedef typename Elem<DT>::T E;
  __shared__ u64 keys[256];
  const int tid = threadIdx.x;
  const size_t t = blockIdx.x;
  const int n = splits * top;
  const u64 mine = tid < n ? pkey[t * n + tid] : 0;
  keys[tid] = mine;
  // a part a lane, at most 64 of them
  Soft s = no_entries();
  const int lane = tid & 63;
  if (lane < splits) {
    const float* q = psum + 3 * (t * splits + lane);
    s.m = q[0];
    s.more = q[1];
    s.zt = q[2];
  }
  join_wave(s);
  // one lane's: where parts tie for the maximum, lanes add their sums in different orders
  s.m = first_lane(s.m);
  s.more = first_lane(s.more);
  s.zt = first_lane(s.zt);
  const float lz = log1pf(s.more);
  if (tid == 0) finish_row<DT>(s, (const E*)logits + t * ld, targets[t], V, t, lz, out);
  __syncthreads();
  if (s.broken()) {
    if (tid < top) store_top(out, t * top + tid, 0, s, lz);
    return;
  }
  int place = 0;
  for (int i = 0; i < n; i += 8) {   // (zeros from n on)
#pragma unroll
    for (int j = 0; j < 8; ++j) place += keys[i + j] > mine;
  }
  if (mine != 0 && place < top) store_top(out, t * top + place, mine, s, lz);
}

// ---- gradient ----
// d x_v = g (onehot - p) - h p (log p + H), g and h the gradients of the log
// probability and of the entropy; at the target 1 - p from log p, which p's rounding would
// lose where it is near 1.  Work-group `id`: part id % splits of a row.  A thread reads each
// entry before it writes it: dlogits may be the logits.  SUMS: the row's sums are not given
// and are formed first, by the one work-group that the row then has (calls of 4096 x 128000 in
// bf16 644 us, 438 with the sums given; of one such row 45 and 11).  Bound by memory: 4096 x
// 128000 in bf16 410 us, 5.1 TB/s.
template <int DT, bool SUMS>
__global__ __launch_bounds__(256) void logprob_grad_kernel(
    const void* logits, size_t ld, int V, const int64_t* __restrict__ targets,
    const float* __restrict__ lse_of, const float* __restrict__ rest_of,
    const float* __restrict__ entropy, const float* __restrict__ dlp,
    const float* __restrict__ dent, int splits, int each, void* dlogits, size_t ldd) {
  typedef typename Elem<DT>::T E;
  constexpr int VE = Elem<DT>::kVec;
  __shared__ Soft red[SUMS ? 4 : 1];
  const int tid = threadIdx.x;
  // the last rows first: what the forward pass read last may still be cached
  const size_t t = (gridDim.x - 1 - blockIdx.x) / (unsigned)splits;
  const int b = (int)(blockIdx.x % (unsigned)splits) * each, e = min(V, b + each);
  const E* row = (const E*)logits + t * ld;
  E* drow = (E*)dlogits + t * ldd;
  const uintptr_t ax = (uintptr_t)(row + b) % 16, ad = (uintptr_t)(drow + b) % 16;
  const int head = min(e - b, (int)((16 - ax) % 16 / sizeof(E)));
  const int nv = (e - b - head) / VE, rest = b + head + nv * VE;
  const int own = tid < head ? b + tid : rest + tid - head;
  const bool has = tid < head || own < e;
  const u32x4* vec = (const u32x4*)(row + b + head);
  float lse, left;
  if constexpr (SUMS) {
    // (by the entries' indices alone, as in the forward pass)
    LaneSums sums = no_sums();
    const int n = V / VE, last = n * VE + tid, lane = tid & 63;
    for (int v0 = tid - lane; v0 < n; v0 += 256) {   // every lane of a wave
      const u32x4 w = v0 + lane < n ? ((const typename Elem<DT>::Any*)row)[v0 + lane]
                                    : minus_inf<DT>();
      float x[VE];
      unpack<DT>(w, x);
      add<DT>(sums, x, lane);
    }
    const float edge[1] = {last < V ? value<DT>(row[last]) : -INFINITY};
    add<DT>(sums, edge, lane);
    Soft s = sums_of(sums);
    if (lane == 0) red[tid >> 6] = s;
    __syncthreads();   // (and every entry is read before the first is written)
    s = red[0];
#pragma unroll
    for (int w = 1; w < 4; ++w) join(s, red[w]);
    lse_parts(s, log1pf(s.more), lse, left);
  } else {
    lse = lse_of[t];
    left = rest_of[t];
  }
  const int64_t target = targets[t];
  const int at = target >= 0 && target < V ? (int)target : -1;
  const float g = target < 0 ? 0.f : target >= V ? __uint_as_float(0x7fc00000u) : dlp[t];
  const float h = dent ? dent[t] : 0.f;
  const float ent = dent ? entropy[t] : 0.f;
  const bool empty = lse == -INFINITY;   // nothing but -infinity: no gradient
  auto grad = [&](float x) __attribute__((always_inline)) {
    const float lp = (x - lse) - left;
    const float c = exp_of<DT>(lp) * fmaf(h, fmaxf(lp, kLeast) + ent, g);
    return empty ? 0.f : -c;
  };
  auto grad_at_target = [&](float x) __attribute__((always_inline)) {
    const float lp = (x - lse) - left;
    const float c = exp_of<DT>(lp) * h * (fmaxf(lp, kLeast) + ent);
    return empty ? 0.f : fmaf(g, -expm1f(lp), -c);
  };
  auto word = [](float x) __attribute__((always_inline)) -> E {
    if constexpr (DT == 0) return x;
    else return to16<DT>(x);
  };
  auto put = [&](int v) __attribute__((always_inline)) {
    const float x = value<DT>(row[v]);
    drow[v] = word(v == at ? grad_at_target(x) : grad(x));
  };
  if (ax != ad) {   // uniform
    for (int v = b + tid; v < e; v += 256) put(v);
    return;
  }
  if (has) put(own);
  u32x4* dvec = (u32x4*)(drow + b + head);
  for (int v = tid; v < nv; v += 256) {
    float x[VE], y[VE];
    unpack<DT>(vec[v], x);
    const int in = at - (b + head + v * VE);   // the target's place here
#pragma unroll
    for (int i = 0; i < VE; ++i) y[i] = grad(x[i]);
    if ((unsigned)in < (unsigned)VE) {
      float its = x[0];
#pragma unroll
      for (int i = 1; i < VE; ++i) its = in == i ? x[i] : its;
      its = grad_at_target(its);
#pragma unroll
      for (int i = 0; i < VE; ++i) y[i] = in == i ? its : y[i];
    }
    u32x4 w;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (DT == 0) w[i] = __float_as_uint(y[i]);
      else w[i] = pack16<DT>(y[2 * i], y[2 * i + 1]);
    }
    dvec[v] = w;
  }
}

namespace {

// Parts a row is cut into: few rows alone would leave CUs idle.
struct LogprobPlan {
  int splits, each;
};
LogprobPlan logprob_plan(int T, int V, int top) {
  LogprobPlan p;
  int splits = 2048 / T;   // eight work-groups a CU
  const int most = V / 4096;
  splits = splits < 1 || most < 1 ? 1 : splits > most ? most : splits;
  // the joining work-group takes a key a thread
  const int cap = top > 4 ? 256 / top : 64;
  if (splits > cap) splits = cap;
  p.each = ((V + splits - 1) / splits + 63) / 64 * 64;
  p.splits = (V + p.each - 1) / p.each;
  return p;
}

template <int DT>
hipError_t logprob_kind(hipStream_t st, const void* logits, size_t ld, int T, int V,
                        const int64_t* targets, int top, const RowOut& out, char* ws) {
  const LogprobPlan p = logprob_plan(T, V, top);
  u64* pkey = (u64*)ws;
  float* psum = (float*)(ws + 8 * (size_t)T * p.splits * top);
  const dim3 grid((unsigned)(T * p.splits));
  if (top > 0)
    hipLaunchKernelGGL((logprob_kernel<DT, true>), grid, dim3(256), 0, st, logits, ld, V, targets,
                       p.splits, p.each, top, out, psum, pkey);
  else
    hipLaunchKernelGGL((logprob_kernel<DT, false>), grid, dim3(256), 0, st, logits, ld, V, targets,
                       p.splits, p.each, top, out, psum, pkey);
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
                             const int64_t* targets, const float* lse, const float* rest,
                             const float* entropy, const float* dlp, const float* dent,
                             void* dlogits, size_t ldd) {
  if (rest) {
    const LogprobPlan p = logprob_plan(T, V, 0);
    hipLaunchKernelGGL((logprob_grad_kernel<DT, false>), dim3((unsigned)(T * p.splits)), dim3(256),
                       0, st, logits, ld, V, targets, lse, rest, entropy, dlp, dent, p.splits,
                       p.each, dlogits, ldd);
  } else {
    hipLaunchKernelGGL((logprob_grad_kernel<DT, true>), dim3((unsigned)T), dim3(256), 0, st, logits,
                       ld, V, targets, lse, rest, entropy, dlp, dent, 1, V, dlogits, ldd);
  }
  return hipGetLastError();
}

}  // namespace

size_t logprob_workspace_bytes(int T, int V, int top) {
  const LogprobPlan p = logprob_plan(T, V, top);
  return p.splits == 1 ? 0 : (size_t)T * p.splits * (8 * (size_t)top + 12);
}

hipError_t launch_token_logprobs(hipStream_t st, int dtype, const void* logits, size_t ld, int T,
                                 int V, const int64_t* targets, int top, float* logprob,
                                 float* entropy, float* lse, float* rest, int32_t* top_index,
                                 float* top_logprob, char* ws) {
  const RowOut out{logprob, entropy, lse, rest, top_logprob, top_index};
  if (dtype == 0) return logprob_kind<0>(st, logits, ld, T, V, targets, top, out, ws);
  if (dtype == kF16) return logprob_kind<kF16>(st, logits, ld, T, V, targets, top, out, ws);
  return logprob_kind<kBF16>(st, logits, ld, T, V, targets, top, out, ws);
}

hipError_t launch_token_logprobs_backward(hipStream_t st, int dtype, const void* logits, size_t ld,
                                          int T, int V, const int64_t* targets, const float* lse,
                                          const float* rest, const float* entropy,
                                          const float* dlp, const float* dent, void* dlogits,
                                          size_t ldd) {
  if (dtype == 0)
    return logprob_grad_kind<0>(st, logits, ld, T, V, targets, lse, rest, entropy, dlp, dent,
                                dlogits, ldd);
  if (dtype == kF16)
    return logprob_grad_kind<kF16>(st, logits, ld, T, V, targets, lse, rest, entropy, dlp, dent,
                                   dlogits, ldd);
  return logprob_grad_kind<kBF16>(st, logits, ld, T, V, targets, lse, rest, entropy, dlp, dent,
                                  dlogits, ldd);
}

}  // namespace jarq
