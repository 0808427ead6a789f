// What the two attention kernels share: parameters, the division of a step's work
// over the CTAs, and the joining of a split item's parts.
//
// Work is counted in units (one tile of keys against one tile of rows), laid out
// sequence by sequence, and every CTA takes an equal share of consecutive units, so
// a step of any mix of lengths ends everywhere at the same time.  An item (a
// sequence, a key head, a tile of rows) that lies across CTAs is split: each part
// leaves (m, l, o) in the workspace, and the CTA that arrives last joins them in
// order.  Lengths are read from device memory, by every CTA for itself.
#pragma once

#include "gs_block.cuh"
#include "gs_sm100.cuh"

#include <cuda.h>

namespace gs {

struct AttnParams {
  CUtensorMap kmap, vmap;   // (64, rows, head_dim / 64) slabs over [pages * kv_heads * page_size][head_dim]
  const uint16_t* q;
  const uint16_t* v;        // the value pages (re-read where a masked tile holds an infinity or NaN)
  uint16_t* out;
  const int32_t* offsets;
  const int32_t* kv_lens;
  const int32_t* table;
  int32_t* cnt;             // [CTAs] arrivals at the item that begins in the CTA and is split (zero between calls)
  float* parts;             // [CTAs][2][rows of a tile][head_dim + 2]
  int* err;
  int64_t q_stride, tokens, pages;
  int32_t n_seqs, width, page_shift, q_heads, kv_heads, group;
  int32_t min_rows, max_rows;   // sequences with that many rows (new tokens x query heads a key head) are this kernel's
  int32_t zero_rest;            // no other kernel runs: zeros for the tokens of sequences above max_rows, and of none
  float scale_log2;             // |scale| log2(e)
  int32_t negate;               // scale < 0: the queries' signs are flipped
};

// attn_rows.cu: sequences of at most attn_rows_most() rows; rows: a bound of theirs
int attn_rows_most();
int attn_rows_box(int page_size);   // rows of a TMA box
int attn_rows_tile();               // keys of a unit
gs_status launch_attn_rows(const AttnParams& P, int head_dim, int rows, int ctas, cudaStream_t s);

// attn_chunk.cu: any number of rows
int attn_chunk_box(int page_size);
int attn_chunk_tile();
int attn_chunk_rows();              // rows of an item
gs_status launch_attn_chunk(const AttnParams& P, int head_dim, int ctas, cudaStream_t s);

struct SeqInfo {
  int tok0, n, rows;   // first new token, new tokens, rows
  int kv;              // length with the new tokens (not cut)
  int cap;             // keys that the page table can hold
  __device__ __forceinline__ int len() const { return max(0, min(kv, cap)); }
  // keys that token j sees
  __device__ __forceinline__ int seen(int j) const {
    const int64_t v = (int64_t)kv - n + j + 1;
    return v <= 0 ? 0 : v < cap ? (int)v : cap;
  }
};

__device__ __forceinline__ SeqInfo seq_info(const AttnParams& P, int r) {
  SeqInfo s;
  const int64_t a = max((int64_t)__ldg(P.offsets + r), (int64_t)0), b = min((int64_t)__ldg(P.offsets + r + 1), P.tokens);
  s.tok0 = (int)a;
  s.n = b > a ? (int)(b - a) : 0;
  const int64_t rows = (int64_t)s.n * P.group;
  s.rows = rows > INT32_MAX ? INT32_MAX : (int)rows;
  s.kv = __ldg(P.kv_lens + r);
  s.cap = P.width << P.page_shift;
  return s;
}

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// A bounded wait for barriers that complete within a microsecond or two: the clock and the
// abort flag are only looked at after many tries (a try itself waits for a while).
__device__ __forceinline__ bool mbar_wait_short(uint64_t* bar, uint32_t parity, volatile int* abort_flag, int* err,
                                                uint64_t limit_ns) {
#pragma unroll 1
  for (int i = 0; i < 64; ++i)
    if (sm100::mbar_try_wait(bar, parity)) return true;
  const uint64_t t0 = sm100::globaltimer_ns();
  while (true) {
#pragma unroll 1
    for (int i = 0; i < 64; ++i)
      if (sm100::mbar_try_wait(bar, parity)) return true;
    if (*abort_flag) return false;
    if (sm100::globaltimer_ns() - t0 > limit_ns) {
      *abort_flag = 1;
      atomicExch(err, kDevErrTimeout);
      return false;
    }
  }
}

// Units are counted in 32 bits (the host refuses steps that could have more).  Traits:
//   row_tiles(s, P)   tiles of rows of a sequence (0: not this kernel's)
//   tiles(s, P, rt)   units of row tile rt, at least 1
//   kLeast, kSnap     the least units worth a CTA; boundaries this close to an item's end move there
//   kOver             what an item costs beside its units, in units: they lie before its first one and hold no work
template <class Traits>
__device__ __forceinline__ int head_units(const AttnParams& P, const SeqInfo& s) {
  const int nr = Traits::row_tiles(s, P);
  int u = 0;
  for (int i = 0; i < nr; ++i) u += Traits::tiles(s, P, i) + Traits::kOver;
  return u;
}

// An item of a sequence: a key head and a row tile
struct Item {
  int h, rt, nt;       // nt: its units, kOver among them
  int first;           // its first unit, from the sequence's first
};
// the item that holds unit `off` of the sequence
template <class Traits>
__device__ __forceinline__ Item item_at(const AttnParams& P, const SeqInfo& s, int off, int per_head) {
  Item it;
  it.h = off / per_head;
  it.first = it.h * per_head;
  const int nr = Traits::row_tiles(s, P);
  for (it.rt = 0; it.rt < nr; ++it.rt) {
    it.nt = Traits::tiles(s, P, it.rt) + Traits::kOver;
    if (off < it.first + it.nt) break;
    it.first += it.nt;
  }
  return it;
}

// total units over `ctas` CTAs: CTA c begins at c share + min(c, rest)
struct Shares {
  int total, ctas, share, rest;
  // at least `least` units a CTA, unless there are CTAs for single items
  __device__ __forceinline__ Shares(int n, int items, int most, int least) {
    total = n;
    ctas = max(1, min(most, max((n + least - 1) / least, items)));
    share = n / ctas;
    rest = n - share * ctas;
  }
  __device__ __forceinline__ int cut(int c) const { return c >= ctas ? total : c * share + min(c, rest); }
  // the first boundary at or after unit v
  __device__ __forceinline__ int first_cut(int v) const {
    const int wide = rest * (share + 1);
    return v <= wide ? (v + share) / (share + 1) : rest + (v - wide + share - 1) / share;
  }
};

// Where a CTA begins and ends, in shared memory; written by divide_work.
struct WorkSlot {
  int at;         // the boundary, moved to an item's end where that is near
  int base;       // units before sequence r
  int r;          // the sequence that holds it (n_seqs: past the last)
  int per_head;   // and its units a key head
  SeqInfo s;
};
struct WorkShared {
  int sums[2][32];
  WorkSlot slot[2];
};

// Called by the whole block; afterwards every thread may read w.slot.  Boundaries within
// Traits::kSnap units of an item's ends move there: a part that short is not worth the
// cost of joining it.  Returns the division.
template <class Traits, int THREADS>
__device__ __forceinline__ Shares divide_work(const AttnParams& P, int cta, WorkShared& w) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  constexpr int kW = THREADS / 32;
  static_assert(kW <= 32 && THREADS % 32 == 0, "block");
  const bool one_pass = P.n_seqs <= THREADS;   // a sequence a thread
  SeqInfo mine;
  int per_head = 0, total = 0, items = 0;
  if (threadIdx.x < 2) w.slot[threadIdx.x].at = INT32_MAX;   // past the last: the total
  if (!one_pass) {
    int u = 0, n = 0;
    for (int r = threadIdx.x; r < P.n_seqs; r += THREADS) {
      mine = seq_info(P, r);
      u += head_units<Traits>(P, mine);
      n += Traits::row_tiles(mine, P);
    }
    u = __reduce_add_sync(0xffffffffu, u);
    n = __reduce_add_sync(0xffffffffu, n);
    if (lane == 0) {
      w.sums[0][warp] = u;
      w.sums[1][warp] = n;
    }
    __syncthreads();
    for (int i = 0; i < kW; ++i) {
      total += w.sums[0][i] * P.kv_heads;
      items += w.sums[1][i] * P.kv_heads;
    }
    __syncthreads();
  }
  int carry = 0;
  for (int r0 = 0; r0 < P.n_seqs; r0 += THREADS) {
    const int r = r0 + (int)threadIdx.x;
    per_head = 0;
    int n = 0;
    if (r < P.n_seqs) {
      mine = seq_info(P, r);
      per_head = head_units<Traits>(P, mine);
      n = Traits::row_tiles(mine, P);
    }
    const int u = per_head * P.kv_heads;
    int incl = u;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const int o = __shfl_up_sync(0xffffffffu, incl, d);
      if (lane >= d) incl += o;
    }
    n = __reduce_add_sync(0xffffffffu, n);
    if (lane == 31) {
      w.sums[0][warp] = incl;
      w.sums[1][warp] = n;
    }
    __syncthreads();
    int base = carry + incl - u;
    for (int i = 0; i < kW; ++i) {
      if (i < warp) base += w.sums[0][i];
      carry += w.sums[0][i];
      if (one_pass) items += w.sums[1][i] * P.kv_heads;
    }
    if (one_pass) total = carry;
    const Shares sh(total, items, (int)gridDim.x, Traits::kLeast);
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int off = sh.cut(min(cta + e, sh.ctas)) - base;
      if (off < 0 || off >= u) continue;
      const Item it = item_at<Traits>(P, mine, off, per_head);
      const int at = off - it.first <= Traits::kSnap + Traits::kOver ? it.first
                     : it.first + it.nt - off <= Traits::kSnap      ? it.first + it.nt
                                                                    : off;
      w.slot[e] = WorkSlot{base + at, base, r, per_head, mine};
    }
    __syncthreads();
    if (carry > sh.cut(min(cta + 1, sh.ctas))) break;   // both boundaries are behind
  }
  return Shares(total, items, (int)gridDim.x, Traits::kLeast);
}

// A stretch of one item's units in a CTA.
struct Segment {
  SeqInfo s;
  int h, rt;           // key head, row tile
  int r;
  int ta, tb;          // the item's units [ta, tb)
  int parts, part;     // parts of the item, and which one this is
  int first_cta;       // the CTA of part 0
};

template <class Traits>
struct Walker {
  const AttnParams& P;
  const Shares sh;
  int cta, pos, end, base, per_head, r;
  SeqInfo s;
  __device__ __forceinline__ Walker(const AttnParams& p, const Shares& shares, const WorkShared& w, int c)
      : P(p), sh(shares), cta(c) {
    pos = min(w.slot[0].at, sh.total);
    end = min(w.slot[1].at, sh.total);
    base = w.slot[0].base;
    r = w.slot[0].r;
    per_head = w.slot[0].per_head;
    s = w.slot[0].s;
  }
  __device__ __forceinline__ bool next(Segment& g) {
    if (pos >= end) return false;
    while (pos >= base + per_head * P.kv_heads) {   // `end` lies inside some sequence, so r stays in range
      base += per_head * P.kv_heads;
      if (++r >= P.n_seqs) return false;
      s = seq_info(P, r);
      per_head = head_units<Traits>(P, s);
    }
    g.s = s;
    g.r = r;
    const Item it = item_at<Traits>(P, s, pos - base, per_head);
    g.h = it.h;
    g.rt = it.rt;
    const int first = base + it.first, last = first + it.nt, stop = min(last, end);
    g.ta = max(0, pos - first - Traits::kOver);
    g.tb = stop - first - Traits::kOver;
    g.parts = 1;
    g.part = 0;
    g.first_cta = cta;
    if (pos != first || stop != last) {
      // the boundaries inside the item that were not moved to its ends
      const int c_lo = sh.first_cut(first + Traits::kSnap + Traits::kOver + 1), c_hi = sh.first_cut(last - Traits::kSnap) - 1;
      g.first_cta = c_lo - 1;
      g.parts = c_hi - c_lo + 2;
      g.part = cta - g.first_cta;
    }
    pos = stop;
    return true;
  }
};

// Zeros for the tokens of no sequence, and (large) of sequences above max_rows, by one warp of every CTA.
__device__ __forceinline__ void zero_rows(const AttnParams& P, int head_dim, int cta, int lane, bool large) {
  const int64_t row16 = (int64_t)P.q_heads * head_dim / 8;   // 16-byte pieces of a token's output
  const auto zero = [&](int64_t t0, int64_t t1) {
    for (int64_t i = t0 * row16 + lane; i < t1 * row16; i += 32) reinterpret_cast<uint4*>(P.out)[i] = make_uint4(0u, 0u, 0u, 0u);
  };
  const int64_t before = min((int64_t)max(0, __ldg(P.offsets)), P.tokens), after = max(0, __ldg(P.offsets + P.n_seqs));
  for (int64_t t = cta; t < before; t += gridDim.x) zero(t, t + 1);
  for (int64_t t = after + cta; t < P.tokens; t += gridDim.x) zero(t, t + 1);
  for (int r = cta; large && r < P.n_seqs; r += (int)gridDim.x) {
    const SeqInfo s = seq_info(P, r);
    if (s.rows > P.max_rows) zero(s.tok0, (int64_t)s.tok0 + s.n);
  }
}

// Where part `part` of a split item lies: a CTA holds at most one part of an item that
// began before it, and at most one of an item that goes on after it.
__device__ __forceinline__ float* part_slot(const AttnParams& P, int first_cta, int part, int rows, int head_dim) {
  return P.parts + ((int64_t)(first_cta + part) * 2 + (part == 0 ? 1 : 0)) * rows * (head_dim + 2);
}

}  // namespace gs
