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
  const uint16_t* k;
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
  int32_t zero_rest;            // write zeros for the sequences above max_rows (no other kernel runs)
  float scale_log2;             // |scale| log2(e)
  int32_t negate;               // scale < 0: the queries' signs are flipped
};

// attn_rows.cu: sequences of at most attn_rows_most() rows; rows: a bound of theirs
int attn_rows_most();
int attn_rows_box(int page_size);   // rows of a TMA box
gs_status launch_attn_rows(const AttnParams& P, int head_dim, int rows, int ctas, cudaStream_t s);

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

// Tiles of an item, and where the items of a sequence lie.  Traits:
//   kTile                                keys of a unit
//   row_tiles(s, P)                      tiles of rows of a sequence (0: not this kernel's)
//   tiles(s, P, rt)                      units of row tile rt, at least 1
struct WorkSlot {   // a boundary between two CTAs
  int64_t base;     // units before sequence r
  int r;
};

// A CTA's share, the same for every thread.
struct WorkRange {
  int64_t total;   // units of the step
  int64_t begin, end;
  int64_t base;    // units before sequence r, which holds `begin`
  int r;
  int ctas;        // that share the units
  int snap;
};

// Boundaries closer than this to an item's ends move there: a part shorter than the
// cost of joining it is not worth its parallelism.  Where shares are long, a shift of
// two units is small beside them; where they are short, joining costs more than four.
__device__ __forceinline__ int snap_units(int64_t total, int ctas) { return total >= (int64_t)16 * ctas ? 2 : 4; }

template <class Traits>
__device__ __forceinline__ int64_t seq_units(const AttnParams& P, const SeqInfo& s) {
  const int nr = Traits::row_tiles(s, P);
  int64_t u = 0;
  for (int i = 0; i < nr; ++i) u += Traits::tiles(s, P, i);
  return u * P.kv_heads;
}

// The item of sequence s that holds unit `off` (counted from the sequence's first)
struct Item {
  int h, rt, nt;       // key head, row tile, units
  int64_t first;       // its first unit, from the sequence's first
};
template <class Traits>
__device__ __forceinline__ Item item_at(const AttnParams& P, const SeqInfo& s, int64_t off, int64_t per_head) {
  Item it;
  it.h = (int)(off / per_head);
  it.first = it.h * per_head;
  const int nr = Traits::row_tiles(s, P);
  for (it.rt = 0; it.rt < nr; ++it.rt) {
    it.nt = Traits::tiles(s, P, it.rt);
    if (off < it.first + it.nt) break;
    it.first += it.nt;
  }
  return it;
}

// Called by the whole block.  red: [34] int64 of shared memory; slots: [2].
template <class Traits, int THREADS>
__device__ __forceinline__ WorkRange divide_work(const AttnParams& P, int cta, int ctas, int64_t* red, WorkSlot* slots) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  constexpr int kW = THREADS / 32;
  static_assert(kW <= 32 && THREADS % 32 == 0, "block");
  int64_t sum = 0;
  for (int r = threadIdx.x; r < P.n_seqs; r += THREADS) sum += seq_units<Traits>(P, seq_info(P, r));
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
  if (lane == 0) red[warp] = sum;
  if (threadIdx.x < 2) slots[threadIdx.x] = WorkSlot{0, P.n_seqs};
  __syncthreads();
  WorkRange w;
  w.total = 0;
  for (int i = 0; i < kW; ++i) w.total += red[i];
  // four units at least: a shorter share would end before its part is joined
  const int64_t most = (w.total + 3) / 4;
  w.ctas = (int)min((int64_t)ctas, max(most, (int64_t)1));
  w.snap = snap_units(w.total, w.ctas);
  const int64_t cut[2] = {min(cta, w.ctas) * w.total / w.ctas, min(cta + 1, w.ctas) * w.total / w.ctas};
  __syncthreads();
  int64_t carry = 0;
  for (int r0 = 0; r0 < P.n_seqs && carry <= cut[1]; r0 += THREADS) {
    const int r = r0 + (int)threadIdx.x;
    const int64_t u = r < P.n_seqs ? seq_units<Traits>(P, seq_info(P, r)) : 0;
    int64_t incl = u;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const int64_t o = __shfl_up_sync(0xffffffffu, incl, d);
      if (lane >= d) incl += o;
    }
    if (lane == 31) red[warp] = incl;
    __syncthreads();
    int64_t before = carry;
    for (int i = 0; i < kW; ++i) {
      if (i < warp) before += red[i];
      carry += red[i];
    }
    const int64_t base = before + incl - u;
#pragma unroll
    for (int e = 0; e < 2; ++e)
      if (cut[e] >= base && cut[e] < base + u) slots[e] = WorkSlot{base, r};
    __syncthreads();
  }
  int64_t at[2];
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    at[e] = cut[e];
    const WorkSlot sl = slots[e];
    if (sl.r < P.n_seqs) {
      const SeqInfo s = seq_info(P, sl.r);
      const int64_t off = cut[e] - sl.base;
      const Item it = item_at<Traits>(P, s, off, seq_units<Traits>(P, s) / P.kv_heads);
      if (off - it.first <= w.snap) at[e] = sl.base + it.first;
      else if (it.first + it.nt - off <= w.snap) at[e] = sl.base + it.first + it.nt;
    }
  }
  w.begin = at[0];
  w.end = at[1];
  w.r = slots[0].r;
  w.base = slots[0].base;
  return w;
}

// A stretch of one item's units in a CTA.
struct Segment {
  SeqInfo s;
  Item it;
  int r;
  int ta, tb;          // its units [ta, tb) of the item's nt
  int parts, part;     // parts of the item, and which one this is
  int first_cta;       // the CTA of part 0
};

template <class Traits>
struct Walker {
  const AttnParams& P;
  WorkRange w;
  int64_t pos, base, units;
  int r;
  SeqInfo s;
  __device__ __forceinline__ Walker(const AttnParams& p, const WorkRange& range)
      : P(p), w(range), pos(range.begin), base(range.base), r(range.r) {
    units = 0;
    if (pos < w.end) {
      s = seq_info(P, r);
      units = seq_units<Traits>(P, s);
    }
  }
  __device__ __forceinline__ bool next(Segment& g, int cta) {
    if (pos >= w.end) return false;
    while (pos >= base + units) {   // `end` lies inside some sequence, so r stays in range
      base += units;
      if (++r >= P.n_seqs) return false;
      s = seq_info(P, r);
      units = seq_units<Traits>(P, s);
    }
    g.s = s;
    g.r = r;
    g.it = item_at<Traits>(P, s, pos - base, units / P.kv_heads);
    const int64_t first = base + g.it.first, last = first + g.it.nt;
    g.ta = (int)(pos - first);
    g.tb = (int)(min(last, w.end) - first);
    pos = first + g.tb;
    // the boundaries floor(c total / ctas) inside the item that were not moved to its ends
    const int64_t lo = first + w.snap + 1, hi = last - w.snap;
    const int64_t c_lo = (lo * w.ctas + w.total - 1) / w.total, c_hi = (hi * w.ctas + w.total - 1) / w.total - 1;
    if (g.ta == 0 && g.tb == g.it.nt) {
      g.parts = 1;
      g.part = 0;
      g.first_cta = cta;
    } else {
      g.first_cta = (int)c_lo - 1;
      g.parts = (int)(c_hi - c_lo) + 2;
      g.part = cta - g.first_cta;
    }
    return true;
  }
};

// Where part `part` of a split item lies: a CTA holds at most one part of an item that
// began before it, and at most one of an item that goes on after it.
__device__ __forceinline__ float* part_slot(const AttnParams& P, int first_cta, int part, int rows, int head_dim) {
  return P.parts + ((int64_t)(first_cta + part) * 2 + (part == 0 ? 1 : 0)) * rows * (head_dim + 2);
}

}  // namespace gs
