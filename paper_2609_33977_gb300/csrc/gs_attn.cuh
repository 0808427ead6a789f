// What the two attention kernels share: parameters, the division of a step's work
// over the CTAs, and the joining of a split item's parts.
//
// Work is counted in units (one tile of keys against one tile of rows), laid out
// sequence by sequence, and every CTA takes an equal share of consecutive units, so
// a step of any mix of lengths ends everywhere at the same time.  An item (a
// sequence, a key head, a tile of rows) that lies across CTAs is split: each part
// leaves (m, l, o) in the workspace, and the CTA that arrives last joins them in
// order, in two levels where there are many (join_step).  Lengths are read from device
// memory, by every CTA for itself.
#pragma once

#include "gs_block.cuh"
#include "gs_sm100.cuh"

#include <cuda.h>

namespace gs {

struct AttnParams {
  CUtensorMap kmap, vmap;   // (64, rows, head_dim / 64) slabs over [pages * kv_heads * page_size][head_dim]
  CUtensorMap qmap;         // chunk kernel: [tokens][q_heads][head_dim], boxes of half_tokens x group x 64
  const uint16_t* q;
  const uint16_t* v;        // the value pages (re-read where a masked tile holds an infinity or NaN)
  uint16_t* out;
  const int32_t* offsets;
  const int32_t* kv_lens;
  const int32_t* table;
  int32_t* cnt;             // [2][CTAs] arrivals (a half of the item each in the chunk kernel) at the group of parts, and at the
                            // split item, that begin in the CTA; zero between calls
  float* parts;             // [CTAs][2] parts
  int* err;
  uint64_t inject_ns;       // test hook: CTA 0 waits so long on a word that nothing sets, in place of its copies (0: off)
  int64_t q_stride, tokens, pages;
  int32_t n_seqs, width, page_shift, q_heads, kv_heads, group;
  uint32_t group_inv;       // floor((2^32 - 1) / group)
  int32_t half_tokens;      // chunk kernel: whole tokens in 128 rows
  int32_t min_rows, max_rows;   // sequences with that many rows (new tokens x query heads a key head) are this kernel's
  int32_t zero_rest;            // no other kernel runs: zeros for the tokens of sequences above max_rows, and of none
  int32_t two_launches;         // chunk kernel: lets the few-row launch behind it begin on SMs that are through; that one: waits
                                // for it at its end, so that whatever follows does too
  float scale_log2;             // |scale| log2(e)
  int32_t negate;               // scale < 0: the queries' signs are flipped
};

// attn_rows.cu: sequences of at most P.max_rows rows, one of the numbers that the kernel's forms hold
int attn_rows_most();
int attn_rows_part(int head_dim);   // floats of a part in the workspace, at most
int attn_rows_held(int rows);       // the least of these numbers that is at least `rows`
int attn_rows_box(int page_size);   // rows of a TMA box
int attn_rows_tile();               // keys of a unit
gs_status launch_attn_rows(const AttnParams& P, int head_dim, int ctas, cudaStream_t s);

// attn_chunk.cu: any number of rows
int attn_chunk_box(int page_size);
int attn_chunk_tile();
int attn_chunk_half_tokens(int group);   // tokens of half an item
int attn_chunk_rows();                   // an item has more rows than this, but for a sequence's last
int attn_chunk_part(int head_dim);       // floats of a part in the workspace
int attn_most_over();                    // what an item costs beside its units, in units, at most
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

// row / group for row >= 0: the quotient by the rounded-down inverse is short by one at most
__device__ __forceinline__ int row_token(const AttnParams& P, int row) {
  int q = (int)__umulhi((uint32_t)row, P.group_inv);
  if (row - q * P.group >= P.group) ++q;
  return q;
}

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// A whole warp's bounded wait, the same answer for all lanes: at most kWaitTries tries of
// up to a microsecond (0.1 s or more in all, 2 s at most), after which the block's abort
// flag is up and every wait ends.  Short code: it is inlined wherever a warp waits, and the
// kernels' loops share the instruction cache with it.
constexpr int kWaitTries = 2000000;
__device__ __forceinline__ bool mbar_wait_warp(uint64_t* bar, uint32_t parity, volatile int* abort_flag) {
#pragma unroll 1
  for (int left = kWaitTries; !__all_sync(0xffffffffu, sm100::mbar_try_wait_sleep(bar, parity, 1000u)); --left) {
    if (left == 0) *abort_flag = 1;
    if (__any_sync(0xffffffffu, *abort_flag != 0)) return false;
  }
  return true;
}
// Test hook, for the warp that a CTA's work begins with: waits on a word that nothing sets (the one after the error
// flag) until the limit, then gives up like every wait that runs out.
__device__ __forceinline__ bool injected_timeout(const AttnParams& P, int cta, volatile int* abort_flag) {
  if (P.inject_ns == 0 || cta != 0) return false;
  const volatile int* never = P.err + 1;
  const uint64_t t0 = sm100::globaltimer_ns();
  bool out = false;
  while (!out && *never == 0) {
    out = sm100::globaltimer_ns() - t0 > P.inject_ns;
    __nanosleep(1000);
  }
  out = __any_sync(0xffffffffu, out);
  if (out) *abort_flag = 1;
  return out;
}
// At a kernel's end, after a block barrier: records that some wait ran out, and gives
// copies in flight time to land.
__device__ __forceinline__ void end_of_waits(volatile int* abort_flag, int* err) {
  if (!*abort_flag) return;
  if (threadIdx.x == 0) atomicExch(err, kDevErrTimeout);
  const uint64_t t0 = sm100::globaltimer_ns();
  while (sm100::globaltimer_ns() - t0 < 2000000ull) {
  }
}
// A value that all lanes share, known as such to the compiler
__device__ __forceinline__ int uniform(int v) { return (int)__reduce_max_sync(0xffffffffu, (uint32_t)v); }

// Units are counted in 32 bits (the host refuses steps that could have more).  Traits:
//   row_tiles(s, P)   tiles of rows of a sequence (0: not this kernel's)
//   tiles(s, P, rt)   units of row tile rt, at least 1
//   kLeast, kSnap     the least units worth a CTA; boundaries this close to an item's end move there
//   kOneTile          no sequence has more than one tile of rows
//   kOver             what an item costs beside its units, in units: they lie before its first one and hold no work
//
// Units of a key head of one sequence per lane (a warp; on: the lane has one).  Long
// sequences, of many row tiles, are summed by the whole warp one after another.
template <class Traits>
__device__ __forceinline__ int head_units(const AttnParams& P, const SeqInfo& s, bool on) {
  const int lane = threadIdx.x & 31;
  const int nr = on ? Traits::row_tiles(s, P) : 0;
  int u = 0;
  if (nr <= 2)
#pragma unroll 1
    for (int i = 0; i < nr; ++i) u += Traits::tiles(s, P, i) + Traits::kOver;
  if constexpr (!Traits::kOneTile) {
    for (uint32_t many = __ballot_sync(0xffffffffu, nr > 2); many; many &= many - 1) {
      const int src = __ffs(many) - 1, n = __shfl_sync(0xffffffffu, nr, src);
      SeqInfo t;
      t.tok0 = 0;
      t.n = __shfl_sync(0xffffffffu, s.n, src);
      t.rows = __shfl_sync(0xffffffffu, s.rows, src);
      t.kv = __shfl_sync(0xffffffffu, s.kv, src);
      t.cap = __shfl_sync(0xffffffffu, s.cap, src);
      int part = 0;
#pragma unroll 1
      for (int i = lane; i < n; i += 32) part += Traits::tiles(t, P, i) + Traits::kOver;
      part = __reduce_add_sync(0xffffffffu, part);
      if (lane == src) u = part;
    }
  }
  return u;
}

// An item of a sequence: a key head and a row tile
struct Item {
  int h, rt, nt;       // nt: its units, kOver among them
  int first;           // its first unit, from the sequence's first
};
// the item that holds unit `off` of the sequence, looked up by a whole warp
template <class Traits>
__device__ __forceinline__ Item item_at(const AttnParams& P, const SeqInfo& s, int off, int per_head) {
  const int lane = threadIdx.x & 31;
  Item it;
  it.h = off / per_head;
  it.first = it.h * per_head;
  it.rt = 0;
  if constexpr (Traits::kOneTile) {
    it.nt = per_head;
    return it;
  }
  const int nr = Traits::row_tiles(s, P);
  while (true) {
    const int mine = it.rt + lane < nr ? Traits::tiles(s, P, it.rt + lane) + Traits::kOver : 0;
    int incl = mine;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const int o = __shfl_up_sync(0xffffffffu, incl, d);
      if (lane >= d) incl += o;
    }
    const uint32_t past = __ballot_sync(0xffffffffu, it.first + incl > off);   // the first of these lanes has it
    if (past) {
      const int src = __ffs(past) - 1;
      it.rt += src;
      it.nt = __shfl_sync(0xffffffffu, mine, src);
      it.first += __shfl_sync(0xffffffffu, incl - mine, src);
      return it;
    }
    it.first += __shfl_sync(0xffffffffu, incl, 31);
    it.rt += 32;
    if (it.rt >= nr) return it;   // not reached: off lies in the head
  }
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
  int r;          // the sequence that holds it; n_seqs: it is the end of all
  int per_head;   // the sequence's units a key head
  Item it;        // the item that holds it
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
  static_assert(kW >= 2 && kW <= 32 && THREADS % 32 == 0, "block");
  const bool one_pass = P.n_seqs <= THREADS;   // a sequence a thread: looked at once
  SeqInfo mine = {0, 0, 0, 0, 0};
  int per_head = 0, base = 0, items = 0;
  Shares sh(0, 0, 1, 1);
  if (threadIdx.x < 2) w.slot[threadIdx.x].r = P.n_seqs;
  // first the sums, then the sequences that hold this CTA's boundaries
#pragma unroll 1
  for (int pass = 0; pass < 2; ++pass) {
    int carry = 0;
#pragma unroll 1
    for (int r0 = 0; r0 < P.n_seqs; r0 += THREADS) {
      const int r = r0 + (int)threadIdx.x;
      if (pass == 0 || !one_pass) {
        const bool on = r < P.n_seqs;
        if (on) mine = seq_info(P, r);
        per_head = head_units<Traits>(P, mine, on);
        const int n = __reduce_add_sync(0xffffffffu, on ? Traits::row_tiles(mine, P) : 0);
        int incl = per_head * P.kv_heads;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
          const int o = __shfl_up_sync(0xffffffffu, incl, d);
          if (lane >= d) incl += o;
        }
        if (lane == 31) {
          w.sums[0][warp] = incl;
          w.sums[1][warp] = n;
        }
        __syncthreads();
        const int sum = lane < kW ? w.sums[0][lane] : 0;
        base = carry + __reduce_add_sync(0xffffffffu, lane < warp ? sum : 0) + incl - per_head * P.kv_heads;
        carry += __reduce_add_sync(0xffffffffu, sum);
        if (pass == 0) items += __reduce_add_sync(0xffffffffu, lane < kW ? w.sums[1][lane] : 0) * P.kv_heads;
        if (!one_pass) __syncthreads();   // the sums are written again
      }
      if (pass == 1) {
#pragma unroll 1
        for (int e = 0; e < 2; ++e) {
          const int off = sh.cut(min(cta + e, sh.ctas)) - base;
          if (off >= 0 && off < per_head * P.kv_heads) {
            w.slot[e].r = r;
            w.slot[e].base = base;
            w.slot[e].per_head = per_head;
            w.slot[e].s = mine;
          }
        }
      }
    }
    if (pass == 0) sh = Shares(carry, items, (int)gridDim.x, Traits::kLeast);
  }
  __syncthreads();
  if (warp < 2) {   // a warp a boundary
    WorkSlot& sl = w.slot[warp];
    const int cut = sh.cut(min(cta + warp, sh.ctas));
    int at = cut;
    Item it = {0, 0, 0, 0};
    if (sl.r < P.n_seqs) {
      const int off = cut - sl.base;
      it = item_at<Traits>(P, sl.s, off, sl.per_head);
      if (off - it.first <= Traits::kSnap + Traits::kOver) at = sl.base + it.first;
      else if (it.first + it.nt - off <= Traits::kSnap) at = sl.base + it.first + it.nt;
    }
    __syncwarp();
    if (lane == 0) {
      sl.at = at;
      sl.it = it;
    }
  }
  __syncthreads();
  return sh;
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

// The segments of a CTA, one after another; for a whole warp.
template <class Traits>
struct Walker {
  const AttnParams& P;
  const Shares sh;
  int cta, pos, end, first, r;   // first: the item's first unit
  int nr;                        // row tiles of the sequence
  Item it;
  SeqInfo s;
  __device__ __forceinline__ Walker(const AttnParams& p, const Shares& shares, const WorkShared& w, int c)
      : P(p), sh(shares), cta(c) {
    pos = w.slot[0].at;
    end = w.slot[1].at;
    it = w.slot[0].it;
    r = w.slot[0].r;
    s = w.slot[0].s;
    first = w.slot[0].base + it.first;
    nr = pos < end ? Traits::row_tiles(s, P) : 0;
  }
  __device__ __forceinline__ bool next(Segment& g) {
    if (pos >= end) return false;
    while (pos >= first + it.nt) {   // the next item: row tiles, then key heads, then sequences
      first += it.nt;
      if (++it.rt >= nr) {
        it.rt = 0;
        if (++it.h >= P.kv_heads) {
          it.h = 0;
          do {
            if (++r >= P.n_seqs) return false;   // not reached: `end` lies inside some sequence
            s = seq_info(P, r);
            nr = Traits::row_tiles(s, P);
          } while (nr == 0);
        }
      }
      it.nt = Traits::tiles(s, P, it.rt) + Traits::kOver;
    }
    g.s = s;
    g.r = r;
    g.h = it.h;
    g.rt = it.rt;
    const int last = first + it.nt, stop = min(last, end);
    g.ta = max(0, pos - first - Traits::kOver);
    g.tb = stop - first - Traits::kOver;
    g.parts = 1;
    g.part = 0;
    g.first_cta = cta;
    if (pos != first || stop != last) {
      // the boundaries inside the item that were not moved to its ends
      const int c_lo = sh.first_cut(first + Traits::kSnap + Traits::kOver + 1), c_hi = sh.first_cut(last - Traits::kSnap) - 1;
      g.first_cta = max(0, min(c_lo - 1, cta));
      g.parts = max(1, min(c_hi - c_lo + 2, sh.ctas - g.first_cta));   // whatever the offsets, inside the workspace
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
#pragma unroll 1
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
__device__ __forceinline__ float* part_slot(const AttnParams& P, int first_cta, int part, int size) {
  return P.parts + ((int64_t)(first_cta + part) * 2 + (part == 0 ? 1 : 0)) * size;
}

// The two levels in which a split item's parts are joined: groups of neighbouring parts, each
// into its first one's place, then the groups into the output.  One CTA joining all P parts
// reads them one behind the other; groups of sqrt(P) are joined by as many CTAs at once.
// Up to `flat` parts are one group.  A group of two or more crosses the end of its first
// CTA's share, and so does an item of two or more: no other has its counter there.
struct JoinStep {
  int first, n, stride;   // parts first, first + stride, ...
  bool last;              // the output follows
};
__device__ __forceinline__ JoinStep join_step(const Segment& g, int level, int flat) {
  int size = g.parts;
  if (size > flat)
#pragma unroll 1
    for (size = 2; size * size < g.parts; ++size) {
    }
  JoinStep j;
  const int groups = (g.parts + size - 1) / size;
  j.first = level == 0 ? g.part - g.part % size : 0;
  j.n = level == 0 ? min(size, g.parts - j.first) : groups;
  j.stride = level == 0 ? 1 : size;
  j.last = level == 1 || groups == 1;
  return j;
}

}  // namespace gs
