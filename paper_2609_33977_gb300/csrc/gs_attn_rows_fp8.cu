// Attention of few rows (new tokens x query heads a key head, at most 32, or 64 in two row
// tiles) over a cache in 8 bits: decoding steps and short chunks.
//
// Bound by HBM, at half the bytes a key of a bf16 cache, so that a key's share of the
// arithmetic counts twice as much.  Keys are the long side of both products (m16n8k16 with
// 16 keys, then 16 channels, as its rows and 8 query rows as its columns), so up to 8 rows
// cost half the instructions that 16 do:
//     S^T = K Q^T,   l = sum exp2(c S - m),   O^T = V^T P^T,   P = exp2(c S + e - M + 6).
// Codes become f16 on their way into the fragments (exactly), two at a time; a key's power
// multiplies its scores in float32.  Queries are moved to f16 by a power of two a row.
// The power 2^e of a value is added to the exponent of its weight, and the numerators have a
// running maximum M of their own beside the softmax's m: the largest of weight times power
// is what P in f16 is counted from, not the largest power, whose key may weigh nothing.  P keeps
// 11 bits: it loses 2^-11 of itself at most, or, below 2^-20 of that largest one, 2^-31 of it.  O's
// unit 2^M goes with its part as an exponent, and is applied after the division by l, so that
// no sum leaves float32's range.  The maxima in use are raised only when a weight or a numerator
// passes 2^8 (a vote instead of an exchange between the lanes that hold a row's keys), so l is at least 1.
// A value of no visible key has weight 0 whatever its power, so a NaN stays with the rows that see it.
//
// A unit is 256 keys of a key head, 64 for each of four pairs of computing warps, and a pair
// has a fetching warp and a ring of its own (TMA, a box a page and operand; 192 KB in all):
// a box costs its warp 80 cycles whatever its size, and pairs need not wait for one another
// before the segment's end.  There a warp's part lies in the last slot, where its own keys
// were.  Up to 16 rows, the two warps of a pair share its keys (tiles of 8 rows: one or two, by
// the segment's own rows); above, its rows.
//
// 16 sequences of 90 to 4000 keys, 32 heads: 43.7 us, 4.9 TB/s (in an earlier form nothing computed 40.3, and parts of split
// items not joined 36.7).  Three of 30001 to 65536 keys, 28/4 heads: 34.6 us, 4.3 TB/s; one of 60000: 24.0; four tokens there
// 38.2.  One of 129 keys: 6.6 us.  24 of 2 to 16000 keys with 2 to 4 new tokens, 16/2 heads of 64: 20.8 us.  Scores that keep
// passing the maximum cost more (keys' heads of sizes 2^-3 to 2^3 at random: 16 x 32 tokens at 2000 keys 124 us, else 103).   With 16 rows as the
// products' rows instead, and one ring for all warps, the first three took 59.9, 40.8 and (129 keys) 7.8.
#include "gs_attn_rows.cuh"

#include <algorithm>
#include <type_traits>

namespace gs {
namespace {
using namespace sm100;

constexpr int kPairs = 4, kSlotKeys = 64;
constexpr int kRingBytes = 192 * 1024;   // of all pairs
constexpr int kTile = kPairs * kSlotKeys;

// Rows of row tile rt of a sequence
__device__ __forceinline__ int tile_rows(const SeqInfo& s, int rt) { return min(kMost, s.rows - kMost * rt); }
// Units of a tile of keys.  Above 16 rows a tile takes about twice as long, and a CTA that has such ones among others ends late:
// 12 sequences of 1 to 4 tokens at 9192 to 32739 keys, 28/4 heads, 63 us, 91 without.  Where all row tiles are alike (known
// from the sizes alone) nothing is to be weighed: four tokens at 60000 keys 36.7 us, 39.2 with (then).
__device__ __forceinline__ int tile_units(const AttnParams& P, const SeqInfo& s, int rt) {
  return tile_rows(s, rt) > 16 && (!P.even || (s.rows > kMost && s.rows <= kMost + 16)) ? 2 : 1;
}

// A segment's first row
template <bool kTwo>
__device__ __forceinline__ int row0(const Segment& g) {
  return kTwo ? kMost * g.rt : 0;
}

// kTwo: sequences of up to two row tiles (the division of work takes 0.3 us longer)
template <bool kTwo>
struct FewTraits {
  static constexpr int kLeast = 4, kSnap = 1, kOver = 1;
  static constexpr bool kOneTile = !kTwo;
  static __device__ __forceinline__ int row_tiles(const SeqInfo& s, const AttnParams& P) {
    return s.rows >= P.min_rows && s.rows <= P.max_rows ? (kTwo && s.rows > kMost ? 2 : 1) : 0;
  }
  static __device__ __forceinline__ int tiles(const SeqInfo& s, const AttnParams& P, int rt) {
    return max(1, (s.len() + kTile - 1) / kTile) * tile_units(P, s, rt);
  }
};

__device__ __forceinline__ void mma16816(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
// the codes of the lower / upper two bytes, as f16
__device__ __forceinline__ uint32_t f16_of_lo(uint32_t codes) {
  uint32_t r;
  asm("{\n\t.reg .b16 lo, hi;\n\tmov.b32 {lo, hi}, %1;\n\tcvt.rn.f16x2.e4m3x2 %0, lo;\n\t}" : "=r"(r) : "r"(codes));
  return r;
}
__device__ __forceinline__ uint32_t f16_of_hi(uint32_t codes) {
  uint32_t r;
  asm("{\n\t.reg .b16 lo, hi;\n\tmov.b32 {lo, hi}, %1;\n\tcvt.rn.f16x2.e4m3x2 %0, hi;\n\t}" : "=r"(r) : "r"(codes));
  return r;
}
// an 8 x 8 matrix of 16-bit elements, a row in four lanes, transposed
__device__ __forceinline__ uint32_t transposed(uint32_t v) {
  uint32_t r;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
  return r;
}
// 2^(exponent field - 127)
__device__ __forceinline__ float power_of(int field) { return __uint_as_float((uint32_t)field << 23); }
__device__ __forceinline__ float power_or_nan(uint32_t code) { return __uint_as_float(code == 255u ? 0x7FC00000u : code << 23); }
// log2 of a power of two (-inf of 0)
__device__ __forceinline__ float lg2(float x) {
  float y;
  asm("lg2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// the larger of each half, numbers before NaN
__device__ __forceinline__ uint32_t max_f16x2(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("max.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
// What O's sums are multiplied by, one after the other: 1 / l and half of the unit's exponent, then the other half.  (At once
// 2^(M - m) may leave float32's range where the result does not.)  M is -inf where no value has a power: O is 0, or NaN.
__device__ __forceinline__ float2 back_from(float m, float l, float M, bool seen) {
  const float f = M == -INFINITY ? 0.f : ex2(0.5f * (M - m) - 3.f);
  return seen ? make_float2(f / l, f) : make_float2(0.f, 0.f);
}
__device__ __forceinline__ void arrive_by(uint64_t* bar, uint32_t count) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0], %1;" ::"r"(smem_u32(bar)), "r"(count) : "memory");
}
// over the lanes that hold other keys of the same rows
__device__ __forceinline__ float keys_max(float v) {
#pragma unroll
  for (int d = 4; d < 32; d <<= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, d));
  return v;
}
__device__ __forceinline__ float keys_sum(float v) {
#pragma unroll
  for (int d = 4; d < 32; d <<= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
  return v;
}

// Parts joined in one level.  (Three sequences of 30001 to 65536 keys, up to 18 parts: two levels cost 1.6 us more; one token at
// 60000 keys, 38 parts: one level 1.5 more than two.)
constexpr int kFlatFp8 = 32;

// 16 bytes from L2 to shared memory
__device__ __forceinline__ void copy16_l2(void* dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_u32(dst)), "l"(src) : "memory");
}
// An arrival, after all that this thread has seen written, and before all that it reads then
__device__ __forceinline__ int arrive_at(int32_t* cnt) {
  int before;
  asm volatile("atom.add.acq_rel.gpu.global.s32 %0, [%1], 1;" : "=r"(before) : "l"(cnt) : "memory");
  return before;
}

// The parts of the CTA's split items (up to two), joined at its end in join_step's levels: the last CTA that comes to a group
// joins it, in order.  (At the end of each segment, which stops the computing warps for two trips to L2: 16 sequences of 90 to
// 4000 keys, 32 heads 45.6 us, three of 30001 to 65536 36.6.)  Code that runs once a launch waits for its instructions more than
// for its data, so it is short: loops, through the warp's share of the ring's memory, which nothing else uses by then.  (A row a
// warp at a time, its parts' factors by shuffles: four tokens at 60000 keys 4.4 us more, 24 sequences of narrow heads 2.5.)
template <int D, bool kTwo, int ROWS, int WARPS, class Meet>
__device__ __forceinline__ void join_late(const AttnParams& P, const Segment* late, int n, int warp, int lane, int* last_s, uint8_t* room,
                                          Meet meet) {
  constexpr int kPart = ROWS * (D + kPartPad), kPieces = D / 4, kMlBytes = 4 * kFlatFp8 * 16;
  constexpr int kChunk = (kRingBytes / WARPS - kMlBytes) / (4 * D * 4);   // parts at a time, of four rows
  bool on[2] = {n > 0, n > 1};
#pragma unroll 1
  for (int level = 0; level < 2 && (on[0] || on[1]); ++level) {
    if (!meet()) return;   // `late` is written, and so are the parts
    const JoinStep j0 = join_step(late[0], level, kFlatFp8), j1 = join_step(late[n - 1], level, kFlatFp8);
    if (threadIdx.x < 2 && on[threadIdx.x]) {
      const Segment& g = late[threadIdx.x];
      const JoinStep j = threadIdx.x ? j1 : j0;
      int last = 1;   // a group of its own: the next level
      if (j.n > 1) {
        int32_t* cnt = P.cnt + level * (int)gridDim.x + g.first_cta + j.first;
        last = arrive_at(cnt) == j.n - 1;
        if (last) *cnt = 0;
      }
      last_s[threadIdx.x] = last;
    }
    if (!meet()) return;
    for (int i = 0; i < 2; ++i) on[i] = on[i] && last_s[i] != 0;
    const int rows0 = on[0] ? late[0].s.rows : 0, rows = rows0 + (on[1] ? late[1].s.rows : 0);
    // A row is one of 8, 16 or all lanes', so that a warp's rows take their steps together; parts come in chunks that fit.
    const int width = rows > 2 * WARPS ? 8 : rows > WARPS ? 16 : 32, l = lane & (width - 1), mine = lane / width;
    const int chunk = kChunk * (width / 8);
    float4* mls = reinterpret_cast<float4*>(room) + mine * kFlatFp8;   // m, l and M of every part
    float4* os = reinterpret_cast<float4*>(room + kMlBytes) + mine * chunk * kPieces;
#pragma unroll 1
    for (int at = warp + WARPS * mine; at - WARPS * mine < rows; at += WARPS * (32 / width)) {
      const int which = at < rows0 ? 0 : 1, row = at - (which ? rows0 : 0);
      const Segment& g = late[which];
      const JoinStep j = which ? j1 : j0;
      const int n_parts = at < rows && j.n > 1 ? j.n : 0;
      const auto part_at = [&](int i) { return part_slot(P, g.first_cta, j.first + i * j.stride, kPart); };
      for (int i = l; i < n_parts; i += width) copy16_l2(mls + i, part_at(i) + ROWS * D + kPartPad * row);
      float mm = -INFINITY, ll = 0.f, top = -INFINITY;
      float4 a[D / 32];
#pragma unroll
      for (int c = 0; c < D / 32; ++c) a[c] = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 1
      for (int c0 = 0; __any_sync(0xffffffffu, c0 < n_parts); c0 += chunk) {
        const int n_here = min(chunk, n_parts - c0);
#pragma unroll 2
        for (int i = 0; i < n_here; ++i) {
          const float4* src = reinterpret_cast<const float4*>(part_at(c0 + i) + row * D);
#pragma unroll
          for (int c = 0; c < D / 32; ++c)
            if (l + width * c < kPieces) copy16_l2(os + i * kPieces + l + width * c, src + l + width * c);
        }
        asm volatile("cp.async.wait_all;" ::: "memory");
        if (c0 == 0) {   // a lane a part: the factor of its O, and its l times the other one, in its maximum's and sum's place
#pragma unroll 1
          for (int i = l; i < n_parts; i += width) mm = fmaxf(mm, mls[i].x), top = fmaxf(top, mls[i].z);
#pragma unroll 1
          for (int d = width / 2; d > 0; d >>= 1) {
            mm = fmaxf(mm, __shfl_xor_sync(0xffffffffu, mm, d));
            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
          }
#pragma unroll 1
          for (int i = l; i < n_parts; i += width) {
            const float4 x = mls[i];
            *reinterpret_cast<float2*>(mls + i) =
                make_float2(ex2(x.z - (top == -INFINITY ? 0.f : top)), x.y * ex2(x.x - (mm == -INFINITY ? 0.f : mm)));
          }
        }
        __syncwarp();
#pragma unroll 4
        for (int i = 0; i < n_here; ++i) {
          const float2 fl = *reinterpret_cast<const float2*>(mls + c0 + i);
          const float f = fl.x;
          ll += fl.y;
#pragma unroll
          for (int c = 0; c < D / 32; ++c)
            if (l + width * c < kPieces) {
              const float4 x = os[i * kPieces + l + width * c];
              a[c].x = fmaf(x.x, f, a[c].x), a[c].y = fmaf(x.y, f, a[c].y), a[c].z = fmaf(x.z, f, a[c].z), a[c].w = fmaf(x.w, f, a[c].w);
            }
        }
        __syncwarp();   // before the next copies
      }
      if (n_parts == 0) continue;
      const int tok = row_token(P, row0<kTwo>(g) + row), hd = row0<kTwo>(g) + row - tok * P.group;
      const float2 back = back_from(mm, ll, top, g.s.seen(tok) > 0);
      float* slot = part_at(0);
#pragma unroll
      for (int c = 0; c < D / 32; ++c) {
        const int piece = l + width * c;
        if (piece >= kPieces) continue;
        if (!j.last)   // in the place of the group's first part
          reinterpret_cast<float4*>(slot + row * D)[piece] = a[c];
        else
          reinterpret_cast<uint2*>(P.out + ((int64_t)(g.s.tok0 + tok) * P.q_heads + g.h * P.group + hd) * D)[piece] =
              make_uint2(pack_bf16(a[c].x * back.x * back.y, a[c].y * back.x * back.y), pack_bf16(a[c].z * back.x * back.y, a[c].w * back.x * back.y));
      }
      if (!j.last && l == 0) *reinterpret_cast<float4*>(slot + ROWS * D + kPartPad * row) = make_float4(mm, ll, top, 0.f);
    }
    on[0] = on[0] && !j0.last;
    on[1] = on[1] && !j1.last;
  }
}

template <int D>
struct RowsCfg {
  static constexpr int kWarps = 2 * kPairs;                     // consumers
  static constexpr int kThreads = (kWarps + kPairs) * 32;       // + the fetching warps
  static constexpr int kRows = kMost;
  static constexpr int kPart = kRows * (D + kPartPad);          // floats of a part in the workspace
  static constexpr int kOpBytes = kSlotKeys * D;
  static constexpr int kSlotBytes = 2 * kOpBytes;
  static constexpr int kStages = kRingBytes / (kPairs * kSlotBytes);
  static constexpr int kPowerBytes = 2 * kSlotKeys;             // of a slot: the keys' powers, then the values'
  static constexpr int kQRow = D * 2 + 16;                      // bytes of a row of queries: rows start in different banks
  static constexpr int kQBytes = kRows * kQRow;
  static constexpr int kQSlots = 2;                             // segments whose queries are here ahead
  static constexpr int kSmem = kPairs * kStages * (kSlotBytes + kPowerBytes) + kQSlots * kQBytes + 1024;
  static constexpr int kRegsFetch = 72, kRegs = 216;
  static_assert(32 * (kWarps * kRegs + kPairs * kRegsFetch) <= kThreads * (65536 / kThreads / 8 * 8), "register split");
  static_assert(kPairs * kStages * kSlotBytes == kRingBytes, "whole slots");
  static_assert(kSmem <= 227 * 1024 - 6 * 1024, "shared memory budget");
};

template <int D, bool kTwo>
__global__ void __launch_bounds__(RowsCfg<D>::kThreads, 1) k_attn_rows_fp8(const __grid_constant__ AttnParams P) {
  using C = RowsCfg<D>;
  constexpr int S = C::kStages, W = C::kWarps;
  extern __shared__ uint8_t af_smem_raw[];
  __shared__ __align__(8) uint64_t full_bar[kPairs][S];
  __shared__ __align__(8) uint64_t empty_bar[kPairs][S];
  __shared__ __align__(8) uint64_t qfull_bar[C::kQSlots], qempty_bar[C::kQSlots];
  __shared__ __align__(8) uint64_t meet_bar;
  __shared__ Segment segs[kPairs][S];    // of the slot, where it is its segment's first; r < 0: the end
  __shared__ WorkShared work;
  __shared__ float2 join_ml[2][W * 16];  // [warp][its rows]: maximum and sum
  __shared__ float join_top[2][W * 16];  // the numerators' maximum
  __shared__ Segment late[2];            // split items' segments of this CTA, joined at its end
  __shared__ int abort_s, last_s[2];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(af_smem_raw) + 1023) & ~uintptr_t(1023));
  uint8_t* ssm = smem + kPairs * S * C::kSlotBytes;
  uint8_t* qsm = ssm + kPairs * S * C::kPowerBytes;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int cta = (int)blockIdx.x;
  if (threadIdx.x == 0) {
    for (int p = 0; p < kPairs; ++p)
      for (int s = 0; s < S; ++s) {
        mbar_init(&full_bar[p][s], 9);    // the codes, and eight lanes' copies of powers
        mbar_init(&empty_bar[p][s], W);   // four of each of the pair; after a join one of each warp
      }
    for (int s = 0; s < C::kQSlots; ++s) {
      mbar_init(&qfull_bar[s], kPairs);
      mbar_init(&qempty_bar[s], W);
    }
    mbar_init(&meet_bar, W);
    abort_s = 0;
    fence_mbar_init();
    prefetch_tmap(&P.kmap);
    prefetch_tmap(&P.vmap);
  }
  if (!P.two_launches) start_of_work();   // else the chunk launch has waited, and lets this one begin after that
  const Shares shares = divide_work<FewTraits<kTwo>, C::kThreads>(P, cta, work);
  volatile int* abort_flag = &abort_s;
  const int box_shift = min(P.page_shift, 6), box = 1 << box_shift;   // rows of a TMA box
  const auto wait_warp = [&](uint64_t* bar, uint32_t parity) {
    return mbar_wait_warp(bar, parity, abort_flag);
  };
  const auto slot_at = [&](int pair, uint32_t st) { return smem + (pair * S + (int)st) * C::kSlotBytes; };
  const auto powers_at = [&](int pair, uint32_t st) { return ssm + (pair * S + (int)st) * C::kPowerBytes; };

  if (warp >= W) {
    // ------------------------------------------------------------ fetch, for one pair, and a part of the queries
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(C::kRegsFetch));
    const int pair = warp - W;
    Walker<FewTraits<kTwo>> walk(P, shares, work, cta);
    Segment g;
    const int32_t no_row = (int32_t)((P.pages * P.kv_heads) << P.page_shift);   // past the last: reads as zeros
    uint32_t st = 0, ph = 1u, qs = 0, qph = 1u;
    bool ok = pair != 0 || !injected_timeout(P, cta, abort_flag);
    while (ok && walk.next(g)) {
      if (tile_units(P, g.s, g.rt) == 2) {   // tiles that begin in the segment: at least one, since it has two units
        g.ta = (g.ta + 1) >> 1;
        g.tb = (g.tb + 1) >> 1;
      }
      if (g.ta >= g.tb) continue;
      if constexpr (kTwo) g.s.rows = tile_rows(g.s, g.rt);   // from here on the segment's own, from row0
      const int len = g.s.len();
      const int64_t trow = (int64_t)g.r * P.width;
      const auto entries = [&](int block) {   // lane i: table entry 32 block + i
        const int e = 32 * block + lane;
        return e < P.width && ((int64_t)e << P.page_shift) < len ? __ldg(P.table + trow + e) : -1;
      };
      int held = (g.ta * kTile + pair * kSlotKeys) >> P.page_shift >> 5;
      int page = entries(held), ahead = entries(held + 1);
      if (!(ok = wait_warp(&qempty_bar[qs], qph))) break;   // every fourth row of the queries
      if (lane == 0) mbar_arrive_expect_tx(&qfull_bar[qs], (uint32_t)((g.s.rows - pair + kPairs - 1) / kPairs * (D * 2)));
      __syncwarp();
      for (int row = pair + kPairs * lane; row < g.s.rows; row += 32 * kPairs) {
        const int tok = row_token(P, row0<kTwo>(g) + row), hd = row0<kTwo>(g) + row - tok * P.group;
        bulk_load(qsm + qs * C::kQBytes + row * C::kQRow,
                  P.q + (int64_t)(g.s.tok0 + tok) * P.q_stride + (int64_t)(g.h * P.group + hd) * D, D * 2, &qfull_bar[qs]);
      }
      if (++qs == C::kQSlots) {
        qs = 0;
        qph ^= 1u;
      }
      for (int t = g.ta; t < g.tb; ++t) {
        const int first_key = t * kTile + pair * kSlotKeys;
        const int valid = min(kSlotKeys, max(0, len - first_key));
        const int boxes = (valid + box - 1) >> box_shift;   // at most 4
        // a slot's table entries lie within one block of 32
        const int block = first_key >> P.page_shift >> 5;
        if (block != held) {
          held = block;
          page = ahead;
          ahead = entries(held + 1);
        }
        if (!wait_warp(&empty_bar[pair][st], ph)) {
          ok = false;
          break;
        }
        uint64_t* full = &full_bar[pair][st];
        if (lane == 0) {
          if (t == g.ta) segs[pair][st] = g;
          mbar_arrive_expect_tx(full, 2u * (uint32_t)(boxes * box * D));
        }
        __syncwarp();
        // lane b fetches box b of the keys, lane 4 + b of the values, and powers of 16 keys by the load path (two bulk copies
        // more a box cost the 16 sequences of the first figure 20 us).  Pages that are not there give zeros.
        const int b = lane & 3, key = first_key + (b << box_shift), key16 = first_key + 16 * b;
        const int pg = __shfl_sync(0xffffffffu, page, (key >> P.page_shift) & 31);
        const int pg16 = __shfl_sync(0xffffffffu, page, (key16 >> P.page_shift) & 31);
        const auto row_of = [&](int p, int k) { return (((int64_t)p * P.kv_heads + g.h) << P.page_shift) + (k & ((1 << P.page_shift) - 1)); };
        if (lane < 8) {
          if (b < boxes)
            tma_load_2d(slot_at(pair, st) + (lane >> 2) * C::kOpBytes + b * (box * D), lane < 4 ? &P.kmap : &P.vmap, full, 0,
                        pg >= 0 && pg < P.pages ? (int32_t)row_of(pg, key) : no_row);
          if (16 * b < valid) {
            const bool has = pg16 >= 0 && pg16 < P.pages;
            copy16(powers_at(pair, st) + (lane >> 2) * kSlotKeys + 16 * b, (lane < 4 ? P.k_scales : P.v_scales) + (has ? row_of(pg16, key16) : 0), has);
          }
          arrive_after_copies(full);
        }
        __syncwarp();
        if (++st == S) {
          st = 0;
          ph ^= 1u;
        }
      }
    }
    if (ok && wait_warp(&empty_bar[pair][st], ph)) {   // the end
      if (lane == 0) {
        segs[pair][st].r = -1;
        mbar_arrive(&full_bar[pair][st]);
      }
      if (lane < 8) mbar_arrive(&full_bar[pair][st]);
    }
    if (pair == 0) zero_rows(P, D, cta, lane, P.zero_rest != 0);
  } else {
    // ------------------------------------------------------------ compute
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(C::kRegs));
    const int pair = warp >> 1, half = warp & 1, gq = lane >> 2, qd = lane & 3;
    constexpr int MT = 2, kSub = 16 * MT;   // tiles of 16 keys between two steps of the running maximum
    uint32_t mph = 0, turn = 0;
    int n_late = 0;   // a CTA has at most one part of an item that began before it, and one of an item that goes on after it
    // the compute warps' barrier, bounded like every wait: false when some role gave up
    const auto meet = [&]() {
      __syncwarp();
      if (lane == 0) mbar_arrive(&meet_bar);
      const bool met = wait_warp(&meet_bar, mph);
      mph ^= 1u;
      return met;
    };
    uint32_t st = 0, ph = 0u, qs = 0, qph = 0u;
    // Byte offset of this lane's row of 16 keys in an operand, for matrices (keys 0-7, 8-15) x (16 channels, the next 16); its
    // swizzle is folded in: columns of 16 channels by an "xor" with their number << 4.
    uint32_t off[kSlotKeys / 16];
#pragma unroll
    for (int i = 0; i < kSlotKeys / 16; ++i) {
      const int key = 16 * i + (lane & 15);
      off[i] = ((uint32_t)(key * D) ^ (uint32_t)((D == 128 ? key & 7 : (key >> 1) & 3) << 4)) ^ ((lane >> 4) << 4);
    }
    // One segment's part (or result), by warps that have NT tiles of 8 rows; split: each warp of a pair half of the rows.  false:
    // some role gave up.
    const auto segment = [&](const Segment& g, auto tiles, auto split_rows) -> bool {
      constexpr int NT = decltype(tiles)::value;
      constexpr bool kSplit = decltype(split_rows)::value;
      const int row_first = kSplit ? 16 * half : 0;
      const int len = g.s.len();
      // Queries: row gq of a tile, channels 4 qd ... + 3 of 16, like the keys' below.  A row's largest magnitude is moved to 2^14,
      // so elements down to 2^-29 of it keep all their bits.  Rows past the last hold whatever the buffer held: nobody reads theirs.
      uint32_t qf[D / 16][NT][2];
      float unit[NT][2];   // what a score is multiplied by, of rows 8 n + 2 qd (+ 1)
      int seen[NT][2];
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        const uint8_t* qr = qsm + qs * C::kQBytes + (row_first + 8 * n + gq) * C::kQRow + 8 * qd;
        uint2 x[D / 16];
        uint32_t top = 0;
#pragma unroll
        for (int ks = 0; ks < D / 16; ++ks) {
          x[ks] = *reinterpret_cast<const uint2*>(qr + 32 * ks);
          top = max(top, max(max(x[ks].x & 0x7FFFu, (x[ks].x >> 16) & 0x7FFFu), max(x[ks].y & 0x7FFFu, (x[ks].y >> 16) & 0x7FFFu)));
        }
        top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
        top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
        const int ex = top >= 0x7F80u ? 141 : max((int)(top >> 7), 15);   // 141: as they are, for an infinity or a NaN
        const float up = power_of(268 - ex) * (P.negate ? -1.f : 1.f), down = P.scale_log2 * power_of(ex - 14);
#pragma unroll
        for (int ks = 0; ks < D / 16; ++ks) {
          qf[ks][n][0] = pack_f16(bf16_lo(x[ks].x) * up, bf16_hi(x[ks].x) * up);
          qf[ks][n][1] = pack_f16(bf16_lo(x[ks].y) * up, bf16_hi(x[ks].y) * up);
        }
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const int row = row_first + 8 * n + 2 * qd + e;
          unit[n][e] = __shfl_sync(0xffffffffu, down, 4 * (2 * qd + e));
          seen[n][e] = row < g.s.rows ? g.s.seen(row_token(P, row0<kTwo>(g) + row)) : 0;
        }
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(&qempty_bar[qs]);
      if (++qs == C::kQSlots) {
        qs = 0;
        qph ^= 1u;
      }
      const int all_see = g.s.seen(0);                 // keys below this are visible to every row
      float o[D / 16][NT][4];                          // channels 16 j + 2 gq (and + 1: the last two), rows 8 n + 2 qd, + 1
      float m[NT][2], l[NT][2], M[NT][2];
      float r[NT][2] = {}, more[NT][2];                // 2^(6 - (M - m)); a step's part of l
      float limit = 0.f;                               // the largest power that a weight times r may meet
      bool unset = true;                               // some row that sees keys has no M yet
#pragma unroll
      for (int n = 0; n < NT; ++n) {
#pragma unroll
        for (int e = 0; e < 2; ++e) m[n][e] = M[n][e] = -INFINITY, l[n][e] = 0.f;
#pragma unroll
        for (int j = 0; j < D / 16; ++j)
#pragma unroll
          for (int e = 0; e < 4; ++e) o[j][n][e] = 0.f;
      }
      for (int t = g.ta; t < g.tb; ++t) {
        if (t > g.ta) {
          // the slot before goes back; the segment's last one is kept for the join
          __syncwarp();
          if (lane == 0) arrive_by(&empty_bar[pair][st], 4);
          if (++st == S) {
            st = 0;
            ph ^= 1u;
          }
          if (!wait_warp(&full_bar[pair][st], ph)) return false;
        }
        const uint32_t kop = smem_u32(slot_at(pair, st)), vop = kop + C::kOpBytes;
#pragma unroll 1
        for (int sub = 0; sub < (kSplit ? 2 : 1); ++sub) {
          const int at = kSplit ? kSub * sub : kSub * half;              // of the slot's keys
          const int key0 = t * kTile + pair * kSlotKeys + at;
          if (key0 >= len) break;                                        // uniform over the warp
          const bool masked = key0 + kSub > all_see;
          const uint8_t* pw = powers_at(pair, st) + at;
          uint32_t kp[MT][2], vp[MT][2];                                 // powers of keys and values 16 i + gq, + 8
#pragma unroll
          for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int b = 0; b < 2; ++b) kp[i][b] = pw[16 * i + 8 * b + gq], vp[i][b] = pw[kSlotKeys + 16 * i + 8 * b + gq];
          float s[MT][NT][4];
#pragma unroll
          for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
              for (int e = 0; e < 4; ++e) s[i][n][e] = 0.f;
#pragma unroll
          for (int c = 0; c < D / 32; ++c)
#pragma unroll
            for (int i = 0; i < MT; ++i) {
              uint32_t kf[4];
              ldsm4(kf, (kop + (at ? off[MT + i] : off[i])) ^ (uint32_t)(c << 5));
#pragma unroll
              for (int b = 0; b < 2; ++b) {
                const uint32_t a[4] = {f16_of_lo(kf[2 * b]), f16_of_lo(kf[2 * b + 1]), f16_of_hi(kf[2 * b]), f16_of_hi(kf[2 * b + 1])};
#pragma unroll
                for (int n = 0; n < NT; ++n) mma16816(s[i][n], a, qf[2 * c + b][n][0], qf[2 * c + b][n][1]);
              }
            }
          float vw[MT][2];   // powers of values
          float most = -INFINITY;
#pragma unroll
          for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int b = 0; b < 2; ++b) {
              const float power = power_or_nan(kp[i][b]);
              vw[i][b] = power_or_nan(vp[i][b]);
              most = fmaxf(most, vw[i][b]);
#pragma unroll
              for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int e = 0; e < 2; ++e) s[i][n][2 * b + e] *= power * unit[n][e];
            }
          if (masked) {
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
              for (int e = 0; e < 2; ++e)
#pragma unroll
                for (int i = 0; i < MT; ++i)
#pragma unroll
                  for (int b = 0; b < 2; ++b)
                    if (key0 + 16 * i + 8 * b + gq >= seen[n][e]) s[i][n][2 * b + e] = -INFINITY;
          }
          // Numerators: a weight times r times its value's power, where every row sees every key, none has passed a maximum in use by
          // more than 2^8 (they count in 2^-6), and weights below float32's range are nothing beside the largest numerator
          // whatever the power.  Otherwise (redo) the maxima are raised, and numerators are formed from exponents.  (Always so,
          // in one loop: 16 x 32 tokens 107 us, 104 thus; by the scores' maxima instead of the results: 111.)
          uint32_t p16[MT][NT][2];   // of two rows, keys 16 i + 8 b + gq
          bool redo = unset || masked;
          if (!redo) {
            bool above = most > limit;
#pragma unroll
            for (int n = 0; n < NT; ++n) {
              float sum[2] = {0.f, 0.f};
              uint32_t top = 0;
#pragma unroll
              for (int i = 0; i < MT; ++i)
#pragma unroll
                for (int b = 0; b < 2; ++b) {
                  const float w0 = ex2(s[i][n][2 * b] - m[n][0]), w1 = ex2(s[i][n][2 * b + 1] - m[n][1]);
                  sum[0] += w0, sum[1] += w1;
                  p16[i][n][b] = pack_f16(w0 * r[n][0] * vw[i][b], w1 * r[n][1] * vw[i][b]);
                  top = max_f16x2(top, p16[i][n][b]);
                }
              // rows that are none have no say: theirs are any numbers
              above |= seen[n][0] > 0 && (sum[0] > 256.f || (top & 0xFFFFu) > 0x7400u);
              above |= seen[n][1] > 0 && (sum[1] > 256.f || (top >> 16) > 0x7400u);
              more[n][0] = sum[0], more[n][1] = sum[1];
            }
            redo = __any_sync(0xffffffffu, above);
          }
          if (redo) {
            unset = false;
            limit = INFINITY;
#pragma unroll
            for (int n = 0; n < NT; ++n) {
              float base[2], base_o[2], so[MT][2][2];
#pragma unroll
              for (int e = 0; e < 2; ++e) {
                float top = -INFINITY, top_o = -INFINITY;
#pragma unroll
                for (int i = 0; i < MT; ++i)
#pragma unroll
                  for (int b = 0; b < 2; ++b) {
                    // a value that the row does not see has no weight, whatever its power
                    const bool none = masked && key0 + 16 * i + 8 * b + gq >= seen[n][e];
                    so[i][b][e] = none ? -INFINITY : s[i][n][2 * b + e] + lg2(vw[i][b]);
                    top = fmaxf(top, s[i][n][2 * b + e]), top_o = fmaxf(top_o, so[i][b][e]);
                  }
                const float mn = fmaxf(m[n][e], keys_max(top)), Mn = fmaxf(M[n][e], keys_max(top_o));
                l[n][e] *= mn == m[n][e] ? 1.f : ex2(m[n][e] - mn);   // m = -inf: 0
                const float f = Mn == M[n][e] ? 1.f : ex2(M[n][e] - Mn);
                m[n][e] = mn;
                M[n][e] = Mn;
                base[e] = mn == -INFINITY ? 0.f : mn, base_o[e] = Mn == -INFINITY ? 0.f : Mn - 6.f;
                if (seen[n][e] > key0) {   // there is something to see from here on
                  const float d = Mn - mn;
                  r[n][e] = ex2(6.f - d);
                  unset |= Mn == -INFINITY;   // no value with a power yet, or none that is a number
                  limit = fminf(limit, d < -100.f ? -1.f : ex2(fminf(d + 90.f, 120.f)));
                }
#pragma unroll
                for (int j = 0; j < D / 16; ++j) o[j][n][e] *= f, o[j][n][2 + e] *= f;
              }
              more[n][0] = more[n][1] = 0.f;
#pragma unroll
              for (int i = 0; i < MT; ++i)
#pragma unroll
                for (int b = 0; b < 2; ++b) {
#pragma unroll
                  for (int e = 0; e < 2; ++e) more[n][e] += ex2(s[i][n][2 * b + e] - base[e]);
                  p16[i][n][b] = pack_f16(ex2(so[i][b][0] - base_o[0]), ex2(so[i][b][1] - base_o[1]));
                }
            }
            unset = __any_sync(0xffffffffu, unset);
          }
#pragma unroll
          for (int n = 0; n < NT; ++n) l[n][0] += more[n][0], l[n][1] += more[n][1];
#pragma unroll
          for (int i = 0; i < MT; ++i) {
            uint32_t pf[NT][2];   // keys 2 qd, + 1 (then + 8) of row gq
#pragma unroll
            for (int n = 0; n < NT; ++n) {
              pf[n][0] = transposed(p16[i][n][0]);
              pf[n][1] = transposed(p16[i][n][1]);
            }
            uint32_t keep[2] = {~0u, ~0u};   // codes past the sequence's end may be those of NaN
            if (masked) {
#pragma unroll
              for (int b = 0; b < 2; ++b) {
                const int key = key0 + 16 * i + 8 * b + 2 * qd;
                keep[b] = (key < len ? 0xFFFFu : 0u) | (key + 1 < len ? 0xFFFF0000u : 0u);
              }
            }
#pragma unroll
            for (int c = 0; c < D / 32; ++c) {
              uint32_t vf[4];   // (keys 0-7, keys 8-15) of channels 32 c ..., then of 32 c + 16 ...: two channels of two keys
              ldsm4t(vf, (vop + (at ? off[MT + i] : off[i])) ^ (uint32_t)(c << 5));
              if (masked)
#pragma unroll
                for (int b = 0; b < 4; ++b) vf[b] &= keep[b & 1];
#pragma unroll
              for (int b = 0; b < 4; ++b) vf[b] = __byte_perm(vf[b], 0u, 0x3120);   // the even channel, the odd one
#pragma unroll
              for (int b = 0; b < 2; ++b) {   // rows of the tile: the even channels of 16, then the odd ones
                const uint32_t a[4] = {f16_of_lo(vf[2 * b]), f16_of_hi(vf[2 * b]), f16_of_lo(vf[2 * b + 1]), f16_of_hi(vf[2 * b + 1])};
#pragma unroll
                for (int n = 0; n < NT; ++n) mma16816(o[2 * c + b][n], a, pf[n][0], pf[n][1]);
              }
            }
          }
        }
      }
      // ---- join the warps, in the slots: a warp's part [16][D] lies in its half of the pair's keys (8 rows) and values
      const auto part_row = [&](int w, int row) -> float* {
        return reinterpret_cast<float*>(slot_at(w >> 1, st) + (row >> 3) * C::kOpBytes + (w & 1) * (32 * D)) + (row & 7) * D;
      };
      ++turn;
      if (kSplit && !meet()) return false;   // both warps of a pair have read all of its keys
      float* slot = g.parts > 1 ? part_slot(P, g.first_cta, g.part, C::kPart) : nullptr;
      float2* ml_of = join_ml[turn & 1];
      float* top_of = join_top[turn & 1];
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const int row = 8 * n + 2 * qd + e;
          const float sum = keys_sum(l[n][e]);
          if (row_first + row < g.s.rows) {
            float* dst = part_row(warp, row) + 2 * gq;
#pragma unroll
            for (int j = 0; j < D / 16; ++j)
              *reinterpret_cast<float2*>(dst + 16 * j) = make_float2(o[j][n][e], o[j][n][2 + e]);
            if (gq == 0) ml_of[warp * 16 + row] = make_float2(m[n][e], sum), top_of[warp * 16 + row] = M[n][e];
          }
        }
      // warps without a row too: the slots that they hand back have to be the ones that all are at
      if (!meet()) return false;
      constexpr int kParts = kSplit ? W / 2 : W;   // of a row
      constexpr int kWidth = kSplit ? 8 : 32 / NT;   // lanes of a row: all rows in one go
      const int row = warp + W * (lane / kWidth), at = lane & (kWidth - 1);
      if (row < g.s.rows) {
        const int hi = kSplit ? row >> 4 : 0, r16 = row & 15;
        const auto warp_of = [&](int i) { return kSplit ? 2 * i + hi : i; };
        float2 ml[kParts];
        float fo[kParts], mm = -INFINITY, ll = 0.f, top = -INFINITY;
#pragma unroll
        for (int i = 0; i < kParts; ++i) {
          ml[i] = ml_of[warp_of(i) * 16 + r16], fo[i] = top_of[warp_of(i) * 16 + r16];
          mm = fmaxf(mm, ml[i].x), top = fmaxf(top, fo[i]);
        }
        const float base = mm == -INFINITY ? 0.f : mm, base_o = top == -INFINITY ? 0.f : top;
#pragma unroll
        for (int i = 0; i < kParts; ++i) ll = fmaf(ml[i].y, ex2(ml[i].x - base), ll), fo[i] = ex2(fo[i] - base_o);
        const int tok = row_token(P, row0<kTwo>(g) + row), hd = row0<kTwo>(g) + row - tok * P.group;
        const float2 back = back_from(mm, ll, top, g.s.seen(tok) > 0);
#pragma unroll
        for (int c = 0; c < (D / 4 + kWidth - 1) / kWidth; ++c) {
          const int piece = at + kWidth * c;
          if (D / 4 < kWidth && piece >= D / 4) break;
          float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
          for (int i = 0; i < kParts; ++i) {
            const float4 x = reinterpret_cast<const float4*>(part_row(warp_of(i), r16))[piece];
            const float f = fo[i];
            a.x = fmaf(x.x, f, a.x), a.y = fmaf(x.y, f, a.y), a.z = fmaf(x.z, f, a.z), a.w = fmaf(x.w, f, a.w);
          }
          if (slot)
            reinterpret_cast<float4*>(slot + row * D)[piece] = a;
          else
            reinterpret_cast<uint2*>(P.out + ((int64_t)(g.s.tok0 + tok) * P.q_heads + g.h * P.group + hd) * D)[piece] =
                make_uint2(pack_bf16(a.x * back.x * back.y, a.y * back.x * back.y), pack_bf16(a.z * back.x * back.y, a.w * back.x * back.y));
        }
        if (slot && at < 2)   // a whole sector
          reinterpret_cast<float4*>(slot + C::kRows * D + kPartPad * row)[at] = at == 0 ? make_float4(mm, ll, top, 0.f) : make_float4(0.f, 0.f, 0.f, 0.f);
      }
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");   // the slots were written here; copies overwrite them
      __syncwarp();
      if (lane < kPairs) mbar_arrive(&empty_bar[lane][st]);
      if (++st == S) {
        st = 0;
        ph ^= 1u;
      }
      if (slot) {
        if (threadIdx.x == 0) late[n_late & 1] = g;
        ++n_late;
      }
      return true;
    };
    while (true) {
      if (!wait_warp(&full_bar[pair][st], ph)) break;
      const Segment g = segs[pair][st];
      if (g.r < 0) {
        join_late<D, kTwo, C::kRows, W>(P, late, min(n_late, 2), warp, lane, last_s, smem + warp * (kRingBytes / W), meet);
        break;
      }
      if (!wait_warp(&qfull_bar[qs], qph)) break;
      using One = std::integral_constant<int, 1>;
      using Two = std::integral_constant<int, 2>;
      if (!(g.s.rows <= 8 ? segment(g, One(), std::false_type()) : g.s.rows <= 16 ? segment(g, Two(), std::false_type())
                                                                                  : segment(g, Two(), std::true_type())))
        break;
    }
  }
  __syncthreads();
  end_of_waits(abort_flag, P.err);
  if (P.two_launches) start_of_work();   // the chunk launch's end: what follows waits for this one only
}

template <int D, bool kTwo>
gs_status rows_launch(const AttnParams& P, int ctas, cudaStream_t s) {
  using C = RowsCfg<D>;
  static const cudaError_t attr = cudaFuncSetAttribute(k_attn_rows_fp8<D, kTwo>, cudaFuncAttributeMaxDynamicSharedMemorySize, C::kSmem);
  if (attr != cudaSuccess) return GS_ERR_CUDA;
  return launch_behind(k_attn_rows_fp8<D, kTwo>, dim3((unsigned)ctas), C::kThreads, C::kSmem, s, P);
}

}  // namespace

// Two row tiles read a sequence's keys twice, but are through sooner than an item of the chunk kernel's with its joins, unless
// there are many items (28/4 heads, us here / in the chunk kernel): 9 tokens at 30000 keys 35.0 / 63.9, 5 at 8000 22.3 / 41.2, nine
// sequences of 1 to 9 at 100 to 9000 29.5 / 50.5, 19 x 9 (76 items) at 2000 30.1 / 39.8, 38 x 9 at 2000 54.5 / 42.3.  The rule asks
// for the items alone, although where they are half of the CTAs the length decides too: 19 x 9 at 8000 keys 89.6 / 79.9.
int attn_rows_fp8_most(int64_t items, int ctas) { return 2 * items <= ctas ? 2 * kMost : kMost; }
int attn_rows_fp8_box(int page_size) { return std::min(page_size, kSlotKeys); }

gs_status launch_attn_rows_fp8(const AttnParams& P, int head_dim, int ctas, cudaStream_t s) {
  if (P.max_rows > kMost) return head_dim == 128 ? rows_launch<128, true>(P, ctas, s) : rows_launch<64, true>(P, ctas, s);
  return head_dim == 128 ? rows_launch<128, false>(P, ctas, s) : rows_launch<64, false>(P, ctas, s);
}

}  // namespace gs
