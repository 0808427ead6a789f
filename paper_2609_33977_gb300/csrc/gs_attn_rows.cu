// Attention of few rows (new tokens x query heads a key head, at most 32): decoding
// steps and short chunks.
//
// Bound by HBM: a sequence's keys and values are read once, for all its rows.  A unit
// is 128 keys of a key head.  One warp fetches (TMA, a box per page and operand, 192 KB
// of units in flight per SM; a segment's queries come with its first unit), eight
// compute with m16n8k16: WR row tiles of 16 x WK shares of the unit's keys, each warp
// with its own running maximum, sum and output, joined over the WK warps once per
// segment, in the segment's last stage.  With one row tile, a warp's keys are read by
// no other warp, so it leaves its part in their place without waiting, and goes on
// unless it has a row to join.  Unused MMA rows cost nothing that matters, a second row
// tile does (16 tokens of 32 heads 69 us with one, 72 with two): WR is 1 up to 16 rows.
//
// The weights enter the second product as bf16 (2^-8 of each at most; the product takes no
// more bits, and the output is rounded to as many), their sums are taken before that.
//
// 16 sequences of 90 to 4000 keys, 32 heads: 70 us, 6.0 TB/s (the fetching alone, nothing
// computed, 70 us).  Three of 30001 to 65536 keys, 28/4 heads: 53 us, 5.6 TB/s (54).  One of
// 60000: 29.5 us, 4.2 TB/s, four tokens there 41.  One of 129 keys: 6.9 us, the look-up of
// the work and three hand-overs one after another.  Heads of 64, 16/2 of them: the first
// 11.9 us, 1.1 TB/s, the second 23 us, 3.2 TB/s.
#include "gs_attn_rows.cuh"

namespace gs {
namespace {
using namespace sm100;

constexpr int kTile = 128;
constexpr int kJoin = 8;   // rows of parts that a warp has under way when it joins them
// Parts joined in one level: the three long sequences above take 53 us, 55 with at most 8, 4 tokens of 28/4 heads at 60000
// keys 42 (always one level: 46).  More go in groups of at most sqrt(256).
constexpr int kFlat = 16;
static_assert(kFlat <= 32, "a lane a part");

// One unit an item beside its keys: the 16 sequences above take 70 us, 82 without.  kLeast 1, 2, 4: no difference.
struct FewTraits {
  static constexpr int kLeast = 2, kSnap = 1, kOver = 1;
  static constexpr bool kOneTile = true;
  static __device__ __forceinline__ int row_tiles(const SeqInfo& s, const AttnParams& P) {
    return s.rows >= P.min_rows && s.rows <= P.max_rows ? 1 : 0;
  }
  static __device__ __forceinline__ int tiles(const SeqInfo& s, const AttnParams&, int) {
    return max(1, (s.len() + kTile - 1) / kTile);
  }
};

__device__ __forceinline__ void mma16816(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ float quad_max(float v) {
  v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, 1));
  return fmaxf(v, __shfl_xor_sync(0xffffffffu, v, 2));
}
__device__ __forceinline__ float quad_sum(float v) {
  v += __shfl_xor_sync(0xffffffffu, v, 1);
  return v + __shfl_xor_sync(0xffffffffu, v, 2);
}
// bit 0 / 16: the low / high half is an infinity or NaN
__device__ __forceinline__ uint32_t nonfinite2(uint32_t v) {
  const uint32_t e = v & 0x7F807F80u;
  return ((e & 0xFFFFu) == 0x7F80u ? 1u : 0u) | ((e >> 16) == 0x7F80u ? 0x10000u : 0u);
}

template <int D, int WR>
struct RowsCfg {
  static constexpr int kWarps = 8;                   // consumers
  static constexpr int kWK = kWarps / WR;
  static constexpr int kThreads = (kWarps + 1) * 32; // + the fetching warp
  static constexpr int kRows = 16 * WR;
  static constexpr int kPart = kRows * (D + kPartPad);   // floats of a part
  static constexpr int kOpBytes = kTile * D * 2;
  static constexpr int kStageBytes = 2 * kOpBytes;   // also what a join needs: kWarps x 16 x D floats
  static constexpr int kQRow = D * 2 + 16;           // bytes of a row of queries: rows start in different banks
  static constexpr int kQBytes = kRows * kQRow;
  static constexpr int kQSlots = 2;                  // segments whose queries are here ahead
  static constexpr int kStages = 192 * 1024 / kStageBytes;
  static constexpr int kSmem = kStages * kStageBytes + kQSlots * kQBytes + 1024;
  static_assert(kWarps * 16 * D * 4 <= kStageBytes, "join");
  static_assert(kSmem <= 227 * 1024 - 4096, "shared memory budget");
};

// a row's D / 32 channels per lane
template <int D>
struct Lane;
template <>
struct Lane<128> {
  using V = float4;
  static __device__ __forceinline__ void unpack(const V& v, float (&a)[4]) { a[0] = v.x, a[1] = v.y, a[2] = v.z, a[3] = v.w; }
  static __device__ __forceinline__ V pack(const float (&a)[4]) { return make_float4(a[0], a[1], a[2], a[3]); }
  static __device__ __forceinline__ void store_bf16(uint16_t* dst, const float (&a)[4], float f) {
    *reinterpret_cast<uint2*>(dst) = make_uint2(pack_bf16(a[0] * f, a[1] * f), pack_bf16(a[2] * f, a[3] * f));
  }
};
template <>
struct Lane<64> {
  using V = float2;
  static __device__ __forceinline__ void unpack(const V& v, float (&a)[2]) { a[0] = v.x, a[1] = v.y; }
  static __device__ __forceinline__ V pack(const float (&a)[2]) { return make_float2(a[0], a[1]); }
  static __device__ __forceinline__ void store_bf16(uint16_t* dst, const float (&a)[2], float f) {
    *reinterpret_cast<uint32_t*>(dst) = pack_bf16(a[0] * f, a[1] * f);
  }
};

template <int D, int WR>
__global__ void __launch_bounds__(RowsCfg<D, WR>::kThreads, 1) k_attn_rows(const __grid_constant__ AttnParams P) {
  using C = RowsCfg<D, WR>;
  using L = Lane<D>;
  constexpr int kSlabs = D / 64, kC = D / 32, WK = C::kWK;
  extern __shared__ uint8_t ar_smem_raw[];
  __shared__ __align__(8) uint64_t full_bar[C::kStages];
  __shared__ __align__(8) uint64_t empty_bar[C::kStages];
  __shared__ __align__(8) uint64_t qempty_bar[C::kQSlots];
  __shared__ __align__(8) uint64_t join_bar, meet_bar;
  __shared__ Segment segs[C::kStages];   // of the unit in a stage, where it is the segment's first; r < 0: the end
  __shared__ WorkShared work;
  __shared__ float2 join_ml[2][C::kWarps * 16];   // [WK][rows]: maximum and sum
  __shared__ int abort_s, last_s, bad_s[4];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(ar_smem_raw) + 1023) & ~uintptr_t(1023));
  uint8_t* qsm = smem + C::kStages * C::kStageBytes;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int cta = (int)blockIdx.x;
  if (threadIdx.x == 0) {
    for (int s = 0; s < C::kStages; ++s) {
      mbar_init(&full_bar[s], 1);
      mbar_init(&empty_bar[s], C::kWarps);
    }
    for (int s = 0; s < C::kQSlots; ++s) mbar_init(&qempty_bar[s], C::kWarps);
    mbar_init(&join_bar, C::kWarps);
    mbar_init(&meet_bar, C::kWarps);
    abort_s = 0;
    for (int i = 0; i < 4; ++i) bad_s[i] = 0;
    fence_mbar_init();
  }
  if (threadIdx.x == C::kWarps * 32) {
    prefetch_tmap(&P.kmap);
    prefetch_tmap(&P.vmap);
  }
  if (!P.two_launches) start_of_work();   // else the chunk launch has waited, and lets this one begin after that
  const Shares shares = divide_work<FewTraits, C::kThreads>(P, cta, work);
  volatile int* abort_flag = &abort_s;
  const int chunk_shift = min(P.page_shift, 7), chunk = 1 << chunk_shift;   // rows of a TMA box
  const auto wait_warp = [&](uint64_t* bar, uint32_t parity) {
    return mbar_wait_warp(bar, parity, abort_flag);
  };

  if (warp == C::kWarps) {
    // ------------------------------------------------------------ fetch
    Walker<FewTraits> walk(P, shares, work, cta);
    Segment g;
    const int32_t no_row = (int32_t)((P.pages * P.kv_heads) << P.page_shift);   // past the last: reads as zeros
    uint32_t st = 0, ph = 1u, qs = 0, qph = 1u;
    bool ok = !injected_timeout(P, cta, abort_flag);
    while (ok && walk.next(g)) {
      const int len = g.s.len();
      const int64_t trow = (int64_t)g.r * P.width;
      int held = -1, page = -1;   // lane i holds table entry 32 held + i
      for (int t = g.ta; t < g.tb; ++t) {
        const int valid = min(kTile, max(0, len - t * kTile));
        const int boxes = (valid + chunk - 1) >> chunk_shift;   // at most 8
        // all boxes of a unit have their table entries within one block of 32
        const int e0 = (t * kTile) >> P.page_shift;
        if (e0 >> 5 != held) {
          held = e0 >> 5;
          const int e = 32 * held + lane;
          page = e < P.width && ((int64_t)e << P.page_shift) < len ? __ldg(P.table + trow + e) : -1;
        }
        const bool first = t == g.ta;
        if (!wait_warp(&empty_bar[st], ph) || (first && !wait_warp(&qempty_bar[qs], qph))) {
          ok = false;
          break;
        }
        uint8_t* stage = smem + st * C::kStageBytes;
        if (lane == 0) {
          if (first) segs[st] = g;
          mbar_arrive_expect_tx(&full_bar[st], 2u * (uint32_t)(boxes * chunk * D * 2) + (first ? (uint32_t)(g.s.rows * D * 2) : 0u));
        }
        __syncwarp();
        // lane b fetches box b of the keys, lane 16 + b of the values
        const int b = lane & 15, key = t * kTile + (b << chunk_shift);
        const int pg = __shfl_sync(0xffffffffu, page, (key >> P.page_shift) & 31);
        if (b < boxes) {
          const int32_t row = pg >= 0 && pg < P.pages
                                  ? (int32_t)((((int64_t)pg * P.kv_heads + g.h) << P.page_shift) + (key & ((1 << P.page_shift) - 1)))
                                  : no_row;
          tma_load_3d(stage + b * (chunk * D * 2) + (lane >> 4) * C::kOpBytes, lane < 16 ? &P.kmap : &P.vmap, &full_bar[st], 0, row, 0);
        }
        if (first) {
          for (int row = lane; row < g.s.rows; row += 32) {
            const int tok = row_token(P, row), hd = row - tok * P.group;
            bulk_load(qsm + qs * C::kQBytes + row * C::kQRow,
                      P.q + (int64_t)(g.s.tok0 + tok) * P.q_stride + (int64_t)(g.h * P.group + hd) * D, D * 2, &full_bar[st]);
          }
          if (++qs == C::kQSlots) {
            qs = 0;
            qph ^= 1u;
          }
        }
        __syncwarp();
        if (++st == C::kStages) {
          st = 0;
          ph ^= 1u;
        }
      }
    }
    if (ok && wait_warp(&empty_bar[st], ph) && lane == 0) {   // the end
      segs[st].r = -1;
      mbar_arrive(&full_bar[st]);
    }
    zero_rows(P, D, cta, lane, P.zero_rest != 0);
  } else {
    // ------------------------------------------------------------ compute
    const int wr = warp / WK, wk = warp % WK, gq = lane >> 2, qd = lane & 3;
    constexpr int kKeys = kTile / WK;              // this warp's keys of a unit: 16 or 32
    constexpr int kSub = kKeys < 32 ? kKeys : 32;  // keys between two steps of the running maximum
    constexpr int kNt = kSub / 8;
    uint32_t jph = 0, mph = 0;
    // the compute warps' barrier, bounded like every wait: false when some role gave up
    const auto meet = [&]() {
      __syncwarp();
      if (lane == 0) mbar_arrive(&meet_bar);
      const bool met = wait_warp(&meet_bar, mph);
      mph ^= 1u;
      return met;
    };
    // A part: [rows][D], then [rows][8] with maximum and sum, the rest zeros: a 32-byte sector that is written in part
    // costs whoever reads it a fill from HBM.
    const auto store_part = [&](float* slot, int row, const float (&a)[kC], float mm, float ll) {
      reinterpret_cast<typename L::V*>(slot + row * D)[lane] = L::pack(a);
      if (lane < 2) reinterpret_cast<float4*>(slot + C::kRows * D + kPartPad * row)[lane] = lane == 0 ? make_float4(mm, ll, 0.f, 0.f) : make_float4(0.f, 0.f, 0.f, 0.f);
    };
    uint32_t st = 0, ph = 0u, turn = 0, qs = 0;
    bool ok = true;
    const int kb = wk * kKeys;
    // Byte offset of a key's row in an operand, and its swizzle: 16-byte column c of slab s is at
    // ((offset + s slab) ^ (c << 4)) for a row whose swizzle is folded into the offset.
    const uint32_t slab = (uint32_t)chunk * 128u;
    const auto row_off = [&](int key) -> uint32_t {
      const int r = key & (chunk - 1);
      return (uint32_t)((key >> chunk_shift) * kSlabs) * slab + (uint32_t)r * 128u + (uint32_t)((r & 7) << 4);
    };
    // keys: matrices (keys 0-7, 8-15) x (columns, columns + 8); values: (keys 0-15) x (columns, columns + 8), transposed
    uint32_t koff[kKeys / 16], voff[kKeys / 16];
#pragma unroll
    for (int i = 0; i < kKeys / 16; ++i) {
      koff[i] = row_off(kb + 16 * i + (lane & 7) + ((lane >> 4) << 3)) ^ (((lane >> 3) & 1) << 4);
      voff[i] = row_off(kb + 16 * i + (lane & 15)) ^ ((lane >> 4) << 4);
    }
    while (true) {
      if (!wait_warp(&full_bar[st], ph)) break;
      const Segment g = segs[st];
      if (g.r < 0) break;
      const int len = g.s.len();
      // rows of this lane: 16 wr + gq and + 8.  Rows past the last hold whatever the buffer held: nobody reads theirs.
      const int row0 = 16 * wr + gq;
      uint32_t qf[D / 16][4];
      int seen[2];
      const uint32_t qa = smem_u32(qsm + qs * C::kQBytes + (16 * wr + (lane & 15)) * C::kQRow + (lane >> 4) * 16);
#pragma unroll
      for (int ks = 0; ks < D / 16; ++ks) ldsm4(qf[ks], qa + 32 * ks);
      if (P.negate) {
#pragma unroll
        for (int ks = 0; ks < D / 16; ++ks)
#pragma unroll
          for (int e = 0; e < 4; ++e) qf[ks][e] ^= 0x80008000u;
      }
#pragma unroll
      for (int hf = 0; hf < 2; ++hf) seen[hf] = row0 + 8 * hf < g.s.rows ? g.s.seen(row_token(P, row0 + 8 * hf)) : 0;
      __syncwarp();
      if (lane == 0) mbar_arrive(&qempty_bar[qs]);
      if (++qs == C::kQSlots) qs = 0;
      const int all_see = g.s.seen(0);                 // keys below this are visible to every row
      const bool on = 16 * wr < g.s.rows;              // a warp without rows only keeps step
      float o[D / 8][4];
      float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
#pragma unroll
      for (int j = 0; j < D / 8; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[j][e] = 0.f;
      uint32_t bad = 0;
      for (int t = g.ta; t < g.tb; ++t) {
        if (t > g.ta) {
          // the stage before goes back; the segment's last one is kept for the join
          __syncwarp();
          if (lane == 0) mbar_arrive(&empty_bar[st]);
          if (++st == C::kStages) {
            st = 0;
            ph ^= 1u;
          }
          if (!wait_warp(&full_bar[st], ph)) {
            ok = false;
            break;
          }
        }
        const uint32_t kop = smem_u32(smem + st * C::kStageBytes), vop = kop + C::kOpBytes;
#pragma unroll
        for (int sub = 0; sub < kKeys / kSub; ++sub) {
          const int key0 = t * kTile + kb + sub * kSub;   // its first key
          if (!on || key0 >= len) break;                  // uniform over the warp
          const bool masked = key0 + kSub > all_see;
          float s[kNt][4];
#pragma unroll
          for (int j = 0; j < kNt; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) s[j][e] = 0.f;
#pragma unroll
          for (int ks = 0; ks < D / 16; ++ks)
#pragma unroll
            for (int j = 0; j < kNt; j += 2) {
              uint32_t kf[4];
              ldsm4(kf, (kop + koff[sub * (kSub / 16) + j / 2] + (ks >> 2) * slab) ^ (uint32_t)((ks & 3) << 5));
              mma16816(s[j], qf[ks], kf[0], kf[1]);
              mma16816(s[j + 1], qf[ks], kf[2], kf[3]);
            }
          float top[2] = {-INFINITY, -INFINITY};
#pragma unroll
          for (int j = 0; j < kNt; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              float v = s[j][e] * P.scale_log2;
              if (masked && key0 + 8 * j + 2 * qd + (e & 1) >= seen[e >> 1]) v = -INFINITY;
              s[j][e] = v;
              top[e >> 1] = fmaxf(top[e >> 1], v);
            }
          float f[2], base[2];
#pragma unroll
          for (int hf = 0; hf < 2; ++hf) {
            const float mn = fmaxf(m[hf], quad_max(top[hf]));
            f[hf] = mn == m[hf] ? 1.f : ex2(m[hf] - mn);   // m = -inf: 0
            m[hf] = mn;
            base[hf] = mn == -INFINITY ? 0.f : mn;
          }
          float sum[2] = {0.f, 0.f};
#pragma unroll
          for (int j = 0; j < kNt; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              s[j][e] = ex2(s[j][e] - base[e >> 1]);
              sum[e >> 1] += s[j][e];
            }
#pragma unroll
          for (int hf = 0; hf < 2; ++hf) l[hf] = l[hf] * f[hf] + sum[hf];
          if (__any_sync(0xffffffffu, f[0] != 1.f || f[1] != 1.f)) {
#pragma unroll
            for (int j = 0; j < D / 8; ++j)
#pragma unroll
              for (int e = 0; e < 4; ++e) o[j][e] *= f[e >> 1];
          }
#pragma unroll
          for (int kk = 0; kk < kSub / 16; ++kk) {
            const uint32_t pf[4] = {pack_bf16(s[2 * kk][0], s[2 * kk][1]), pack_bf16(s[2 * kk][2], s[2 * kk][3]),
                                    pack_bf16(s[2 * kk + 1][0], s[2 * kk + 1][1]), pack_bf16(s[2 * kk + 1][2], s[2 * kk + 1][3])};
            const uint32_t va = vop + voff[sub * (kSub / 16) + kk];
            if (!masked) {
#pragma unroll
              for (int j = 0; j < D / 8; j += 2) {
                uint32_t vf[4];   // (keys 0-7, keys 8-15) of columns 8 j, then of 8 j + 8
                ldsm4t(vf, (va + (j >> 3) * slab) ^ (uint32_t)((j & 7) << 4));
                mma16816(o[j], pf, vf[0], vf[1]);
                mma16816(o[j + 1], pf, vf[2], vf[3]);
              }
            } else {
              // Keys past the end become zeros.  A weight of zero does not silence an infinity or a NaN: those of
              // keys that only some rows see are left out, and added at the join where they are seen.
              uint32_t keep[2];
              int part[2];   // bit 0 / 1: key 2 qd / 2 qd + 1 (+ 8) is one that not every row sees
#pragma unroll
              for (int b = 0; b < 2; ++b) {
                const int key = key0 + 16 * kk + 8 * b + 2 * qd;
                keep[b] = (key < len ? 0xFFFFu : 0u) | (key + 1 < len ? 0xFFFF0000u : 0u);
                part[b] = (key >= all_see ? 1 : 0) | (key + 1 >= all_see ? 2 : 0);
              }
#pragma unroll
              for (int j = 0; j < D / 8; j += 2) {
                uint32_t vf[4];
                ldsm4t(vf, (va + (j >> 3) * slab) ^ (uint32_t)((j & 7) << 4));
#pragma unroll
                for (int b = 0; b < 4; ++b) {
                  vf[b] &= keep[b & 1];
                  const uint32_t nf = nonfinite2(vf[b]);
                  uint32_t drop = 0;
                  if ((nf & 1u) && (part[b & 1] & 1)) drop |= 0xFFFFu;
                  if ((nf >> 16) && (part[b & 1] & 2)) drop |= 0xFFFF0000u;
                  bad |= drop;
                  vf[b] &= ~drop;
                }
                mma16816(o[j], pf, vf[0], vf[1]);
                mma16816(o[j + 1], pf, vf[2], vf[3]);
              }
            }
          }
        }
      }
      if (!ok) break;
      // ---- join the WK warps of every row tile, in the stage: [row][D] of warp w lies where its own keys and values
      // were (one row tile), else in w's eighth
      ++turn;
      if (WR > 1 && !meet()) break;
      const auto part_row = [&](int w, int row) -> float* {
        uint8_t* stage = smem + st * C::kStageBytes;
        if (WR > 1) return reinterpret_cast<float*>(stage) + (w * C::kRows + row) * D;
        // 16 keys: kSlabs pieces of 2 KB in each operand, 2048 / (4 D) rows a piece
        constexpr int kPer = 512 / D;
        const int piece = row / kPer, key = 16 * w, op = piece / kSlabs, sl = piece % kSlabs;
        return reinterpret_cast<float*>(stage + op * C::kOpBytes + ((key >> chunk_shift) * kSlabs + sl) * slab +
                                        (key & (chunk - 1)) * 128) + (row % kPer) * D;
      };
      if (turn > 1u && WR == 1) {   // the join before is through: its barrier may be used again
        if (!wait_warp(&join_bar, jph)) break;
        jph ^= 1u;
      }
      if (on) {
#pragma unroll
        for (int hf = 0; hf < 2; ++hf) {
          const int row = row0 + 8 * hf;
          const float sum = quad_sum(l[hf]);
          if (row < g.s.rows) {
            float* dst = part_row(wk, row) + 2 * qd;
#pragma unroll
            for (int j = 0; j < D / 8; ++j) *reinterpret_cast<float2*>(dst + 8 * j) = make_float2(o[j][2 * hf], o[j][2 * hf + 1]);
            if (qd == 0) join_ml[turn & 1][wk * C::kRows + row] = make_float2(m[hf], sum);
          }
        }
        if (bad) bad_s[turn & 3] = 1;
      }
      if constexpr (WR == 1) {
        __syncwarp();
        if (lane == 0) mbar_arrive(&join_bar);
        if (warp < g.s.rows && !wait_warp(&join_bar, jph)) break;   // the others look when they come to the next join
      } else {
        if (!meet()) break;
      }
      const bool fix = bad_s[turn & 3] != 0;
      if (threadIdx.x == 0) bad_s[(turn + 2) & 3] = 0;
      float* slot = g.parts > 1 ? part_slot(P, g.first_cta, g.part, C::kPart) : nullptr;
      for (int row = warp; row < g.s.rows; row += C::kWarps) {   // a warp a row
        const float2 ml = lane < WK ? join_ml[turn & 1][lane * C::kRows + row] : make_float2(-INFINITY, 0.f);
        float mm = ml.x;
#pragma unroll
        for (int d = WK / 2; d > 0; d >>= 1) mm = fmaxf(mm, __shfl_xor_sync(0xffffffffu, mm, d));
        mm = __shfl_sync(0xffffffffu, mm, 0);
        const float fw = ex2(ml.x - (mm == -INFINITY ? 0.f : mm));
        float ll = ml.y * fw;
#pragma unroll
        for (int d = WK / 2; d > 0; d >>= 1) ll += __shfl_xor_sync(0xffffffffu, ll, d);
        ll = __shfl_sync(0xffffffffu, ll, 0);
        float a[kC];
#pragma unroll
        for (int c = 0; c < kC; ++c) a[c] = 0.f;
#pragma unroll
        for (int w = 0; w < WK; ++w) {
          const float f = __shfl_sync(0xffffffffu, fw, w);
          float v[kC];
          L::unpack(reinterpret_cast<const typename L::V*>(part_row(w, row))[lane], v);
#pragma unroll
          for (int c = 0; c < kC; ++c) a[c] = fmaf(v[c], f, a[c]);
        }
        const int tok = row_token(P, row), hd = row - tok * P.group, vis = g.s.seen(tok);
        if (fix) {   // infinities and NaN of keys that only some rows see
          const int end = min(min(len, g.tb * kTile), vis);
#pragma unroll 1
          for (int key = max(all_see, g.ta * kTile); key < end; ++key) {
            const int pg = __ldg(P.table + (int64_t)g.r * P.width + (key >> P.page_shift));
            if (pg < 0 || pg >= P.pages) continue;
            const uint16_t* vr =
                P.v + ((((int64_t)pg * P.kv_heads + g.h) << P.page_shift) + (key & ((1 << P.page_shift) - 1))) * D + kC * lane;
#pragma unroll
            for (int c = 0; c < kC; ++c) {
              const float v = bf16_lo(vr[c]);
              if (!isfinite(v)) a[c] += v;
            }
          }
        }
        if (slot) {
          store_part(slot, row, a, mm, ll);
        } else {
          L::store_bf16(P.out + ((int64_t)(g.s.tok0 + tok) * P.q_heads + g.h * P.group + hd) * D + kC * lane, a,
                        vis > 0 ? 1.f / ll : 0.f);
        }
      }
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");   // the stage was written here; copies overwrite it
      __syncwarp();
      if (lane == 0) mbar_arrive(&empty_bar[st]);
      if (++st == C::kStages) {
        st = 0;
        ph ^= 1u;
      }
      if (slot) {
        // ---- the last of the item's CTAs joins its parts, in order
#pragma unroll 1
        for (int level = 0; level < 2; ++level) {
          const JoinStep j = join_step(g, level, kFlat);
          if (j.n > 1) {
            __threadfence();
            if (!(ok = meet())) break;
            if (threadIdx.x == 0) {
              int32_t* cnt = P.cnt + level * (int)gridDim.x + g.first_cta + j.first;
              last_s = atomicAdd(cnt, 1) == j.n - 1;
              if (last_s) *cnt = 0;
              __threadfence();
            }
            if (!(ok = meet())) break;
            if (!last_s) break;
            for (int row = warp; row < g.s.rows; row += C::kWarps) {   // a warp a row, a lane a part's maximum and sum
              const auto part_at = [&](int i) { return part_slot(P, g.first_cta, j.first + i * j.stride, C::kPart); };
              float2 ml = __ldcg(reinterpret_cast<const float2*>(part_at(min(lane, j.n - 1)) + C::kRows * D + kPartPad * row));
              if (lane >= j.n) ml = make_float2(-INFINITY, 0.f);
              float mm = ml.x;
#pragma unroll
              for (int d = 16; d > 0; d >>= 1) mm = fmaxf(mm, __shfl_xor_sync(0xffffffffu, mm, d));
              const float fp = ex2(ml.x - (mm == -INFINITY ? 0.f : mm));
              float ll = ml.y * fp, a[kC];
#pragma unroll
              for (int d = 16; d > 0; d >>= 1) ll += __shfl_xor_sync(0xffffffffu, ll, d);
#pragma unroll
              for (int c = 0; c < kC; ++c) a[c] = 0.f;
#pragma unroll 1
              for (int p0 = 0; p0 < j.n; p0 += kJoin) {
                typename L::V v[kJoin];
#pragma unroll
                for (int i = 0; i < kJoin; ++i)
                  v[i] = __ldcg(reinterpret_cast<const typename L::V*>(part_at(min(p0 + i, j.n - 1)) + row * D) + lane);
#pragma unroll
                for (int i = 0; i < kJoin; ++i) {
                  const float f = __shfl_sync(0xffffffffu, fp, (p0 + i) & 31);
                  float x[kC];
                  L::unpack(v[i], x);
                  if (p0 + i < j.n) {
#pragma unroll
                    for (int c = 0; c < kC; ++c) a[c] = fmaf(x[c], f, a[c]);
                  }
                }
              }
              if (!j.last) {   // in the place of the group's first part
                store_part(part_at(0), row, a, mm, ll);
              } else {
                const int tok = row_token(P, row), hd = row - tok * P.group;
                L::store_bf16(P.out + ((int64_t)(g.s.tok0 + tok) * P.q_heads + g.h * P.group + hd) * D + kC * lane, a,
                              g.s.seen(tok) > 0 ? 1.f / ll : 0.f);
              }
            }
          }
          if (j.last) break;
        }
        if (!ok) break;
      }
    }
  }
  __syncthreads();
  end_of_waits(abort_flag, P.err);
  if (P.two_launches) start_of_work();   // the chunk launch's end: what follows waits for this one only
}

template <int D, int WR>
gs_status rows_launch(const AttnParams& P, int ctas, cudaStream_t s) {
  using C = RowsCfg<D, WR>;
  static const cudaError_t attr = cudaFuncSetAttribute(k_attn_rows<D, WR>, cudaFuncAttributeMaxDynamicSharedMemorySize, C::kSmem);
  if (attr != cudaSuccess) return GS_ERR_CUDA;
  return launch_behind(k_attn_rows<D, WR>, dim3((unsigned)ctas), C::kThreads, C::kSmem, s, P);
}

}  // namespace

int attn_rows_most() { return kMost; }

int attn_rows_part(int head_dim) { return kMost * (head_dim + kPartPad); }

int attn_rows_box(int page_size) { return page_size < kTile ? page_size : kTile; }

int attn_rows_tile() { return kTile; }

int attn_rows_held(int rows) { return rows <= 16 ? 16 : 32; }

gs_status launch_attn_rows(const AttnParams& P, int head_dim, int ctas, cudaStream_t s) {
  const bool one = P.max_rows == 16;
  if (head_dim == 128) return one ? rows_launch<128, 1>(P, ctas, s) : rows_launch<128, 2>(P, ctas, s);
  return one ? rows_launch<64, 1>(P, ctas, s) : rows_launch<64, 2>(P, ctas, s);
}

}  // namespace gs
