// Attention of few rows (new tokens x query heads a key head, at most 64): decoding
// steps and short chunks.
//
// Bound by HBM: a sequence's keys and values are read once, for all its rows.  A unit
// is 64 keys of a key head.  One warp fetches (TMA, one box per page and operand, a
// ring of 5-6 units = 160-192 KB in flight per SM), the others compute with m16n8k16:
// WR row tiles of 16 x WK shares of the unit's keys, each warp with its own running
// maximum, sum and output, joined over the WK warps once per item.  An MMA row holds
// a query; unused rows cost nothing that matters (the tensor pipe is 5-20 % busy).
#include "gs_attn.cuh"

#include <mutex>

namespace gs {
namespace {
using namespace sm100;

constexpr int kTile = 64;
constexpr uint64_t kArWaitLimitNs = 2000000000ull;

struct FewTraits {
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
__device__ __forceinline__ void ldsm4(uint32_t (&v)[4], uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3])
               : "r"(addr)
               : "memory");
}
__device__ __forceinline__ void ldsm4t(uint32_t (&v)[4], uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3])
               : "r"(addr)
               : "memory");
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

template <int D, int WR, int WK>
struct RowsCfg {
  static constexpr int kWarps = WR * WK;             // consumers
  static constexpr int kThreads = (kWarps + 1) * 32; // + the fetching warp
  static constexpr int kRows = 16 * WR;
  static constexpr int kOpBytes = kTile * D * 2;
  static constexpr int kStageBytes = 2 * kOpBytes;
  static constexpr int kJoinBytes = WK * kRows * (D + 2) * 4;
  static constexpr int kStages = (224 * 1024 - kJoinBytes) / kStageBytes;
  static constexpr int kSmem = kStages * kStageBytes + kJoinBytes + 1024;
  static_assert(kStages >= 4 && kSmem <= 227 * 1024 - 1024, "shared memory budget");
};

template <int D, int WR, int WK>
__global__ void __launch_bounds__(RowsCfg<D, WR, WK>::kThreads, 1) k_attn_rows(const __grid_constant__ AttnParams P) {
  using C = RowsCfg<D, WR, WK>;
  constexpr int kSlabs = D / 64;
  extern __shared__ uint8_t ar_smem_raw[];
  __shared__ __align__(8) uint64_t full_bar[C::kStages];
  __shared__ __align__(8) uint64_t empty_bar[C::kStages];
  __shared__ int64_t red[34];
  __shared__ WorkSlot slots[2];
  __shared__ int abort_s, last_s, bad_s[2];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(ar_smem_raw) + 1023) & ~uintptr_t(1023));
  float* join = reinterpret_cast<float*>(smem + C::kStages * C::kStageBytes);   // [WK][rows][D], then [WK][rows][2]
  float* join_ml = join + WK * C::kRows * D;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int cta = (int)blockIdx.x;
  if (threadIdx.x == 0) {
    for (int s = 0; s < C::kStages; ++s) {
      mbar_init(&full_bar[s], 1);
      mbar_init(&empty_bar[s], C::kWarps);
    }
    abort_s = 0;
    bad_s[0] = bad_s[1] = 0;
    fence_mbar_init();
  }
  const WorkRange range = divide_work<FewTraits, C::kThreads>(P, cta, (int)gridDim.x, red, slots);
  __syncthreads();
  volatile int* abort_flag = &abort_s;
  const int chunk = min(1 << P.page_shift, kTile), chunk_shift = min(P.page_shift, 6);   // rows of a TMA box

  if (warp == C::kWarps) {
    // ------------------------------------------------------------ fetch
    Walker<FewTraits> walk(P, range);
    Segment g;
    const int32_t no_row = (int32_t)((P.pages * P.kv_heads) << P.page_shift);   // past the last: reads as zeros
    uint32_t st = 0, ph = 1u;
    bool ok = true;
    const int per_tile = kTile >> chunk_shift;   // boxes of a whole unit and operand (1, 2 or 4)
    while (ok && walk.next(g, cta)) {
      const int len = g.s.len();
      const int64_t trow = (int64_t)g.r * P.width;
      int held = -1, page = -1;   // lane i holds table entry 32 held + i
      for (int t = g.ta; t < g.tb; ++t) {
        const int valid = min(kTile, max(0, len - t * kTile));
        const int boxes = (valid + chunk - 1) >> chunk_shift;
        // all boxes of a unit have their table entries within one block of 32
        const int e0 = (t * kTile) >> P.page_shift;
        if (e0 >> 5 != held) {
          held = e0 >> 5;
          const int e = 32 * held + lane;
          page = e < P.width && ((int64_t)e << P.page_shift) < len ? __ldg(P.table + trow + e) : -1;
        }
        if (!__all_sync(0xffffffffu, mbar_wait_bounded(&empty_bar[st], ph, abort_flag, P.err, kArWaitLimitNs, kDevErrTimeout))) {
          ok = false;
          break;
        }
        uint8_t* stage = smem + st * C::kStageBytes;
        if (lane == 0) mbar_arrive_expect_tx(&full_bar[st], 2u * (uint32_t)(boxes * chunk * D * 2));
        __syncwarp();
        const int b = lane & 15, key = t * kTile + (b << chunk_shift);
        const int pg = __shfl_sync(0xffffffffu, page, (key >> P.page_shift) & 31);
        if (b < boxes) {
          const int32_t row = pg >= 0 && pg < P.pages
                                  ? (int32_t)((((int64_t)pg * P.kv_heads + g.it.h) << P.page_shift) + (key & ((1 << P.page_shift) - 1)))
                                  : no_row;
          uint8_t* dst = stage + b * (chunk * D * 2);
          if (lane < 16) tma_load_3d(dst, &P.kmap, &full_bar[st], 0, row, 0);
          else tma_load_3d(dst + C::kOpBytes, &P.vmap, &full_bar[st], 0, row, 0);
        }
        __syncwarp();
        if (++st == C::kStages) {
          st = 0;
          ph ^= 1u;
        }
      }
    }
    (void)per_tile;
  } else {
    // ------------------------------------------------------------ compute
    const int wr = warp / WK, wk = warp % WK, gq = lane >> 2, qd = lane & 3;
    constexpr int kKeys = kTile / WK;         // this warp's keys of a unit
    constexpr int kNt = kKeys / 8;
    const auto bar_compute = [&]() { asm volatile("bar.sync 1, %0;" ::"n"(C::kWarps * 32) : "memory"); };
    Walker<FewTraits> walk(P, range);
    Segment g;
    uint32_t st = 0, ph = 0u, turn = 0;
    bool ok = true;
    // a lane's ldmatrix row: keys (K) or keys of the transposed blocks (V), and its 16-byte column
    const int kb = wk * kKeys;
    const auto tile_addr = [&](uint32_t op, int key, int col16) -> uint32_t {   // col16: 16-byte column of the row
      const int box = key >> chunk_shift, r = key & (chunk - 1), slab = col16 >> 3;
      return op + (uint32_t)(((box * kSlabs + slab) << chunk_shift) + r) * 128u + (uint32_t)(((col16 & 7) ^ (r & 7)) << 4);
    };
    while (ok && walk.next(g, cta)) {
      const int len = g.s.len();
      // rows of this lane: 16 wr + gq and + 8
      const int row0 = 16 * wr + gq;
      uint32_t qf[D / 16][4];
      int seen[2];
#pragma unroll
      for (int hf = 0; hf < 2; ++hf) {
        const int row = row0 + 8 * hf;
        const bool on = row < g.s.rows;
        const int tok = on ? row / P.group : 0, hd = on ? row - tok * P.group : 0;
        seen[hf] = on ? g.s.seen(tok) : 0;
        const uint32_t* src = reinterpret_cast<const uint32_t*>(P.q + (int64_t)(g.s.tok0 + tok) * P.q_stride +
                                                                (int64_t)(g.it.h * P.group + hd) * D) + qd;
        const uint32_t flip = P.negate ? 0x80008000u : 0u;
#pragma unroll
        for (int ks = 0; ks < D / 16; ++ks) {
          qf[ks][hf] = on ? __ldg(src + 8 * ks) ^ flip : 0u;
          qf[ks][hf + 2] = on ? __ldg(src + 8 * ks + 4) ^ flip : 0u;
        }
      }
      const int all_see = g.s.seen(0);                 // keys below this are visible to every row
      const bool work = 16 * wr < g.s.rows;            // a warp without rows only keeps step
      float o[D / 8][4];
      float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
#pragma unroll
      for (int j = 0; j < D / 8; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[j][e] = 0.f;
      uint32_t bad = 0;
      for (int t = g.ta; t < g.tb; ++t) {
        if (!__all_sync(0xffffffffu, mbar_wait_bounded(&full_bar[st], ph, abort_flag, P.err, kArWaitLimitNs, kDevErrTimeout))) {
          ok = false;
          break;
        }
        if (work) {
          const uint32_t kop = smem_u32(smem + st * C::kStageBytes), vop = kop + C::kOpBytes;
          const int key0 = t * kTile + kb;             // the warp's first key
          const bool masked = key0 + kKeys > all_see;
          float s[kNt][4];
#pragma unroll
          for (int j = 0; j < kNt; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) s[j][e] = 0.f;
          // two key tiles (16 keys) and one 16-deep step per ldmatrix: matrices (keys 0-7, 8-15) x (columns, columns + 8)
#pragma unroll
          for (int ks = 0; ks < D / 16; ++ks)
#pragma unroll
            for (int j = 0; j < kNt; j += 2) {
              uint32_t kf[4];
              ldsm4(kf, tile_addr(kop, kb + 8 * j + (lane & 7) + ((lane >> 4) << 3), 2 * ks + ((lane >> 3) & 1)));
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
          float f[2];
#pragma unroll
          for (int hf = 0; hf < 2; ++hf) {
            const float mn = fmaxf(m[hf], quad_max(top[hf]));
            f[hf] = mn == m[hf] ? 1.f : ex2(m[hf] - mn);   // m = -inf: 0
            m[hf] = mn;
          }
          const float base[2] = {m[0] == -INFINITY ? 0.f : m[0], m[1] == -INFINITY ? 0.f : m[1]};
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
          for (int kk = 0; kk < kKeys / 16; ++kk) {
            const uint32_t pf[4] = {pack_bf16(s[2 * kk][0], s[2 * kk][1]), pack_bf16(s[2 * kk][2], s[2 * kk][3]),
                                    pack_bf16(s[2 * kk + 1][0], s[2 * kk + 1][1]), pack_bf16(s[2 * kk + 1][2], s[2 * kk + 1][3])};
            // which keys of this lane's fragments exist: 2 qd, 2 qd + 1, and the same + 8
            uint32_t keep[2] = {0xFFFFFFFFu, 0xFFFFFFFFu};
            if (masked) {
#pragma unroll
              for (int b = 0; b < 2; ++b) {
                const int key = key0 + 16 * kk + 8 * b + 2 * qd;
                keep[b] = (key < len ? 0xFFFFu : 0u) | (key + 1 < len ? 0xFFFF0000u : 0u);
              }
            }
#pragma unroll
            for (int j = 0; j < D / 8; j += 2) {
              uint32_t vf[4];   // (keys 0-7, keys 8-15) of columns 8 j, then of 8 j + 8
              ldsm4t(vf, tile_addr(vop, kb + 16 * kk + (lane & 15), j + (lane >> 4)));
              if (masked) {
#pragma unroll
                for (int b = 0; b < 4; ++b) {
                  vf[b] &= keep[b & 1];
                  const uint32_t nf = nonfinite2(vf[b]);   // a weight of zero does not silence it: the join adds it where seen
                  const int key = key0 + 16 * kk + 8 * (b & 1) + 2 * qd;
                  uint32_t drop = 0;
                  if ((nf & 1u) && key >= all_see) drop |= 0xFFFFu;
                  if ((nf >> 16) && key + 1 >= all_see) drop |= 0xFFFF0000u;
                  bad |= drop;
                  vf[b] &= ~drop;
                }
              }
              mma16816(o[j], pf, vf[0], vf[1]);
              mma16816(o[j + 1], pf, vf[2], vf[3]);
            }
          }
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(&empty_bar[st]);
        if (++st == C::kStages) {
          st = 0;
          ph ^= 1u;
        }
      }
      if (!ok) break;
      // ---- join the WK warps of every row tile
      ++turn;
      if (work) {
#pragma unroll
        for (int hf = 0; hf < 2; ++hf) {
          const int row = row0 + 8 * hf;
          float* dst = join + ((size_t)wk * C::kRows + row) * D + 2 * qd;
#pragma unroll
          for (int j = 0; j < D / 8; ++j) *reinterpret_cast<float2*>(dst + 8 * j) = make_float2(o[j][2 * hf], o[j][2 * hf + 1]);
          const float sum = quad_sum(l[hf]);
          if (qd == 0) *reinterpret_cast<float2*>(join_ml + ((size_t)wk * C::kRows + row) * 2) = make_float2(m[hf], sum);
        }
        if (bad) bad_s[turn & 1] = 1;
      }
      bar_compute();
      const bool fix = bad_s[turn & 1] != 0;
      if (threadIdx.x == 0) bad_s[(turn + 1) & 1] = 0;
      float* slot = g.parts > 1 ? part_slot(P, g.first_cta, g.part, C::kRows, D) : nullptr;
      const int key_end = min(len, g.tb * kTile), key_begin = max(all_see, g.ta * kTile);
      for (int i = threadIdx.x; i < g.s.rows * (D / 4); i += C::kWarps * 32) {
        const int row = i / (D / 4), d = 4 * (i % (D / 4));
        float mm = -INFINITY, ll = 0.f;
#pragma unroll
        for (int w = 0; w < WK; ++w) mm = fmaxf(mm, join_ml[(w * C::kRows + row) * 2]);
        const float b = mm == -INFINITY ? 0.f : mm;
        float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int w = 0; w < WK; ++w) {
          const float2 ml = *reinterpret_cast<const float2*>(join_ml + (w * C::kRows + row) * 2);
          const float fw = ex2(ml.x - b);
          const float4 v = *reinterpret_cast<const float4*>(join + ((size_t)w * C::kRows + row) * D + d);
          ll = fmaf(ml.y, fw, ll);
          a.x = fmaf(v.x, fw, a.x);
          a.y = fmaf(v.y, fw, a.y);
          a.z = fmaf(v.z, fw, a.z);
          a.w = fmaf(v.w, fw, a.w);
        }
        const int tok = row / P.group, hd = row - tok * P.group, vis = g.s.seen(tok);
        if (fix) {   // infinities and NaN of keys that only some rows see
          for (int key = key_begin; key < min(key_end, vis); ++key) {
            const int pg = __ldg(P.table + (int64_t)g.r * P.width + (key >> P.page_shift));
            if (pg < 0 || pg >= P.pages) continue;
            const uint16_t* vr = P.v + ((((int64_t)pg * P.kv_heads + g.it.h) << P.page_shift) + (key & ((1 << P.page_shift) - 1))) * D + d;
            const float v0 = bf16_lo(vr[0]), v1 = bf16_lo(vr[1]), v2 = bf16_lo(vr[2]), v3 = bf16_lo(vr[3]);
            if (!isfinite(v0)) a.x += v0;
            if (!isfinite(v1)) a.y += v1;
            if (!isfinite(v2)) a.z += v2;
            if (!isfinite(v3)) a.w += v3;
          }
        }
        if (slot) {
          *reinterpret_cast<float4*>(slot + (size_t)row * D + d) = a;
          if (d == 0) *reinterpret_cast<float2*>(slot + (size_t)C::kRows * D + 2 * row) = make_float2(mm, ll);
        } else {
          const float inv = vis > 0 ? 1.f / ll : 0.f;
          *reinterpret_cast<uint2*>(P.out + ((int64_t)(g.s.tok0 + tok) * P.q_heads + g.it.h * P.group + hd) * D + d) =
              make_uint2(pack_bf16(a.x * inv, a.y * inv), pack_bf16(a.z * inv, a.w * inv));
        }
      }
      if (slot) {
        // ---- the last of the item's CTAs joins its parts, in order
        __threadfence();
        bar_compute();
        if (threadIdx.x == 0) {
          const int got = atomicAdd(P.cnt + g.first_cta, 1);
          last_s = got == g.parts - 1;
          if (last_s) P.cnt[g.first_cta] = 0;
          __threadfence();
        }
        bar_compute();
        if (last_s) {
          for (int i = threadIdx.x; i < g.s.rows * (D / 4); i += C::kWarps * 32) {
            const int row = i / (D / 4), d = 4 * (i % (D / 4));
            float mm = -INFINITY, ll = 0.f;
            float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
            for (int p = 0; p < g.parts; ++p) {
              const float* sp = part_slot(P, g.first_cta, p, C::kRows, D);
              const float2 ml = __ldcg(reinterpret_cast<const float2*>(sp + (size_t)C::kRows * D + 2 * row));
              const float4 v = __ldcg(reinterpret_cast<const float4*>(sp + (size_t)row * D + d));
              const float mn = fmaxf(mm, ml.x), b = mn == -INFINITY ? 0.f : mn;
              const float f0 = ex2(mm - b), f1 = ex2(ml.x - b);
              ll = ll * f0 + ml.y * f1;
              a.x = a.x * f0 + v.x * f1;
              a.y = a.y * f0 + v.y * f1;
              a.z = a.z * f0 + v.z * f1;
              a.w = a.w * f0 + v.w * f1;
              mm = mn;
            }
            const int tok = row / P.group, hd = row - tok * P.group;
            const float inv = g.s.seen(tok) > 0 ? 1.f / ll : 0.f;
            *reinterpret_cast<uint2*>(P.out + ((int64_t)(g.s.tok0 + tok) * P.q_heads + g.it.h * P.group + hd) * D + d) =
                make_uint2(pack_bf16(a.x * inv, a.y * inv), pack_bf16(a.z * inv, a.w * inv));
          }
        }
      }
      bar_compute();   // the join buffers may be written again
    }
    // ---- rows that nothing computes: tokens of no sequence, and sequences of more rows than were announced
    const int64_t row16 = (int64_t)P.q_heads * D / 8;   // 16-byte pieces of a token's output
    const auto zero = [&](int64_t t0, int64_t t1) {
      for (int64_t i = t0 * row16 + threadIdx.x; i < t1 * row16; i += C::kWarps * 32)
        reinterpret_cast<uint4*>(P.out)[i] = make_uint4(0u, 0u, 0u, 0u);
    };
    const int64_t before = min((int64_t)max(0, __ldg(P.offsets)), P.tokens), after = max(0, __ldg(P.offsets + P.n_seqs));
    for (int64_t t = cta; t < before; t += gridDim.x) zero(t, t + 1);
    for (int64_t t = after + cta; t < P.tokens; t += gridDim.x) zero(t, t + 1);
    if (P.zero_rest)
      for (int r = cta; r < P.n_seqs; r += (int)gridDim.x) {
        const SeqInfo s = seq_info(P, r);
        if (s.rows > P.max_rows) zero(s.tok0, (int64_t)s.tok0 + s.n);
      }
  }
  __syncthreads();
  if (abort_s) {
    // a role gave up: give copies in flight time to land
    const uint64_t t0 = globaltimer_ns();
    while (globaltimer_ns() - t0 < 2000000ull) {
    }
  }
}

template <int D, int WR, int WK>
gs_status rows_launch(const AttnParams& P, int ctas, cudaStream_t s) {
  using C = RowsCfg<D, WR, WK>;
  static const cudaError_t attr =
      cudaFuncSetAttribute(k_attn_rows<D, WR, WK>, cudaFuncAttributeMaxDynamicSharedMemorySize, C::kSmem);
  if (attr != cudaSuccess) return GS_ERR_CUDA;
  k_attn_rows<D, WR, WK><<<(unsigned)ctas, C::kThreads, C::kSmem, s>>>(P);
  note_launch();
  return cudaGetLastError() == cudaSuccess ? GS_OK : GS_ERR_CUDA;
}

}  // namespace

int attn_rows_most() { return 64; }

int attn_rows_box(int page_size) { return page_size < kTile ? page_size : kTile; }

// rows: an upper bound of the rows of the sequences that are this kernel's
gs_status launch_attn_rows(const AttnParams& P, int head_dim, int rows, int ctas, cudaStream_t s) {
  if (head_dim == 128)
    return rows <= 16 ? rows_launch<128, 1, 4>(P, ctas, s) : rows <= 32 ? rows_launch<128, 2, 4>(P, ctas, s)
                                                                        : rows_launch<128, 4, 2>(P, ctas, s);
  return rows <= 16 ? rows_launch<64, 1, 4>(P, ctas, s) : rows <= 32 ? rows_launch<64, 2, 4>(P, ctas, s)
                                                                     : rows_launch<64, 4, 2>(P, ctas, s);
}

}  // namespace gs
