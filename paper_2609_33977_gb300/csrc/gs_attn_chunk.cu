// Attention of many rows (new tokens x query heads a key head): chunks of a prompt,
// whole prompts.
//
// Bound by the tensor cores (4 head_dim FLOP a visible pair) and by the exponentials
// beside them.  An item is up to 256 rows of a key head (whole tokens, two halves)
// against its visible keys, a unit 64 keys.  A half has 128 lanes, one per softmax warpgroup, whose thread
// i owns row i, so that maxima and sums need no exchange.  Per half and unit:
//     S = Q K^T (tcgen05, both operands in shared memory, S in TMEM), the thread
//     reads its row of S, writes P = exp2(c S - m) beside it as bf16, and
//     O += P V (A = P in TMEM, B = V as stored, i.e. MN-major), O stays in TMEM.
// P has 8 significant bits because the bf16 product takes no more: each weight is off by
// 2^-8 of itself at most, like noise over the keys; the output, which is rounded to as many
// bits, has a relative error of 0.0021 against 64 bits, 0.0016 without that (prompts of up
// to 4096 tokens).  The sums of weights are float32, from before that rounding.
// P has its own columns (two buffers), so that S of the next unit can be formed as
// soon as this one has been read, under its exponentials.  Each half has two MMA
// warps, for S and for P V: a warp's waits and issue of both in turn took longer than
// the exponentials.  (P over S, in units of 64 or 128 keys, chains S, exponentials and P V
// behind each other: 1.3 to 2 times the time.)
// O is rescaled only when a row's maximum grew by more than 2^8 (each row for
// itself), else the old maximum stays in use: exact, since both the sum and O carry it.
//
// Keys and values arrive page by page (TMA) in rings of five 16 KB slots each.  Values
// of a unit that some row does not see are looked over first: rows past the sequence's
// end become zeros, and infinities and NaN are taken out (a weight of zero would not
// silence them) and added at the end to the rows that see them.
//
// 8192 new tokens, 40 heads: 513 us, 1340 TFLOP/s of the pairs that are seen; 4096: 154 us,
// 1115; prompts of 4096, 1023, 1777 and 300: 204 us, 1060; 512 tokens at 8192 keys, 28/4
// heads: 65 us, 890.  Heads of 64, 16/2 of them: 4096 new tokens 62 us, 550, and 512 at 8192
// keys 38 us, 435 (the exponentials are as many, the products half).  What short items lose is their ends: the first keys' way to the
// exponentials, and the last output's way out of TMEM (some 6000 cycles an item in all,
// a unit takes 1550).
//
// TMEM: per half S (64 columns) and two P (32 each) from column 0 / 128, O from 256 / 384.
//
// Over a cache in 8 bits (k8) eight more warps turn the codes of a unit, as they arrive, into the bf16 tiles that the products
// read: a code's bits moved to where bf16 has its own, times 2^(120 + e), exactly.  Every item converts the keys that it sees, so
// half as many warps, or short items, wait for the conversion; otherwise it costs issue slots and shared memory's time, and the softmax
// its registers (144 a thread instead of 200).  Prompts as above 267 us, 807 TFLOP/s (235 if nothing is converted; four converting
// warps and 168 registers 323); 4096 tokens 202; 512 at 8192 keys 83.4; 64 at 8192, whose items have one half, 49.5.  Queries of one
// half in TMEM, for one buffer of P a half instead of two: 341.
#include "gs_attn.cuh"

namespace gs {
namespace {
using namespace sm100;

constexpr int kCT = 64;                        // keys of a unit
constexpr int kHalf = 128;                     // lanes of a half
constexpr int kPartRows = 2 * kHalf;           // rows of a part in the workspace
constexpr int kPartPad = 2;                    // floats of a row of it beside the output's
constexpr int kSegs = 4;
constexpr int kFlat = 6;                       // parts joined in one level (16 tokens at 60000 keys, 28/4 heads: 52 us; always one level: 95)

// kOver 4 / 5 / 6 / 8: prompts as above 201 / 204 / 206 / 209 us, 6 x 1024 tokens of 32 heads 84 / 82 / 83 / 87, a mixed
// step of 681 tokens 78 / 78 / 77 / 80; 0 (with longer ends: 275 against 231 at 5, the mixed step 132 against 82).
// kSnap 1 / 3 / 6 (then): prompts 224 / 221 / 222, the mixed step 82 / 82 / 84.  kLeast 6 / 8 / 12: 30 tokens at 8192 keys
// (28/4 heads) 39 / 34 / 36, 64 tokens 35 / 37 / 38.
struct ChunkTraits {
  static constexpr int kLeast = 8, kSnap = 3, kOver = 5;
  static constexpr bool kOneTile = false;
  // A half holds whole tokens (P.half_tokens: group x that of its 128 lanes are used), an item two halves.
  static __device__ __forceinline__ int row_tiles(const SeqInfo& s, const AttnParams& P) {
    if (s.rows < P.min_rows || s.rows > P.max_rows) return 0;
    const int t = 2 * P.half_tokens;
    return (s.n + t - 1) / t;
  }
  // units that the tokens before `end` of a sequence see
  static __device__ __forceinline__ int units_of(const SeqInfo& s, int end) {
    return max(1, (s.seen(min(end, s.n) - 1) + kCT - 1) / kCT);
  }
  static __device__ __forceinline__ int tiles(const SeqInfo& s, const AttnParams& P, int rt) {
    return units_of(s, 2 * (rt + 1) * P.half_tokens);
  }
};

template <int D, bool k8>
struct ChunkCfg {
  // warps: keys, values, S x 2, P V x 2, two value checkers; two softmax warpgroups; in 8 bits four converters of keys and
  // four of values (no checkers)
  static constexpr int kThreads = k8 ? 768 : 512;
  static constexpr int kRing = k8 ? 3 : 5;             // slots of keys, and as many of values, as the products read them
  static constexpr int kRawRing = k8 ? 4 : kRing;      // slots that they arrive in: codes, converted into the others
  static constexpr int kCleaners = k8 ? 4 : 2;         // warps that have a part in a slot of values (of keys, in 8 bits)
  static constexpr int kRegsOther = k8 ? 48 : 56, kRegsSoftmax = k8 ? 144 : 200;
  static_assert(32 * ((kThreads / 32 - 8) * kRegsOther + 8 * kRegsSoftmax) <= kThreads * (65536 / kThreads / 8 * 8), "register split");
  // parts under way at once in a join (2 and 4: the same within 2 %; in 8 bits, where registers are short, 1 is 2 % faster than 3)
  static constexpr int kJoin = k8 ? 1 : 3;
  static constexpr int kOpBytes = kCT * D * 2;         // a unit's keys or values
  static constexpr int kRawBytes = kCT * D * (k8 ? 1 : 2);
  static constexpr int kQBytes = kHalf * D * 2;        // a half's queries
  static constexpr int kSmem = 2 * kQBytes + 2 * kRing * kOpBytes + (k8 ? 2 * kRawRing * kRawBytes : 0) + 1024;
  static constexpr int kSlabs = D / 64;
};

// The MMA warps run converged, and one lane (`on`) issues: guarded instructions instead of a branch keep the operands in
// uniform registers, which the tensor instructions take.
__device__ __forceinline__ void mma_ss(uint32_t d_tmem, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t accumulate,
                                       uint32_t on) {
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "setp.ne.b32 q, %5, 0;\n\t"
      "@q tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
      ::"r"(d_tmem), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate), "r"(on)
      : "memory");
}
// A in TMEM
__device__ __forceinline__ void mma_ts(uint32_t d_tmem, uint32_t a_tmem, uint64_t bdesc, uint32_t idesc, uint32_t accumulate,
                                       uint32_t on) {
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "setp.ne.b32 q, %5, 0;\n\t"
      "@q tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
      ::"r"(d_tmem), "r"(a_tmem), "l"(bdesc), "r"(idesc), "r"(accumulate), "r"(on)
      : "memory");
}
__device__ __forceinline__ void commit_to(uint64_t* bar, uint32_t on) {
  asm volatile(
      "{\n\t.reg .pred q;\n\t"
      "setp.ne.b32 q, %1, 0;\n\t"
      "@q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t}" ::"r"(smem_u32(bar)), "r"(on)
      : "memory");
}
__device__ __forceinline__ void tmem_st_x32(uint32_t taddr, const uint32_t (&v)[32]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,"
      "%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31,%32};" ::"r"(taddr),
      "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]), "r"(v[9]), "r"(v[10]),
      "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15]), "r"(v[16]), "r"(v[17]), "r"(v[18]), "r"(v[19]), "r"(v[20]),
      "r"(v[21]), "r"(v[22]), "r"(v[23]), "r"(v[24]), "r"(v[25]), "r"(v[26]), "r"(v[27]), "r"(v[28]), "r"(v[29]), "r"(v[30]),
      "r"(v[31])
      : "memory");
}
// Shared-memory descriptors, 128-byte swizzle, 8-row groups 1024 bytes apart: the upper word is the same for all, the lower
// one has the address and, for the values (MN-major), the distance of their 64-channel blocks.
constexpr uint32_t kDescHi = (1024u >> 4) | (1u << 14) | (2u << 29);
__device__ __forceinline__ uint32_t desc_lo(uint32_t saddr, uint32_t block) { return (saddr >> 4) | ((block >> 4) << 16); }
__device__ __forceinline__ uint64_t desc(uint32_t lo) { return ((uint64_t)kDescHi << 32) | lo; }
__device__ __forceinline__ float max3(float a, float b, float c) { return fmaxf(fmaxf(a, b), c); }
__device__ __forceinline__ uint32_t nonfinite2(uint32_t v) {   // bits of the halves that are an infinity or NaN
  const uint32_t e = v & 0x7F807F80u;
  return ((e & 0xFFFFu) == 0x7F80u ? 0xFFFFu : 0u) | ((e >> 16) == 0x7F80u ? 0xFFFF0000u : 0u);
}

// two float32 at once
__device__ __forceinline__ uint64_t pair(uint32_t lo, uint32_t hi) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "r"(lo), "r"(hi));
  return r;
}
__device__ __forceinline__ void unpair(uint64_t v, uint32_t& lo, uint32_t& hi) { asm("mov.b64 {%0, %1}, %2;" : "=r"(lo), "=r"(hi) : "l"(v)); }
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t d;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
  return d;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
  uint64_t d;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}

// from L2, in program order: loads that are written together are under way together
__device__ __forceinline__ float4 load_part(const float* p) {
  float4 v;
  asm volatile("ld.global.cg.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "l"(p));
  return v;
}
__device__ __forceinline__ float2 load_ml(const float* p) {
  float2 v;
  asm volatile("ld.global.cg.v2.f32 {%0, %1}, [%2];" : "=f"(v.x), "=f"(v.y) : "l"(p));
  return v;
}

// within a unit in the last place (the output is rounded to 8 bits of fraction)
__device__ __forceinline__ float reciprocal(float x) {
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// 64 bytes at an address that is a multiple of 16: whole 32-byte sectors where it is one of 32
__device__ __forceinline__ void store_sectors(uint16_t* p, const uint32_t (&w)[16]) {
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    if ((reinterpret_cast<uintptr_t>(p) & 16) == 0) {
      asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p + 16 * i), "r"(w[8 * i]), "r"(w[8 * i + 1]),
                   "r"(w[8 * i + 2]), "r"(w[8 * i + 3]), "r"(w[8 * i + 4]), "r"(w[8 * i + 5]), "r"(w[8 * i + 6]), "r"(w[8 * i + 7])
                   : "memory");
    } else {
      uint4* q = reinterpret_cast<uint4*>(p + 16 * i);
      q[0] = make_uint4(w[8 * i], w[8 * i + 1], w[8 * i + 2], w[8 * i + 3]);
      q[1] = make_uint4(w[8 * i + 4], w[8 * i + 5], w[8 * i + 6], w[8 * i + 7]);
    }
  }
}

// 16 bytes of shared memory in one access (a choice among them by lane makes four of it otherwise, with bank conflicts: 283 us
// for the prompts below)
__device__ __forceinline__ uint4 load16(uint32_t at) {
  uint4 v;
  asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at) : "memory");
  return v;
}
__device__ __forceinline__ void store16(uint32_t at, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}
// two bf16 times a power of two (twice the same)
__device__ __forceinline__ uint32_t times(uint32_t x, uint32_t m) {
  asm("mul.rn.bf16x2 %0, %0, %1;" : "+r"(x) : "r"(m));
  return x;
}
// Two e4m3 codes of a word as bf16, times m.  A code's four exponent and three fraction bits are moved to where bf16 has the
// ends of its own, which makes them 2^-120 of their value (zeros and subnormals too); the product is exact.  kPick: the codes into
// the upper bytes.  m = 2^(120 + e) is a bf16 up to e = 7, the power kHighPower.
// Values become 2^-kDown of what they are, which the division by the sum of weights gives back: sums of up to 2^16 of the largest
// (448 * 2^119, weights of up to 2^8) stay in float32's range so, and the smallest codes (2^-109) are still bf16's least number.
constexpr uint32_t kHighPower = 134u, kDown = 24u;
template <uint32_t kPick>
__device__ __forceinline__ uint32_t bf16_of(uint32_t codes, uint32_t m) {
  const uint32_t t = __byte_perm(codes, 0u, kPick);
  return times((t & 0x80008000u) | ((t >> 4) & 0x07F007F0u), m);
}
// two bf16: 0 x + c
__device__ __forceinline__ uint32_t times_zero(uint32_t x, uint32_t c) {
  uint32_t d;
  asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(d) : "r"(x), "r"(0u), "r"(c));
  return d;
}

template <int D, bool k8>
__global__ void __launch_bounds__(ChunkCfg<D, k8>::kThreads, 1) k_attn_chunk(const __grid_constant__ AttnParams P) {
  using C = ChunkCfg<D, k8>;
  constexpr int kRing = C::kRing, kRawRing = C::kRawRing;
  extern __shared__ uint8_t ac_smem_raw[];
  // of keys, of values: bytes have landed, the slot they landed in is free
  __shared__ __align__(8) uint64_t full_bars[2][kRawRing], empty_bars[2][kRawRing];
  // values looked over; in 8 bits, keys or values converted, and the slot of the converted ones free
  __shared__ __align__(8) uint64_t clean_bars[2][kRing], done_bars[2][k8 ? kRing : 1];
  uint64_t(&kfull_bar)[kRawRing] = full_bars[0];
  uint64_t(&kempty_bar)[kRawRing] = empty_bars[0];
  uint64_t(&vfull_bar)[kRawRing] = full_bars[1];
  uint64_t(&vempty_bar)[kRawRing] = empty_bars[1];
  uint64_t(&clean_bar)[kRing] = clean_bars[1];
  __shared__ __align__(16) uint8_t powers[2][k8 ? kRawRing : 1][k8 ? kCT : 16];            // of keys, of values
  __shared__ __align__(8) uint64_t seg_full[kSegs], seg_empty[kSegs];
  __shared__ __align__(8) uint64_t q_bar[2], qempty_bar[2];   // a half's queries are in shared memory, are not needed any more
  __shared__ __align__(8) uint64_t s_bar[2];           // S is in TMEM (and the P V is over whose P this unit's replaces)
  __shared__ __align__(8) uint64_t sfree_bar[2];       // S has been read
  __shared__ __align__(8) uint64_t p_bar[2][2];        // [half][buffer]: P is in TMEM, O is rescaled
  __shared__ __align__(8) uint64_t o_bar[2][2];        // [half][buffer]: P V is over
  __shared__ __align__(8) uint64_t join_bar[2];
  __shared__ __align__(8) uint64_t drain_bar[4];
  __shared__ Segment segs[kSegs];
  __shared__ WorkShared work;
  __shared__ uint32_t tmem_base_s;
  __shared__ int abort_s, bad_s[kSegs], last_s[2];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(ac_smem_raw) + 1023) & ~uintptr_t(1023));
  uint8_t* ring_k = smem + 2 * C::kQBytes;
  uint8_t* ring_v = ring_k + kRing * C::kOpBytes;
  uint8_t* raw_k = k8 ? ring_v + kRing * C::kOpBytes : ring_k;   // where keys and values arrive
  uint8_t* raw_v = k8 ? raw_k + kRawRing * C::kRawBytes : ring_v;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int cta = (int)blockIdx.x;
  if (threadIdx.x == 0) {
    for (int s = 0; s < kRawRing; ++s) {
      mbar_init(&kfull_bar[s], 1);
      mbar_init(&kempty_bar[s], k8 ? C::kCleaners : 2);   // both MMA warps
      mbar_init(&vfull_bar[s], 1);
      mbar_init(&vempty_bar[s], k8 ? C::kCleaners : 2);
    }
    for (int s = 0; s < kRing; ++s) {
      mbar_init(&clean_bar[s], C::kCleaners);
      if constexpr (k8) {
        mbar_init(&clean_bars[0][s], C::kCleaners);
        mbar_init(&done_bars[0][s], 2);
        mbar_init(&done_bars[1][s], 2);
      }
    }
    for (int s = 0; s < kSegs; ++s) {
      mbar_init(&seg_full[s], 1);
      mbar_init(&seg_empty[s], k8 ? 21 : 15);   // every warp that has a part in it but the one that fills it
    }
    for (int h = 0; h < 2; ++h) {
      mbar_init(&q_bar[h], 1);
      mbar_init(&qempty_bar[h], 1);
      mbar_init(&s_bar[h], 1);
      mbar_init(&sfree_bar[h], 4);
      for (int b = 0; b < 2; ++b) {
        mbar_init(&p_bar[h][b], 4);
        mbar_init(&o_bar[h][b], 1);
      }
      mbar_init(&join_bar[h], 4);
    }
    for (int i = 0; i < 4; ++i) mbar_init(&drain_bar[i], 1);
    abort_s = 0;
    fence_mbar_init();
    prefetch_tmap(&P.kmap);
    prefetch_tmap(&P.vmap);
    prefetch_tmap(&P.qmap);
  }
  if (warp == 2) {
    tmem_alloc(&tmem_base_s, 512);
    tmem_relinquish();
  }
  start_of_work();
  if (P.two_launches) asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const Shares shares = divide_work<ChunkTraits, C::kThreads>(P, cta, work);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = (uint32_t)uniform((int)tmem_base_s);
  volatile int* abort_flag = &abort_s;
  const int box_shift = min(P.page_shift, 6), box = 1 << box_shift;   // rows of a TMA box
  const auto wait_warp = [&](uint64_t* bar, uint32_t parity) {
    return mbar_wait_warp(bar, parity, abort_flag);
  };
  // A half's units end where its last row's keys end.
  const auto half_tok = [&](const Segment& g, int h) { return (2 * g.rt + h) * P.half_tokens; };   // its first token
  const auto half_end = [&](const Segment& g, int h) { return min(g.tb, ChunkTraits::units_of(g.s, half_tok(g, h + 1))); };
  const auto halves = [&](const Segment& g) { return g.s.n > half_tok(g, 1) ? 2 : 1; };

  if (warp < 8 || warp >= 16) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(C::kRegsOther));
    uint32_t sg = 0, sph = 0;          // segment slot and its phase
    const auto next_seg = [&]() {
      __syncwarp();
      if (lane == 0) mbar_arrive(&seg_empty[sg]);
      if (++sg == kSegs) {
        sg = 0;
        sph ^= 1u;
      }
    };
    if (warp < 2) {
      // ---------------------------------------------------------- copies: warp 0 keys (it also walks the work), warp 1 values
      const bool keys = warp == 0;
      Walker<ChunkTraits> walk(P, shares, work, cta);
      Segment g;
      const int32_t no_row = (int32_t)((P.pages * P.kv_heads) << P.page_shift);   // past the last: reads as zeros
      uint64_t* full_bar = keys ? kfull_bar : vfull_bar;
      uint64_t* empty_bar = keys ? kempty_bar : vempty_bar;
      uint8_t* ring = keys ? raw_k : raw_v;
      uint32_t slot = 0, ph = 1u, qph0 = 1u, qph1 = 1u;
      bool ok = !keys || !injected_timeout(P, cta, abort_flag);
      while (ok) {
        if (keys) {
          const bool more = walk.next(g);
          if (!wait_warp(&seg_empty[sg], sph ^ 1u)) break;
          if (lane == 0) {
            if (!more) g.r = -1;
            segs[sg] = g;
            bad_s[sg] = 0;
            mbar_arrive(&seg_full[sg]);
          }
          __syncwarp();
          if (++sg == kSegs) {
            sg = 0;
            sph ^= 1u;
          }
          if (!more) break;
          for (int h = 0; h < halves(g) && ok; ++h) {   // queries: rows of (token, head), a slab of 64 channels a box
            if (g.ta >= half_end(g, h)) continue;
            if (!wait_warp(&qempty_bar[h], h ? qph1 : qph0)) {
              ok = false;
              break;
            }
            if (h) qph1 ^= 1u;
            else qph0 ^= 1u;
            if (elect_one()) {
              mbar_arrive_expect_tx(&q_bar[h], (uint32_t)(P.half_tokens * P.group * D * 2));
#pragma unroll
              for (int sl = 0; sl < C::kSlabs; ++sl)
                tma_load_3d(smem + h * C::kQBytes + sl * (kHalf * 128), &P.qmap, &q_bar[h], 64 * sl, g.h * P.group,
                            g.s.tok0 + half_tok(g, h));
            }
            __syncwarp();
          }
          if (!ok) break;
        } else {
          if (!wait_warp(&seg_full[sg], sph)) break;
          g = segs[sg];
          next_seg();
          if (g.r < 0) break;
        }
        const int len = g.s.len();
        const int64_t trow = (int64_t)g.r * P.width;
        int held = -1, page = -1;   // lane i holds table entry 32 held + i
        for (int t = g.ta; t < g.tb; ++t) {
          const int valid = min(kCT, max(0, len - t * kCT));
          const int boxes = (valid + box - 1) >> box_shift;   // at most 4
          const int e0 = (t * kCT) >> P.page_shift;
          if (e0 >> 5 != held) {
            held = e0 >> 5;
            const int e = 32 * held + lane;
            page = e < P.width && ((int64_t)e << P.page_shift) < len ? __ldg(P.table + trow + e) : -1;
          }
          const int key = t * kCT + ((lane & 3) << box_shift);
          const int pg = __shfl_sync(0xffffffffu, page, (key >> P.page_shift) & 31);
          const int32_t row = pg >= 0 && pg < P.pages
                                  ? (int32_t)((((int64_t)pg * P.kv_heads + g.h) << P.page_shift) + (key & ((1 << P.page_shift) - 1)))
                                  : no_row;
          if (!wait_warp(&empty_bar[slot], ph)) {
            ok = false;
            break;
          }
          uint8_t* dst = ring + slot * C::kRawBytes;
          uint64_t* full = &full_bar[slot];
          if constexpr (k8) {   // a box's codes, row after row, and its powers
            const bool mine = lane < boxes, there = mine && row != no_row;
            uint8_t* to = powers[keys ? 0 : 1][slot] + (lane << box_shift);
            const uint32_t n = (uint32_t)__popc(__ballot_sync(0xffffffffu, there));
            if (mine && !there) {   // the codes arrive as zeros
              for (int i = 0; i < box; i += 16) *reinterpret_cast<uint4*>(to + i) = make_uint4(0u, 0u, 0u, 0u);
              asm volatile("fence.proxy.async.shared::cta;" ::: "memory");   // copies follow into the same place
            }
            __syncwarp();
            if (lane == 0) mbar_arrive_expect_tx(full, (uint32_t)(boxes * box * D) + n * (uint32_t)box);
            __syncwarp();
            if (mine) tma_load_2d(dst + lane * (box * D), keys ? &P.kmap : &P.vmap, full, 0, row);
            if (there) bulk_load(to, (keys ? P.k_scales : P.v_scales) + row, (uint32_t)box, full);
            __syncwarp();
            if (++slot == kRawRing) {
              slot = 0;
              ph ^= 1u;
            }
            continue;
          }
          if (elect_one()) mbar_arrive_expect_tx(full, (uint32_t)(boxes * box * D * 2));
          __syncwarp();
          // Keys: slabs of 64 channels x 64 keys.  Values: box after box, each with its slabs.
#pragma unroll 1
          for (int b = 0; b < boxes; ++b) {
            const int32_t r = __shfl_sync(0xffffffffu, row, b);
            if (elect_one()) {
              if (!keys) {
                tma_load_3d(dst + b * (box * D * 2), &P.vmap, full, 0, r, 0);
              } else if (box == kCT) {
                tma_load_3d(dst, &P.kmap, full, 0, r, 0);
              } else {
#pragma unroll
                for (int sl = 0; sl < C::kSlabs; ++sl) tma_load_3d(dst + sl * (kCT * 128) + b * (box * 128), &P.kmap, full, 0, r, sl);
              }
            }
            __syncwarp();
          }
          if (++slot == kRing) {
            slot = 0;
            ph ^= 1u;
          }
        }
      }
    } else if (warp < 6) {
      // ---------------------------------------------------------- MMA issuers: S of half 0, 1, P V of half 0, 1
      const int role = uniform(warp) - 2, h = role & 1;
      const uint32_t one = elect_one() ? 1u : 0u;
      const uint32_t t_s = tmem + h * 128, t_p = t_s + kCT, t_o = tmem + 256 + h * 128;
      // Units are counted over all segments (n); P of unit n is in buffer n & 1.
      uint32_t n = 0, slot = 0, ph = 0u;
      bool ok = true;
      const auto next_slot = [&]() {
        if (++slot == kRing) {
          slot = 0;
          ph ^= 1u;
        }
      };
      const auto over = [&](uint32_t unit) { return wait_warp(&o_bar[h][unit & 1u], (unit >> 1) & 1u); };
      if (role < 2) {
        const uint32_t idesc = idesc_bf16_f32(kHalf, kCT) | (P.negate ? 1u << 13 : 0u);   // bit 13: minus A
        const uint32_t q_lo = desc_lo(smem_u32(smem + h * C::kQBytes), 16), k_lo = desc_lo(smem_u32(ring_k), 16);
        uint32_t qph = 0u;
        while (ok) {
          if (!wait_warp(&seg_full[sg], sph)) break;
          const Segment g = segs[sg];
          next_seg();
          if (g.r < 0) break;
          const int n_units = uniform(g.tb - g.ta);
          const int units = uniform(h < halves(g) ? max(0, half_end(g, h) - g.ta) : 0);   // this half's
          if (units > 0) {
            ok = wait_warp(&q_bar[h], qph);
            qph ^= 1u;
          }
          for (int u = 0; u < n_units && ok; ++u) {
            ok = wait_warp(k8 ? &clean_bars[0][slot] : &kfull_bar[slot], ph);
            if (u < units) {
              ok = ok && (n == 0u || wait_warp(&sfree_bar[h], (n - 1u) & 1u)) && (n < 2u || over(n - 2u));
              if (!ok) break;
              tc_fence_after();
              const uint32_t b = k_lo + slot * (C::kOpBytes >> 4);
#pragma unroll
              for (int kk = 0; kk < D / 16; ++kk)
                mma_ss(t_s, desc(q_lo + (((kk >> 2) * (kHalf * 128) + (kk & 3) * 32) >> 4)),
                       desc(b + (((kk >> 2) * (kCT * 128) + (kk & 3) * 32) >> 4)), idesc, kk == 0 ? 0u : 1u, one);
              commit_to(&s_bar[h], one);
              commit_to(k8 ? &done_bars[0][slot] : &kempty_bar[slot], one);
              if (u == units - 1) commit_to(&qempty_bar[h], one);
              ++n;
            } else if (lane == 0) {
              mbar_arrive(k8 ? &done_bars[0][slot] : &kempty_bar[slot]);   // this half's part of handing the slot back
            }
            next_slot();
          }
        }
      } else {
        const uint32_t idesc = idesc_bf16_f32(kHalf, D) | (1u << 16);   // bit 16: B is MN-major
        const int lay_shift = k8 ? 6 : box_shift, lay = 1 << lay_shift;   // keys that lie together: converted ones all do
        const uint32_t vblock = (uint32_t)lay * 128u;
        const uint32_t v_lo = desc_lo(smem_u32(ring_v), vblock);
        uint32_t v_off[kCT / 16];   // of 16 keys in a slot
#pragma unroll
        for (int kk = 0; kk < kCT / 16; ++kk)
          v_off[kk] = ((uint32_t)((16 * kk) >> lay_shift) * (vblock * C::kSlabs) + (uint32_t)((16 * kk) & (lay - 1)) * 128u) >> 4;
        while (ok) {
          if (!wait_warp(&seg_full[sg], sph)) break;
          const Segment g = segs[sg];
          next_seg();
          if (g.r < 0) break;
          const int n_units = uniform(g.tb - g.ta);
          const int units = uniform(h < halves(g) ? max(0, half_end(g, h) - g.ta) : 0);
          for (int u = 0; u < n_units && ok; ++u) {
            ok = wait_warp(&clean_bar[slot], ph);
            if (u < units) {
              ok = ok && wait_warp(&p_bar[h][n & 1u], (n >> 1) & 1u);
              if (!ok) break;
              tc_fence_after();
              const uint32_t v = v_lo + slot * (C::kOpBytes >> 4), p = t_p + (n & 1u) * (kCT / 2);
#pragma unroll
              for (int kk = 0; kk < kCT / 16; ++kk) mma_ts(t_o, p + 8 * kk, desc(v + v_off[kk]), idesc, kk > 0 ? 1u : (uint32_t)u, one);
              commit_to(&o_bar[h][n & 1u], one);
              commit_to(k8 ? &done_bars[1][slot] : &vempty_bar[slot], one);
              ++n;
            } else if (lane == 0) {
              mbar_arrive(k8 ? &done_bars[1][slot] : &vempty_bar[slot]);
            }
            next_slot();
          }
        }
      }
      // whatever was issued is over before TMEM goes back
      __syncwarp();
      commit_to(&drain_bar[role], one);
#pragma unroll 1
      for (int left = kWaitTries; left > 0 && !__all_sync(0xffffffffu, mbar_try_wait_sleep(&drain_bar[role], 0u, 1000u)); --left) {
      }
    } else if (k8 && warp < 8) {
      if (P.zero_rest && warp == 6) zero_rows(P, D, cta, lane, false);
    } else if constexpr (k8) {
      // ---------------------------------------------------------- codes to bf16: 16 keys of a unit, or 16 values, a warp
      const int mine = warp & 3;
      const int v = warp >= 20 ? 1 : 0;   // addresses by 32-bit numbers: registers are short
      // A lane 16 codes a step, kStep keys a step; the row of a key has kLanes lanes.  Few and wide accesses: shared memory is
      // busy with the products' operands, and answers late.
      constexpr int kLanes = D / 16, kStep = 32 / kLanes, kSteps = 16 / kStep;
      const int row = lane / kLanes, col = lane % kLanes;
      const bool odd = (col >> 2) & 1;   // these lanes store their second half first, into other banks than the rest
      const uint32_t src0 = smem_u32(v ? raw_v : raw_k) + (uint32_t)((16 * mine + row) * D + 16 * col);
      const uint32_t up = v ? 120u - kDown : 120u;
      const uint32_t dst0 = smem_u32(v ? ring_v : ring_k) + (uint32_t)((16 * mine + row) * 128 + (col >> 2) * (kCT * 128));
      uint32_t raw = 0, rph = 0u, slot = 0, ph = 1u;
      bool ok = true;
      while (ok) {
        if (!wait_warp(&seg_full[sg], sph)) break;
        const Segment g = segs[sg];
        const uint32_t at = sg;
        if (g.r < 0) break;
        const int len = g.s.len(), all_see = g.s.seen(half_tok(g, 0));
        for (int t = g.ta; t < g.tb && ok; ++t) {
          const int key0 = t * kCT + 16 * mine;
          if (!(ok = wait_warp(&full_bars[v][raw], rph))) break;
          uint32_t power[kSteps];
          uint4 codes[kSteps];   // all of them under way before the first is waited for, and before the place for them is free
#pragma unroll
          for (int i = 0; i < kSteps; ++i) {
            codes[i] = load16(src0 + raw * C::kRawBytes + i * (kStep * D));
            power[i] = powers[v][raw][16 * mine + i * kStep + row];
          }
          if (!(ok = wait_warp(&done_bars[v][slot], ph))) break;
          const uint32_t dst = dst0 + slot * C::kOpBytes;
#pragma unroll
          for (int i = 0; i < kSteps; ++i) {
            const int k = i * kStep + row;   // of this warp's 16
            const uint4 c = codes[i];
            const uint32_t code = power[i];
            const uint32_t m = (code == 0u ? 0u : min(code, kHighPower) + up << 7) * 0x10001u;
            const uint32_t x0 = odd ? c.z : c.x, x1 = odd ? c.w : c.y, x2 = odd ? c.x : c.z, x3 = odd ? c.y : c.w;
            const uint32_t q = (2 * (col & 3) + odd) ^ ((16 * mine + k) & 7);
            store16(dst + i * (kStep * 128) + (q << 4), bf16_of<0x1404>(x0, m), bf16_of<0x3424>(x0, m), bf16_of<0x1404>(x1, m), bf16_of<0x3424>(x1, m));
            store16(dst + i * (kStep * 128) + ((q ^ 1u) << 4), bf16_of<0x1404>(x2, m), bf16_of<0x3424>(x2, m), bf16_of<0x1404>(x3, m), bf16_of<0x3424>(x3, m));
          }
          // What that does not do: powers above 2^7 and NaN; and values past the end, or NaN and not seen by some row, become zeros,
          // since a weight of zero would not silence them.
          const uint4 pw = load16(smem_u32(&powers[v][raw][16 * mine]));
          const uint32_t high = __vcmpgtu4(pw.x, 0x86868686u) | __vcmpgtu4(pw.y, 0x86868686u) | __vcmpgtu4(pw.z, 0x86868686u) |
                                __vcmpgtu4(pw.w, 0x86868686u);
          if (__builtin_expect(high || (v && key0 + 16 > len), 0)) {
            __syncwarp();
#pragma unroll 1
            for (int k = 0; k < 16; ++k) {
              const uint32_t code = powers[v][raw][16 * mine + k];
              const bool held = key0 + k < len, cut = v && key0 + k >= all_see && (code == 255u || !held);
              if (cut && held) bad_s[at] = 1;
              if ((!cut && code <= kHighPower) || lane >= D / 8) continue;
              const uint32_t to = smem_u32(v ? ring_v : ring_k) + slot * C::kOpBytes + (lane >> 3) * (kCT * 128) + (16 * mine + k) * 128 + ((lane & 7) << 4);
              const uint32_t m = cut ? 0u : code == 255u ? 0x7FC07FC0u : (code - kHighPower + 127u << 7) * 0x10001u;
              const uint4 x = load16(to);   // finite: zeros times a NaN are NaN too
              store16(to, times(x.x, m), times(x.y, m), times(x.z, m), times(x.w, m));
            }
          }
          asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
          __syncwarp();
          if (lane == 0) {
            mbar_arrive(&empty_bars[v][raw]);
            mbar_arrive(&clean_bars[v][slot]);
          }
          if (++raw == kRawRing) {
            raw = 0;
            rph ^= 1u;
          }
          if (++slot == kRing) {
            slot = 0;
            ph ^= 1u;
          }
        }
        next_seg();
      }
    } else {
      // ---------------------------------------------------------- values that some row does not see
      uint32_t vs = 0, vph = 0u;
      bool ok = true;
      const int mine = warp - 6;
      while (ok) {
        if (!wait_warp(&seg_full[sg], sph)) break;
        const Segment g = segs[sg];
        const uint32_t at = sg;
        if (g.r < 0) break;
        const int len = g.s.len(), all_see = g.s.seen(half_tok(g, 0));
        for (int t = g.ta; t < g.tb; ++t) {
          if (!wait_warp(&vfull_bar[vs], vph)) {
            ok = false;
            break;
          }
          const int key0 = t * kCT;
          if (key0 + kCT > all_see) {
            // 16 keys at a time, of one box (a page has 16 at least): a key's row is kSlabs pieces of 128 bytes, whose swizzle
            // does not matter here.  A lane has 16 bytes of one key in kStep.
            constexpr int kPieces = D / 8, kStep = 32 / kPieces, kDeep = 16 / kStep;
            const int from = max(0, all_see - key0), end = min(kCT, max(0, len - key0)), piece = lane % kPieces;
            bool bad = false;
#pragma unroll 1
            for (int k0 = (from & ~15) + 16 * mine; k0 < kCT; k0 += 16 * C::kCleaners) {
              uint8_t* base = ring_v + vs * C::kOpBytes + (((k0 >> box_shift) * C::kSlabs + (piece >> 3)) << box_shift) * 128 +
                              ((k0 & (box - 1)) + lane / kPieces) * 128 + (piece & 7) * 16;
              uint4 x[kDeep];
              uint32_t any[4] = {0u, 0u, 0u, 0u};   // bf16 pairs: sums of 0 x, NaN where some x is an infinity or NaN
#pragma unroll
              for (int i = 0; i < kDeep; ++i) x[i] = *reinterpret_cast<const uint4*>(base + i * (kStep * 128));
#pragma unroll
              for (int i = 0; i < kDeep; ++i) {
                any[0] = times_zero(x[i].x, any[0]);
                any[1] = times_zero(x[i].y, any[1]);
                any[2] = times_zero(x[i].z, any[2]);
                any[3] = times_zero(x[i].w, any[3]);
              }
              // +-0 sums: an exponent of ones stays one in the "or" of all four
              if (nonfinite2(any[0] | any[1] | any[2] | any[3]) == 0u && k0 + 16 <= end) continue;   // the rule: nothing to do
#pragma unroll 1
              for (int i = 0; i < kDeep; ++i) {
                const int k = k0 + i * kStep + lane / kPieces;
                if (k < from) continue;   // every row sees it
                uint4* at16 = reinterpret_cast<uint4*>(base + i * (kStep * 128));
                uint4 v = k < end ? *at16 : make_uint4(0u, 0u, 0u, 0u);
                const uint32_t n[4] = {nonfinite2(v.x), nonfinite2(v.y), nonfinite2(v.z), nonfinite2(v.w)};
                bad |= (n[0] | n[1] | n[2] | n[3]) != 0u;
                *at16 = make_uint4(v.x & ~n[0], v.y & ~n[1], v.z & ~n[2], v.w & ~n[3]);
              }
            }
            if (bad) bad_s[at] = 1;
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
          }
          __syncwarp();
          if (lane == 0) mbar_arrive(&clean_bar[vs]);
          if (++vs == kRing) {
            vs = 0;
            vph ^= 1u;
          }
        }
        next_seg();
      }
      if (P.zero_rest && mine == 0) zero_rows(P, D, cta, lane, false);
    }
  } else {
    // ------------------------------------------------------------ softmax: a row a thread
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(C::kRegsSoftmax));
    const int h = (warp - 8) >> 2, quarter = warp & 3;
    const uint32_t lane_base = (uint32_t)(32 * quarter) << 16;
    const uint32_t ts = tmem + h * 128 + lane_base, to = tmem + 256 + h * 128 + lane_base;
    uint32_t sg = 0, sph = 0, n = 0, j_ph = 0u;   // n: units so far
    const auto meet = [&]() {   // the warpgroup's barrier, bounded like every wait
      __syncwarp();
      if (lane == 0) mbar_arrive(&join_bar[h]);
      const bool met = wait_warp(&join_bar[h], j_ph);
      j_ph ^= 1u;
      return met;
    };
    const float c = P.scale_log2;
    const uint64_t c2 = pair(__float_as_uint(c), __float_as_uint(c));
    // this half's next segment and its slot; false: no more, or some role gave up
    const auto next_segment = [&](Segment& g, uint32_t& at) {
      while (true) {
        if (!wait_warp(&seg_full[sg], sph)) return false;
        g = segs[sg];
        at = sg;
        if (++sg == kSegs) {
          sg = 0;
          sph ^= 1u;
        }
        if (g.r < 0) return false;
        if (h < halves(g)) return true;
        __syncwarp();
        if (lane == 0) mbar_arrive(&seg_empty[at]);
      }
    };
    // this thread's row of a segment
    struct Row {
      int tok, hd, vis;
      bool on;
    };
    const auto row_of = [&](const Segment& g) {
      const int i = 32 * quarter + lane, t = row_token(P, i);
      Row r;
      r.tok = half_tok(g, h) + t;
      r.hd = i - t * P.group;
      r.on = t < P.half_tokens && r.tok < g.s.n;
      r.vis = r.on ? g.s.seen(r.tok) : 0;
      return r;
    };
    Segment g;
    uint32_t at;
    bool more = next_segment(g, at);
    Row row = {0, 0, 0, false};
    if (more) row = row_of(g);
    while (more) {
      const int end = half_end(g, h);
      const int all_see = g.s.seen(half_tok(g, h));
      float m = -INFINITY, l = 0.f;
      bool ok = true;
      uint32_t s[2][32];
      // S of unit n on its way to registers, and there
      const auto fetch_s = [&]() {
        if (!wait_warp(&s_bar[h], n & 1u)) return false;
        tc_fence_after();
        tmem_ld_x32(ts, s[0]);
        tmem_ld_x32(ts + 32, s[1]);
        return true;
      };
      const auto have_s = [&]() {
        tmem_wait_ld();
        reg_fence(s[0]);
        reg_fence(s[1]);
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&sfree_bar[h]);
      };
      if (g.ta < end) {
        ok = fetch_s();
        if (ok) have_s();
      }
      for (int t = g.ta; t < end && ok; ++t) {
        const int key0 = t * kCT;
        if (key0 + kCT > all_see) {
          const int v = row.vis - key0;
#pragma unroll
          for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int e = 0; e < 32; ++e)
              if (32 * i + e >= v) s[i][e] = 0xFF800000u;   // -inf
        }
        float top[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint32_t* q = &s[i >> 1][16 * (i & 1)];
          top[i] = fmaxf(__uint_as_float(q[0]), __uint_as_float(q[1]));
#pragma unroll
          for (int e = 2; e < 16; e += 2) top[i] = max3(top[i], __uint_as_float(q[e]), __uint_as_float(q[e + 1]));
        }
        const float mt = fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3]));
        float f = 1.f;
        if ((mt - m) * c > 8.f) {   // m = -inf: always, once a key is seen
          f = ex2((m - mt) * c);
          m = mt;
        }
        if (t > g.ta && __any_sync(0xffffffffu, f != 1.f)) {
          if (!wait_warp(&o_bar[h][(n - 1u) & 1u], ((n - 1u) >> 1) & 1u)) {   // the product before is in O
            ok = false;
            break;
          }
          tc_fence_after();
#pragma unroll 1
          for (int i = 0; i < D / 32; ++i) {
            uint32_t o[32];
            tmem_ld_x32(to + 32 * i, o);
            tmem_wait_ld();
            reg_fence(o);
#pragma unroll
            for (int e = 0; e < 32; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * f);
            tmem_st_x32(to + 32 * i, o);
          }
        }
        const float mc = m == -INFINITY ? 0.f : m * c;
        const uint64_t mc2 = pair(__float_as_uint(-mc), __float_as_uint(-mc));
        uint32_t p[32];
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int e = 0; e < 32; e += 2) {
            uint32_t a, b;
            unpair(fma2(pair(s[i][e], s[i][e + 1]), c2, mc2), a, b);
            s[i][e] = __float_as_uint(ex2(__uint_as_float(a)));
            s[i][e + 1] = __float_as_uint(ex2(__uint_as_float(b)));
            p[16 * i + e / 2] = pack_bf16(__uint_as_float(s[i][e]), __uint_as_float(s[i][e + 1]));
          }
        tmem_st_x32(ts + kCT + (n & 1u) * (kCT / 2), p);
        uint64_t sum[4] = {0ull, 0ull, 0ull, 0ull};   // while the store is under way
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int e = 0; e < 16; e += 2) sum[i] = add2(sum[i], pair(s[i >> 1][16 * (i & 1) + e], s[i >> 1][16 * (i & 1) + e + 1]));
        uint32_t s0, s1;
        unpair(add2(add2(sum[0], sum[1]), add2(sum[2], sum[3])), s0, s1);
        l = l * f + (__uint_as_float(s0) + __uint_as_float(s1));
        const uint32_t buf = n++ & 1u;
        if (t + 1 < end) ok = fetch_s();   // the next one, beside the store
        tmem_wait_st();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&p_bar[h][buf]);
        if (t + 1 < end && ok) have_s();
      }
      if (!ok) break;
      // ---- this segment's result, 32 channels at a time: to the output, or (phase 0) to the item's parts in the workspace,
      // which the warpgroups that arrive last join in their order (phases 1 and 2, join_step's levels).
      // Parts: [D / 4][256 rows][4], then [256][2].
      if (g.ta < end) {
        if (!wait_warp(&o_bar[h][(n - 1u) & 1u], ((n - 1u) >> 1) & 1u)) break;
        tc_fence_after();
      }
      // the row in the output (its elements fit memory, so rows fit 32 bits)
      const uint32_t mine = row.on ? (uint32_t)(g.s.tok0 + row.tok) * (uint32_t)P.q_heads + (uint32_t)(g.h * P.group + row.hd) : ~0u;
      const int ri = h * kHalf + 32 * quarter + lane;
      // Rows that exist, in whole 128-byte lines: a sector that is written in part costs whoever reads it a fill from HBM
      // (9 tokens of 28/4 heads at 30000 keys 50 us, 43 so).
      const bool some = __shfl_sync(0xffffffffu, row.on, lane & ~7);
      const int ri_read = some ? ri : ri - lane;
      JoinStep j = {g.part, 1, 1, g.parts == 1};
      float mm = m, sum = l;
#pragma unroll 1
      for (int phase = 0; phase < 3; ++phase) {
        if (phase > 0) {
          j = join_step(g, phase - 1, kFlat);
          if (j.n == 1) continue;   // a group of its own: the next level
          __threadfence();
          if (!(ok = meet())) break;
          if (quarter == 0 && lane == 0) {
            int32_t* cnt = P.cnt + 2 * ((phase - 1) * (int)gridDim.x + g.first_cta + j.first) + h;
            last_s[h] = atomicAdd(cnt, 1) == j.n - 1;
            if (last_s[h]) *cnt = 0;
            __threadfence();
          }
          if (!(ok = meet())) break;
          if (!last_s[h]) break;
          mm = -INFINITY;
#pragma unroll 1
          for (int p0 = 0; p0 < j.n; p0 += 4) {
            float2 ml[4];
#pragma unroll
            for (int i = 0; i < 4; ++i)
              ml[i] = load_ml(part_slot(P, g.first_cta, j.first + min(p0 + i, j.n - 1) * j.stride, kPartRows * (D + kPartPad)) + D * kPartRows + 2 * ri_read);
            mm = fmaxf(max3(mm, ml[0].x, ml[1].x), fmaxf(ml[2].x, ml[3].x));
          }
        }
        float* slot = j.last ? nullptr : part_slot(P, g.first_cta, j.first, kPartRows * (D + kPartPad));
#pragma unroll 1
        for (int c0 = 0; c0 < D; c0 += 32) {
          float o[32];
#pragma unroll
          for (int e = 0; e < 32; ++e) o[e] = 0.f;
          if (phase == 0) {
            if (g.ta < end) {
              uint32_t v[32];
              tmem_ld_x32(to + c0, v);
              tmem_wait_ld();
              reg_fence(v);
#pragma unroll
              for (int e = 0; e < 32; ++e) o[e] = __uint_as_float(v[e]);
            }
          } else {
            // kJoin parts' pieces under way at once, at clamped addresses
            constexpr int kJoin = C::kJoin;
            sum = 0.f;
            const float base = mm == -INFINITY ? 0.f : mm;
            if (!__any_sync(0xffffffffu, some)) break;
#pragma unroll 1
            for (int p0 = 0; p0 < j.n; p0 += kJoin) {
              float2 ml[kJoin];
              float4 v[kJoin][8];
#pragma unroll
              for (int i = 0; i < kJoin; ++i) {
                const float* sp = part_slot(P, g.first_cta, j.first + min(p0 + i, j.n - 1) * j.stride, kPartRows * (D + kPartPad));
                ml[i] = load_ml(sp + D * kPartRows + 2 * ri_read);
#pragma unroll
                for (int e = 0; e < 8; ++e) v[i][e] = load_part(sp + (size_t)((c0 + 4 * e) * kPartRows + 4 * ri_read));
              }
#pragma unroll
              for (int i = 0; i < kJoin; ++i) {
                if (p0 + i >= j.n) break;
                const float fp = ml[i].x == mm ? 1.f : ex2((ml[i].x - base) * c);
                sum = fmaf(ml[i].y, fp, sum);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                  o[4 * e] = fmaf(v[i][e].x, fp, o[4 * e]);
                  o[4 * e + 1] = fmaf(v[i][e].y, fp, o[4 * e + 1]);
                  o[4 * e + 2] = fmaf(v[i][e].z, fp, o[4 * e + 2]);
                  o[4 * e + 3] = fmaf(v[i][e].w, fp, o[4 * e + 3]);
                }
              }
            }
          }
          if (slot) {
            if (!some) continue;
#pragma unroll
            for (int e = 0; e < 32; e += 4)
              *reinterpret_cast<float4*>(slot + (size_t)((c0 + e) * kPartRows + 4 * ri)) = make_float4(o[e], o[e + 1], o[e + 2], o[e + 3]);
            continue;
          }
          // A lane has a whole row: 64 bytes of it, in two sectors.
          if (row.on) {
            const float inv = row.vis > 0 ? reciprocal(sum) * (k8 ? (float)(1u << kDown) : 1.f) : 0.f;
            uint32_t w[16];
#pragma unroll
            for (int e = 0; e < 16; ++e) w[e] = pack_bf16(o[2 * e] * inv, o[2 * e + 1] * inv);
            store_sectors(P.out + (int64_t)mine * D + c0, w);
          }
        }
        if (phase == 0 && bad_s[at]) {
          // infinities and NaN of keys that only some rows see: added to what has just been written
          __syncwarp();
          const int stop = min(g.tb * kCT, row.vis);
#pragma unroll 1
          for (int key = max(g.s.seen(half_tok(g, 0)), g.ta * kCT); key < stop; ++key) {
            const int pg = __ldg(P.table + (int64_t)g.r * P.width + (key >> P.page_shift));
            if (pg < 0 || pg >= P.pages) continue;
            const int64_t in_pages = (((int64_t)pg * P.kv_heads + g.h) << P.page_shift) + (key & ((1 << P.page_shift) - 1));
            if (k8 && __ldg(P.v_scales + in_pages) != 255) continue;   // in 8 bits all of it, or nothing
            const uint16_t* vr = P.v + in_pages * D;
#pragma unroll 1
            for (int e = 0; e < D; ++e) {
              const float x = k8 ? __uint_as_float(0x7FC00000u) : bf16_lo(__ldg(vr + e));
              if (isfinite(x)) continue;
              if (slot) {
                slot[(size_t)((e & ~3) * kPartRows + 4 * ri + (e & 3))] += x;
              } else {
                volatile uint16_t* to16 = P.out + (int64_t)mine * D + e;
                *to16 = (uint16_t)pack_bf16(bf16_lo(*to16) + x, 0.f);
              }
            }
          }
        }
        if (!slot) break;
        *reinterpret_cast<float2*>(slot + (size_t)(D * kPartRows + 2 * ri)) = make_float2(mm, sum);
      }
      if (!ok) break;
      __syncwarp();
      if (lane == 0) mbar_arrive(&seg_empty[at]);
      tc_fence_before();   // O may be overwritten once the next P is announced
      more = next_segment(g, at);
      if (more) row = row_of(g);
    }
  }
  tc_fence_before();
  __syncthreads();
  end_of_waits(abort_flag, P.err);
  if (warp == 2) {
    tc_fence_after();
    tmem_dealloc(tmem, 512);
  }
}

template <int D, bool k8>
gs_status chunk_launch(const AttnParams& P, int ctas, cudaStream_t s) {
  using C = ChunkCfg<D, k8>;
  static const cudaError_t attr = cudaFuncSetAttribute(k_attn_chunk<D, k8>, cudaFuncAttributeMaxDynamicSharedMemorySize, C::kSmem);
  if (attr != cudaSuccess) return GS_ERR_CUDA;
  return launch_behind(k_attn_chunk<D, k8>, dim3((unsigned)ctas), C::kThreads, C::kSmem, s, P);
}

}  // namespace

int attn_chunk_box(int page_size) { return page_size < kCT ? page_size : kCT; }

int attn_chunk_tile() { return kCT; }

int attn_chunk_rows() { return kHalf; }   // two halves, each of more than half its lanes

int attn_most_over() { return ChunkTraits::kOver; }

int attn_chunk_part(int head_dim) { return kPartRows * (head_dim + kPartPad); }

int attn_chunk_half_tokens(int group) { return kHalf / group; }

gs_status launch_attn_chunk(const AttnParams& P, int head_dim, int ctas, cudaStream_t s) {
  if (P.k_scales) return head_dim == 128 ? chunk_launch<128, true>(P, ctas, s) : chunk_launch<64, true>(P, ctas, s);
  return head_dim == 128 ? chunk_launch<128, false>(P, ctas, s) : chunk_launch<64, false>(P, ctas, s);
}

}  // namespace gs
