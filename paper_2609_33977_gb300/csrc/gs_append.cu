// A chunk's queries and keys turned by their positions' angles, and its keys and
// values written into the pages of the cache:
//     (a, b) -> (a c - b s, b c + a s)   for channels a = x[i], b = x[i + D/2],
// c and s the angle table's rows of the token's position.
//
// Bound by HBM at long chunks (every element of q, k, v read and written once),
// by latency at few tokens: the look-up of a token's sequence, its length, its page
// are loads that wait for one another.  A block takes a part of one token's heads, a
// thread 8 channel pairs of a head: two 16-byte loads and stores.  (Blocks of 512
// threads 2.6 us, of 128 2.4, for 16 tokens of 32 + 2 x 32 heads.  Two or four tokens a
// block: 7 and 40 % slower at 3000 tokens, since a thread's loads then queue behind each
// other's look-ups.)  Up to 32 sequences are looked up by every warp for itself, one load
// each and a ballot; more by the whole block (us at these 16 tokens and at 3000 of
// 28 + 2 x 4 heads: 2.5 and 11.3 by a warp, 2.7 and 11.5 by the block).
//
// 3000 tokens of 28 + 2 x 4 heads of 128: 11 us, 5.2 TB/s; 16 tokens of 32 + 2 x 32: 1.8 us.
//
// Into 8 bits (k8): a head's threads agree on the largest magnitude, as float bits, whose
// exponent (one more past 1.75, the fraction of 448) gives the power of two; it takes the place
// of the bf16 rounding, so that keys are rounded once.  The same tokens 11.5 and 2.0 us, and 4096 of 40 + 2 x 40 heads 44.8 (4.7
// TB/s; with one head a thread 49.9, but the 3000 of 28 + 2 x 4 would take 13.7 with two, a quarter of the threads idle).
#include "gs_block.cuh"

namespace gs {
namespace {

constexpr int kAppThreads = 128;   // at most
constexpr int kTwoTokens = 256;    // from so many tokens on, two heads a thread, where that leaves an eighth of the threads idle at most

struct AppendParams {
  const uint16_t* q;
  const uint16_t* k;
  const uint16_t* v;
  uint16_t* q_out;
  uint16_t* k_pages;
  uint16_t* v_pages;
  uint8_t* k_scales;   // 8 bits only; the pages are codes then
  uint8_t* v_scales;
  const float* cos_t;
  const float* sin_t;
  const int32_t* offsets;
  const int32_t* kv_lens;
  const int32_t* table;
  int64_t q_stride, k_stride, v_stride, n_pos, pages;
  int32_t n_seqs, width, page_shift, q_heads, kv_heads, head_dim, parts;
};

// e4m3 codes of four float32, the first in the lowest byte
__device__ __forceinline__ uint32_t pack_e4m3(float a, float b, float c, float d) {
  uint16_t lo, hi;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(lo) : "f"(b), "f"(a));
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(hi) : "f"(d), "f"(c));
  return (uint32_t)lo | ((uint32_t)hi << 16);
}

// H: heads of a thread, as far apart as all blocks of a token have threads
template <bool k8, int H>
__global__ void __launch_bounds__(kAppThreads) k_cache_append(const AppendParams P) {
  start_of_work();
  const int64_t t = blockIdx.x / (unsigned)P.parts;
  const int per = P.head_dim / 16;   // threads of a head
  const int first_item = (int)(blockIdx.x % (unsigned)P.parts) * (int)blockDim.x + (int)threadIdx.x;
  const int64_t D = P.head_dim;
  int head[H], kind[H];   // kinds: q, k, v
  bool on[H];
  uint4 a[H], b[H];
  const int i = first_item % per;
#pragma unroll
  for (int h = 0; h < H; ++h) {
    head[h] = (first_item + h * P.parts * (int)blockDim.x) / per;
    on[h] = head[h] < P.q_heads + 2 * P.kv_heads;
    kind[h] = head[h] < P.q_heads ? 0 : head[h] < P.q_heads + P.kv_heads ? 1 : 2;
    head[h] -= kind[h] == 0 ? 0 : kind[h] == 1 ? P.q_heads : P.q_heads + P.kv_heads;
    // before the look-up: neither needs the other.  Threads past the last head read the first one's.
    const uint16_t* src = (kind[h] == 0 ? P.q + t * P.q_stride : kind[h] == 1 ? P.k + t * P.k_stride : P.v + t * P.v_stride) +
                          (on[h] ? head[h] * D : 0);
    a[h] = __ldcs(reinterpret_cast<const uint4*>(src) + i);
    b[h] = __ldcs(reinterpret_cast<const uint4*>(src + D / 2) + i);
  }
  int seq;
  int64_t pos = -1;
  if (P.n_seqs <= 32) {
    const int s = min((int)(threadIdx.x & 31), P.n_seqs - 1);
    const int first = __ldg(P.offsets + s), end = __ldg(P.offsets + s + 1), kv = __ldg(P.kv_lens + s);
    seq = __popc(__ballot_sync(0xffffffffu, (int)(threadIdx.x & 31) < P.n_seqs && end <= t));
    const int64_t mine = t >= first ? (int64_t)kv - ((int64_t)end - first) + (t - first) : -1;
    const int64_t got = __shfl_sync(0xffffffffu, mine, seq & 31);
    if (seq < P.n_seqs) pos = got;
  } else {
    seq = block_count_le(P.offsets, P.n_seqs, (int)t);
    if (seq < P.n_seqs) {
      const int64_t first = __ldg(P.offsets + seq), end = __ldg(P.offsets + seq + 1);
      if (t >= first) pos = (int64_t)__ldg(P.kv_lens + seq) - (end - first) + (t - first);
    }
  }
  if (!k8 && H == 1 && !on[0]) return;   // in 8 bits a warp's threads meet below
  const bool turn = pos >= 0 && pos < P.n_pos;
  int64_t page = -1;
  // one head a thread: loads that its kind needs; two: all of them, without a branch before the next one's
  if (turn && (H > 1 || kind[0] != 0) && (pos >> P.page_shift) < P.width)
    page = __ldg(P.table + (int64_t)seq * P.width + (pos >> P.page_shift));
  float c[8], n[8];
  const auto load_angles = [&]() {
    const float4* cp = reinterpret_cast<const float4*>(P.cos_t + pos * (D / 2) + 8 * i);
    const float4* sp = reinterpret_cast<const float4*>(P.sin_t + pos * (D / 2) + 8 * i);
    const float4 c0 = __ldg(cp), c1 = __ldg(cp + 1), s0 = __ldg(sp), s1 = __ldg(sp + 1);
    c[0] = c0.x, c[1] = c0.y, c[2] = c0.z, c[3] = c0.w, c[4] = c1.x, c[5] = c1.y, c[6] = c1.z, c[7] = c1.w;
    n[0] = s0.x, n[1] = s0.y, n[2] = s0.z, n[3] = s0.w, n[4] = s1.x, n[5] = s1.y, n[6] = s1.z, n[7] = s1.w;
  };
  if constexpr (!k8) {
    // One head a thread: the angles are loaded where they are used.  (In one path with 8 bits, which
    // converts what it does not turn too: 44 registers instead of 40; 3000 tokens of 28 + 2 x 4 heads, out of L2, 9.1 us, not 8.4.)
    if (H > 1 && turn) load_angles();
#pragma unroll
    for (int h = 0; h < H; ++h) {
      uint32_t aw[4] = {a[h].x, a[h].y, a[h].z, a[h].w}, bw[4] = {b[h].x, b[h].y, b[h].z, b[h].w};
      if (turn && kind[h] != 2) {
        if (H == 1) load_angles();
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float al = bf16_lo(aw[e]), ah = bf16_hi(aw[e]), bl = bf16_lo(bw[e]), bh = bf16_hi(bw[e]);
          aw[e] = pack_bf16(al * c[2 * e] - bl * n[2 * e], ah * c[2 * e + 1] - bh * n[2 * e + 1]);
          bw[e] = pack_bf16(bl * c[2 * e] + al * n[2 * e], bh * c[2 * e + 1] + ah * n[2 * e + 1]);
        }
      }
      if (!on[h]) continue;
      uint16_t* dst;
      if (kind[h] == 0) {
        dst = P.q_out + (t * P.q_heads + head[h]) * D;
      } else {
        if (page < 0 || page >= P.pages) continue;   // no place for this token
        const int64_t slot = pos & ((1 << P.page_shift) - 1);
        dst = (kind[h] == 1 ? P.k_pages : P.v_pages) + (((page * P.kv_heads + head[h]) << P.page_shift) + slot) * D;
      }
      reinterpret_cast<uint4*>(dst)[i] = make_uint4(aw[0], aw[1], aw[2], aw[3]);
      reinterpret_cast<uint4*>(dst + D / 2)[i] = make_uint4(bw[0], bw[1], bw[2], bw[3]);
    }
    return;
  }
  if (turn && (H > 1 || kind[0] != 2)) load_angles();
#pragma unroll
  for (int h = 0; h < H; ++h) {
    uint32_t aw[4] = {a[h].x, a[h].y, a[h].z, a[h].w}, bw[4] = {b[h].x, b[h].y, b[h].z, b[h].w};
    float ak[8], bk[8];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float al = bf16_lo(aw[e]), ah = bf16_hi(aw[e]), bl = bf16_lo(bw[e]), bh = bf16_hi(bw[e]);
      ak[2 * e] = al, ak[2 * e + 1] = ah, bk[2 * e] = bl, bk[2 * e + 1] = bh;
      if (turn && kind[h] != 2) {
        ak[2 * e] = al * c[2 * e] - bl * n[2 * e], ak[2 * e + 1] = ah * c[2 * e + 1] - bh * n[2 * e + 1];
        bk[2 * e] = bl * c[2 * e] + al * n[2 * e], bk[2 * e + 1] = bh * c[2 * e + 1] + ah * n[2 * e + 1];
        aw[e] = pack_bf16(ak[2 * e], ak[2 * e + 1]);
        bw[e] = pack_bf16(bk[2 * e], bk[2 * e + 1]);
      }
    }
    const bool placed = page >= 0 && page < P.pages;
    const int64_t slot = pos & ((1 << P.page_shift) - 1);
    const int64_t row = placed ? ((page * P.kv_heads + head[h]) << P.page_shift) + slot : 0;
    uint32_t top = 0;   // bits of magnitudes: ordered like them, NaN above all
    if (H > 1 || kind[h] != 0) {
#pragma unroll
      for (int e = 0; e < 8; ++e) top = max(top, max(__float_as_uint(ak[e]) & 0x7FFFFFFFu, __float_as_uint(bk[e]) & 0x7FFFFFFFu));
    }
    for (int d = per / 2; d > 0; d >>= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, d));   // a head's threads need each other
    if (on[h] && kind[h] != 0 && placed) {
      const bool finite = top < 0x7F800000u;
      const int code = finite ? min(max((int)(top >> 23) - 8 + ((top & 0x7FFFFFu) > 0x600000u ? 1 : 0), 27), 246) : 255;
      const float inv = finite ? __uint_as_float((uint32_t)(254 - code) << 23) : 0.f;
      uint8_t* dst = reinterpret_cast<uint8_t*>(kind[h] == 1 ? P.k_pages : P.v_pages) + row * D + 8 * i;
#pragma unroll
      for (int e = 0; e < 8; ++e) ak[e] = finite ? ak[e] * inv : 0.f, bk[e] = finite ? bk[e] * inv : 0.f;
      *reinterpret_cast<uint2*>(dst) = make_uint2(pack_e4m3(ak[0], ak[1], ak[2], ak[3]), pack_e4m3(ak[4], ak[5], ak[6], ak[7]));
      *reinterpret_cast<uint2*>(dst + D / 2) = make_uint2(pack_e4m3(bk[0], bk[1], bk[2], bk[3]), pack_e4m3(bk[4], bk[5], bk[6], bk[7]));
      if (i == 0) (kind[h] == 1 ? P.k_scales : P.v_scales)[row] = (uint8_t)code;
    }
    if (!on[h] || kind[h] != 0) continue;
    uint16_t* dst = P.q_out + (t * P.q_heads + head[h]) * D;
    reinterpret_cast<uint4*>(dst)[i] = make_uint4(aw[0], aw[1], aw[2], aw[3]);
    reinterpret_cast<uint4*>(dst + D / 2)[i] = make_uint4(bw[0], bw[1], bw[2], bw[3]);
  }
}

}  // namespace

gs_status launch_cache_append(const gs_paged_cache& c, const CacheScales& sc, const gs_seq_batch& b, const void* q, int64_t q_stride, int32_t q_heads,
                              const void* k, int64_t k_stride, const void* v, int64_t v_stride, const float* cos_t,
                              const float* sin_t, int64_t n_pos, void* q_out, cudaStream_t s) {
  AppendParams P;
  P.q = static_cast<const uint16_t*>(q);
  P.k = static_cast<const uint16_t*>(k);
  P.v = static_cast<const uint16_t*>(v);
  P.q_out = static_cast<uint16_t*>(q_out);
  P.k_pages = static_cast<uint16_t*>(c.k_dev);
  P.v_pages = static_cast<uint16_t*>(c.v_dev);
  P.k_scales = sc.k;
  P.v_scales = sc.v;
  P.cos_t = cos_t;
  P.sin_t = sin_t;
  P.offsets = b.offsets_dev;
  P.kv_lens = b.kv_lens_dev;
  P.table = b.table_dev;
  P.q_stride = q_stride;
  P.k_stride = k_stride;
  P.v_stride = v_stride;
  P.n_pos = n_pos;
  P.pages = c.pages;
  P.n_seqs = b.n;
  P.width = b.table_width;
  P.page_shift = __builtin_ctz((unsigned)c.page_size);
  P.q_heads = q_heads;
  P.kv_heads = c.kv_heads;
  P.head_dim = c.head_dim;
  const int items = (q_heads + 2 * c.kv_heads) * (c.head_dim / 16);
  // Blocks of a token, as even as whole warps allow
  const auto threads_of = [&](int heads) {
    const int parts = (items + heads * kAppThreads - 1) / (heads * kAppThreads);
    return (unsigned)((items + heads * parts - 1) / (heads * parts) + 31) / 32 * 32;
  };
  const auto parts_of = [&](int heads) { return (items + heads * kAppThreads - 1) / (heads * kAppThreads); };
  const bool two = b.tokens >= kTwoTokens && (int64_t)threads_of(2) * 2 * parts_of(2) * 8 <= (int64_t)items * 9;
  const unsigned threads = threads_of(two ? 2 : 1);
  P.parts = parts_of(two ? 2 : 1);
  const int64_t blocks = b.tokens * P.parts;
  if (blocks > INT32_MAX) return GS_ERR_UNSUPPORTED;
  const auto kernel = sc.k ? (two ? k_cache_append<true, 2> : k_cache_append<true, 1>) : (two ? k_cache_append<false, 2> : k_cache_append<false, 1>);
  return launch_behind(kernel, dim3((unsigned)blocks), threads, 0, s, P);
}

}  // namespace gs
