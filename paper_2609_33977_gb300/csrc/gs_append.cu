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
#include "gs_block.cuh"

namespace gs {
namespace {

constexpr int kAppThreads = 128;   // at most

struct AppendParams {
  const uint16_t* q;
  const uint16_t* k;
  const uint16_t* v;
  uint16_t* q_out;
  uint16_t* k_pages;
  uint16_t* v_pages;
  const float* cos_t;
  const float* sin_t;
  const int32_t* offsets;
  const int32_t* kv_lens;
  const int32_t* table;
  int64_t q_stride, k_stride, v_stride, n_pos, pages;
  int32_t n_seqs, width, page_shift, q_heads, kv_heads, head_dim, parts;
};

__global__ void __launch_bounds__(kAppThreads) k_cache_append(const AppendParams P) {
  start_of_work();
  const int64_t t = blockIdx.x / (unsigned)P.parts;
  const int per = P.head_dim / 16;   // threads of a head
  const int item = (int)(blockIdx.x % (unsigned)P.parts) * (int)blockDim.x + (int)threadIdx.x;
  int head = item / per;
  const int i = item % per;
  const bool on = head < P.q_heads + 2 * P.kv_heads;
  const int kind = head < P.q_heads ? 0 : head < P.q_heads + P.kv_heads ? 1 : 2;   // q, k, v
  head -= kind == 0 ? 0 : kind == 1 ? P.q_heads : P.q_heads + P.kv_heads;
  const int64_t D = P.head_dim;
  // before the look-up: neither needs the other.  Threads past the last head read the first one's.
  const uint16_t* src = (kind == 0 ? P.q + t * P.q_stride : kind == 1 ? P.k + t * P.k_stride : P.v + t * P.v_stride) +
                        (on ? head * D : 0);
  uint4 a = __ldcs(reinterpret_cast<const uint4*>(src) + i), b = __ldcs(reinterpret_cast<const uint4*>(src + D / 2) + i);
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
  if (!on) return;
  const bool turn = pos >= 0 && pos < P.n_pos;
  int64_t page = -1;
  if (turn && kind != 0 && (pos >> P.page_shift) < P.width) page = __ldg(P.table + (int64_t)seq * P.width + (pos >> P.page_shift));
  if (turn && kind != 2) {
    uint32_t ax[4] = {a.x, a.y, a.z, a.w}, bx[4] = {b.x, b.y, b.z, b.w};
    const float4* cp = reinterpret_cast<const float4*>(P.cos_t + pos * (D / 2) + 8 * i);
    const float4* sp = reinterpret_cast<const float4*>(P.sin_t + pos * (D / 2) + 8 * i);
    const float4 c0 = __ldg(cp), c1 = __ldg(cp + 1), s0 = __ldg(sp), s1 = __ldg(sp + 1);
    const float c[8] = {c0.x, c0.y, c0.z, c0.w, c1.x, c1.y, c1.z, c1.w};
    const float n[8] = {s0.x, s0.y, s0.z, s0.w, s1.x, s1.y, s1.z, s1.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float al = bf16_lo(ax[e]), ah = bf16_hi(ax[e]), bl = bf16_lo(bx[e]), bh = bf16_hi(bx[e]);
      ax[e] = pack_bf16(al * c[2 * e] - bl * n[2 * e], ah * c[2 * e + 1] - bh * n[2 * e + 1]);
      bx[e] = pack_bf16(bl * c[2 * e] + al * n[2 * e], bh * c[2 * e + 1] + ah * n[2 * e + 1]);
    }
    a = make_uint4(ax[0], ax[1], ax[2], ax[3]);
    b = make_uint4(bx[0], bx[1], bx[2], bx[3]);
  }
  uint16_t* dst;
  if (kind == 0) {
    dst = P.q_out + (t * P.q_heads + head) * D;
  } else {
    if (page < 0 || page >= P.pages) return;   // no place for this token
    const int64_t slot = pos & ((1 << P.page_shift) - 1);
    dst = (kind == 1 ? P.k_pages : P.v_pages) + (((page * P.kv_heads + head) << P.page_shift) + slot) * D;
  }
  reinterpret_cast<uint4*>(dst)[i] = a;
  reinterpret_cast<uint4*>(dst + D / 2)[i] = b;
}

}  // namespace

gs_status launch_cache_append(const gs_paged_cache& c, const gs_seq_batch& b, const void* q, int64_t q_stride, int32_t q_heads,
                              const void* k, int64_t k_stride, const void* v, int64_t v_stride, const float* cos_t,
                              const float* sin_t, int64_t n_pos, void* q_out, cudaStream_t s) {
  AppendParams P;
  P.q = static_cast<const uint16_t*>(q);
  P.k = static_cast<const uint16_t*>(k);
  P.v = static_cast<const uint16_t*>(v);
  P.q_out = static_cast<uint16_t*>(q_out);
  P.k_pages = static_cast<uint16_t*>(c.k_dev);
  P.v_pages = static_cast<uint16_t*>(c.v_dev);
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
  P.parts = (items + kAppThreads - 1) / kAppThreads;
  const unsigned threads = (unsigned)((items + P.parts - 1) / P.parts + 31) / 32 * 32;
  const int64_t blocks = b.tokens * P.parts;
  if (blocks > INT32_MAX) return GS_ERR_UNSUPPORTED;
  return launch_behind(k_cache_append, dim3((unsigned)blocks), threads, 0, s, P);
}

}  // namespace gs
