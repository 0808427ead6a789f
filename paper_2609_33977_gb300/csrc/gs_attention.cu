// Causal attention of a step's new tokens over a paged cache.
//
// One warp per (token, query head): 32 keys at a time, one per lane for the scores
// (a lane reads its key's whole row), then each lane owns head_dim / 32 channels of
// the output.  Running maximum and sum in float32.
#include "gs_attn.cuh"

#include <cmath>

namespace gs {
namespace {

template <int D>
__global__ void __launch_bounds__(128) k_attention_simple(const AttnParams P) {
  __shared__ float qs[4][D];
  const int64_t t = blockIdx.x;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int head = (int)blockIdx.y * 4 + warp;
  const int seq = block_count_le(P.offsets, P.n_seqs, (int)t);
  if (head >= P.q_heads || seq >= P.n_seqs || seq_info(P, seq).rows < P.min_rows) return;
  int64_t seen = 0;
  if (seq < P.n_seqs) {
    const int64_t first = P.offsets[seq], end = P.offsets[seq + 1];
    if (t >= first) seen = (int64_t)P.kv_lens[seq] - (end - first) + (t - first) + 1;
    seen = min(seen, (int64_t)P.width << P.page_shift);
  }
  constexpr int C = D / 32;
  for (int i = lane; i < D; i += 32) qs[warp][i] = bf16_lo(P.q[t * P.q_stride + head * D + i]);
  __syncwarp();
  const int kvh = head / (P.q_heads / P.kv_heads);
  float m = -INFINITY, l = 0.f, o[C];
#pragma unroll
  for (int c = 0; c < C; ++c) o[c] = 0.f;
  const auto row = [&](int64_t j) -> int64_t {   // -1: no such page
    const int64_t page = P.table[(int64_t)seq * P.width + (j >> P.page_shift)];
    if (page < 0 || page >= P.pages) return -1;
    return ((page * P.kv_heads + kvh) << P.page_shift) + (j & ((1 << P.page_shift) - 1));
  };
  for (int64_t j0 = 0; j0 < seen; j0 += 32) {
    const int64_t j = j0 + lane;
    float s = -INFINITY;
    int64_t at = -1;
    if (j < seen) {
      at = row(j);
      s = 0.f;
      if (at >= 0)
        for (int i = 0; i < D; ++i) s = fmaf(qs[warp][i], bf16_lo(P.k[at * D + i]), s);
      s *= P.negate ? -P.scale_log2 : P.scale_log2;
    }
    float top = s;
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
    const float mn = fmaxf(m, top), base = mn == -INFINITY ? 0.f : mn;
    const float p = j < seen ? ex2(s - base) : 0.f;
    const float f = m == -INFINITY ? 0.f : ex2(m - base);
    float sum = p;
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
    l = l * f + sum;
    m = mn;
#pragma unroll
    for (int c = 0; c < C; ++c) o[c] *= f;
    const int n = (int)min((int64_t)32, seen - j0);
    for (int i = 0; i < n; ++i) {
      const float w = __shfl_sync(0xffffffffu, p, i);
      const int64_t a = __shfl_sync(0xffffffffu, at, i);
      if (a >= 0)
#pragma unroll
        for (int c = 0; c < C; ++c) o[c] = fmaf(w, bf16_lo(P.v[a * D + lane + 32 * c]), o[c]);
    }
  }
  const float inv = seen > 0 ? 1.f / l : 0.f;
#pragma unroll
  for (int c = 0; c < C; ++c) P.out[(t * P.q_heads + head) * D + lane + 32 * c] = (uint16_t)pack_bf16(o[c] * inv, 0.f);
}

}  // namespace

// counters, then the parts of split items (16-byte aligned)
constexpr int64_t kCounterBytes = 4096;
static_assert(kCounterBytes >= 4 * 256, "one counter a CTA");

int attention_ctas() { return sm_count() < 256 ? sm_count() : 256; }

size_t attention_workspace_bytes(const gs_paged_cache& c, const gs_seq_batch&, int32_t) {
  return (size_t)kCounterBytes + (size_t)attention_ctas() * 2 * 64 * (size_t)(c.head_dim + 2) * 4;
}

gs_status launch_paged_attention(const gs_paged_cache& c, const gs_seq_batch& b, const void* q, int64_t q_stride,
                                 int32_t q_heads, float scale, void* out, void* ws, cudaStream_t s) {
  AttnParams P;
  P.q = static_cast<const uint16_t*>(q);
  P.k = static_cast<const uint16_t*>(c.k_dev);
  P.v = static_cast<const uint16_t*>(c.v_dev);
  P.out = static_cast<uint16_t*>(out);
  P.offsets = b.offsets_dev;
  P.kv_lens = b.kv_lens_dev;
  P.table = b.table_dev;
  P.cnt = static_cast<int32_t*>(ws);
  P.parts = reinterpret_cast<float*>(static_cast<uint8_t*>(ws) + kCounterBytes);
  P.err = device_error_flag();
  if (!P.err) return GS_ERR_CUDA;
  P.q_stride = q_stride;
  P.tokens = b.tokens;
  P.pages = c.pages;
  P.n_seqs = b.n;
  P.width = b.table_width;
  P.page_shift = __builtin_ctz((unsigned)c.page_size);
  P.q_heads = q_heads;
  P.kv_heads = c.kv_heads;
  P.group = q_heads / c.kv_heads;
  P.scale_log2 = std::fabs(scale) * 1.4426950408889634f;
  P.negate = scale < 0.f;
  const uint64_t rows = (uint64_t)c.pages * c.kv_heads * c.page_size;
  const uint32_t box = (uint32_t)attn_rows_box(c.page_size);
  if (!encode_tmap_slabs_bf16(&P.kmap, c.k_dev, (uint64_t)c.head_dim, rows, box, (uint32_t)c.head_dim / 64) ||
      !encode_tmap_slabs_bf16(&P.vmap, c.v_dev, (uint64_t)c.head_dim, rows, box, (uint32_t)c.head_dim / 64))
    return GS_ERR_CUDA;
  const int64_t most = (int64_t)b.max_new * P.group;
  P.min_rows = 1;
  P.max_rows = attn_rows_most();
  P.zero_rest = most <= attn_rows_most();
  gs_status st = launch_attn_rows(P, c.head_dim, most < attn_rows_most() ? (int)most : attn_rows_most(), attention_ctas(), s);
  if (st != GS_OK || P.zero_rest) return st;
  P.min_rows = attn_rows_most() + 1;
  const dim3 grid((unsigned)b.tokens, (unsigned)((q_heads + 3) / 4));
  if (c.head_dim == 128) k_attention_simple<128><<<grid, 128, 0, s>>>(P);
  else k_attention_simple<64><<<grid, 128, 0, s>>>(P);
  note_launch();
  return cudaGetLastError() == cudaSuccess ? GS_OK : GS_ERR_CUDA;
}

}  // namespace gs
