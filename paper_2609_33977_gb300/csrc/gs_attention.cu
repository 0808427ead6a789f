// Attention over a paged cache: which kernel serves which sequence, workspace, launch.
#include "gs_attn.cuh"

#include <algorithm>
#include <cmath>

namespace gs {
namespace {

// Arrival counters (two levels; two halves in the chunk kernel), then the parts of split
// items, each kernel's its own: the two launches of a step overlap.
constexpr int kMaxCtas = 256;
constexpr int64_t kCounterBytes = GS_ATTENTION_COUNTER_BYTES;
static_assert(kCounterBytes >= 6 * 4 * kMaxCtas, "six counters a CTA");

int attention_ctas() { return std::min(sm_count(), kMaxCtas); }

size_t parts_bytes(int size) { return (size_t)attention_ctas() * 2 * (size_t)size * 4; }

// The few-row kernel serves sequences of at most attn_rows_most() = 32 rows (over 8 bits up to 64, see there), the chunk kernel
// the others.  Us in the few-row / the chunk kernel, 128-wide heads: 7 rows  one token at 129
// keys (28/4 heads) 6.9 / 10.0,  28 rows  16 x 4 tokens at 2000 keys 28.9 / 29.1,  32 rows
// 16 x 32 (32 heads) 102.9 / 104.6;  above, in a few-row form for 64 rows and before the chunk
// kernel's last steps,  16 x 9 41 / 34,  16 x 64 156 / 117.
// Over 8 bits: 32 rows  16 x 32 (32 heads, 2000 keys) 103 / 137,  28 rows  4 tokens at 60000 keys 38.2 / 75.
// Where all sequences are as long as the longest (known from the sizes alone), one launch does
// (4096 tokens of 40 heads 154 us, both launches 158); otherwise the host cannot tell, and both
// kernels look for theirs, the second on SMs that the first is through with (a mixed step of
// 681 tokens 77 us, one launch behind the other 80).
struct Kernels {
  bool few, chunk;
};
int few_most(const gs_paged_cache& c, const CacheScales& sc, const gs_seq_batch& b) {
  return sc.k ? attn_rows_fp8_most((int64_t)b.n * c.kv_heads, attention_ctas()) : attn_rows_most();
}
Kernels kernels_of(const gs_paged_cache& c, const CacheScales& sc, const gs_seq_batch& b, int32_t group) {
  const int64_t most = (int64_t)b.max_new * group;
  if (most <= few_most(c, sc, b)) return {true, false};
  return {b.tokens != (int64_t)b.n * b.max_new, true};
}

// Rows of D codes, swizzled over their D bytes; copied as D / 2 pairs of bytes.
bool encode_rows_fp8(CUtensorMap* map, const void* base, uint64_t D, uint64_t rows, uint32_t box) {
  return encode_tmap_2d_bf16_swz(map, base, D / 2, rows, (uint32_t)D / 2, box, (int)D);
}

}  // namespace

bool attention_units_fit(const gs_paged_cache& c, const gs_seq_batch& b, int32_t q_heads) {
  const double rows = (double)b.tokens * (q_heads / c.kv_heads), cap = (double)b.table_width * c.page_size;
  const double items = (rows / attn_chunk_rows() + b.n + 1.0) * c.kv_heads;
  const double units = items * (cap / std::min(attn_rows_tile(), attn_chunk_tile()) + 1.0 + attn_most_over());
  // the key behind a sequence's last tile is still a number of 32 bits
  return rows < 1e9 && units < 2e9 && cap <= 2147483648.0 - 256.0;
}

size_t attention_workspace_bytes(const gs_paged_cache& c, const CacheScales& sc, const gs_seq_batch& b, int32_t q_heads) {
  const Kernels k = kernels_of(c, sc, b, q_heads / c.kv_heads);
  return (size_t)kCounterBytes + (k.chunk ? parts_bytes(attn_chunk_part(c.head_dim)) : 0) +
         (k.few ? parts_bytes(attn_rows_part(c.head_dim)) : 0);
}

gs_status launch_paged_attention(const gs_paged_cache& c, const CacheScales& sc, const gs_seq_batch& b, const void* q, int64_t q_stride,
                                 int32_t q_heads, float scale, void* out, void* ws, cudaStream_t s) {
  AttnParams P;
  P.q = static_cast<const uint16_t*>(q);
  P.v = static_cast<const uint16_t*>(c.v_dev);
  P.out = static_cast<uint16_t*>(out);
  P.k_scales = sc.k;
  P.v_scales = sc.v;
  P.offsets = b.offsets_dev;
  P.kv_lens = b.kv_lens_dev;
  P.table = b.table_dev;
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
  P.group_inv = 0xFFFFFFFFu / (uint32_t)P.group;
  P.half_tokens = 0;
  P.even = b.tokens == (int64_t)b.n * b.max_new;
  // a scale of zero weighs all keys alike: so does one this small, and masked scores (-inf) stay what they are
  P.scale_log2 = std::max(std::fabs(scale) * 1.4426950408889634f, 1e-36f);
  P.negate = scale < 0.f;
  const uint64_t rows = (uint64_t)c.pages * c.kv_heads * c.page_size, D = (uint64_t)c.head_dim;
  const uint32_t slabs = (uint32_t)D / 64;
  const Kernels k = kernels_of(c, sc, b, P.group);
  P.two_launches = k.few && k.chunk;
  int32_t* cnt = static_cast<int32_t*>(ws);
  uint8_t* parts = static_cast<uint8_t*>(ws) + kCounterBytes;
  if (k.chunk) {   // first: it is the longer one, and the other fills the SMs as they come free
    const uint32_t box = (uint32_t)attn_chunk_box(c.page_size);
    // keys of a page smaller than a unit arrive slab by slab; codes row by row, as they lie
    if (sc.k) {
      if (!encode_tmap_2d_bf16(&P.kmap, c.k_dev, D / 2, rows, (uint32_t)D / 2, box, false) ||
          !encode_tmap_2d_bf16(&P.vmap, c.v_dev, D / 2, rows, (uint32_t)D / 2, box, false))
        return GS_ERR_CUDA;
    } else if (!encode_tmap_slabs_bf16(&P.kmap, c.k_dev, D, rows, box, (int)box == attn_chunk_tile() ? slabs : 1u) ||
               !encode_tmap_slabs_bf16(&P.vmap, c.v_dev, D, rows, box, slabs)) {
      return GS_ERR_CUDA;
    }
    P.half_tokens = attn_chunk_half_tokens(P.group);
    const uint64_t dims[3] = {D, (uint64_t)q_heads, (uint64_t)b.tokens}, strides[2] = {D * 2, (uint64_t)q_stride * 2};
    const uint32_t qbox[3] = {64, (uint32_t)P.group, (uint32_t)P.half_tokens};
    if (!encode_tmap_nd_bf16(&P.qmap, q, 3, dims, strides, qbox, 128)) return GS_ERR_CUDA;
    P.cnt = cnt;
    P.parts = reinterpret_cast<float*>(parts);
    P.min_rows = k.few ? few_most(c, sc, b) + 1 : 1;
    P.max_rows = INT32_MAX;
    P.zero_rest = !k.few;
    P.inject_ns = take_injected_wait(kInjectAttnChunk);
    const gs_status st = launch_attn_chunk(P, c.head_dim, attention_ctas(), s);
    if (st != GS_OK || !k.few) return st;
  }
  const uint32_t box = (uint32_t)(sc.k ? attn_rows_fp8_box(c.page_size) : attn_rows_box(c.page_size));
  if (!(sc.k ? encode_rows_fp8(&P.kmap, c.k_dev, D, rows, box) && encode_rows_fp8(&P.vmap, c.v_dev, D, rows, box)
             : encode_tmap_slabs_bf16(&P.kmap, c.k_dev, D, rows, box, slabs) && encode_tmap_slabs_bf16(&P.vmap, c.v_dev, D, rows, box, slabs)))
    return GS_ERR_CUDA;
  P.cnt = cnt + 4 * kMaxCtas;
  P.parts = reinterpret_cast<float*>(parts + (k.chunk ? parts_bytes(attn_chunk_part(c.head_dim)) : 0));
  P.min_rows = 1;
  const int most = (int)std::min((int64_t)b.max_new * P.group, (int64_t)few_most(c, sc, b));
  P.max_rows = sc.k ? (most > attn_rows_most() ? few_most(c, sc, b) : attn_rows_most()) : attn_rows_held(most);
  P.zero_rest = !k.chunk;
  P.inject_ns = take_injected_wait(kInjectAttnRows);
  return sc.k ? launch_attn_rows_fp8(P, c.head_dim, attention_ctas(), s) : launch_attn_rows(P, c.head_dim, attention_ctas(), s);
}

}  // namespace gs
