// C ABI of the operators around a block's projections: argument checks and dispatch.
#include "gs_block.cuh"

#include <cmath>

using namespace gs;

namespace {

bool aligned(const void* p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

// [a, a + na) and [b, b + nb) share bytes
bool overlap(const void* a, size_t na, const void* b, size_t nb) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return a && b && na && nb && x < y + nb && y < x + na;
}

gs_status check_cache(const gs_paged_cache* c) {
  if (!c || !c->k_dev || !c->v_dev || !aligned(c->k_dev, 16) || !aligned(c->v_dev, 16)) return GS_ERR_INVALID_ARG;
  if (c->pages <= 0 || c->kv_heads <= 0 || c->page_size <= 0 || c->head_dim <= 0) return GS_ERR_INVALID_ARG;
  if (c->page_size < 16 || c->page_size > 256 || (c->page_size & (c->page_size - 1)) != 0) return GS_ERR_UNSUPPORTED;
  if (c->head_dim != 64 && c->head_dim != 128) return GS_ERR_UNSUPPORTED;
  // rows of the cache are counted in 32 bits (a TMA coordinate)
  if (c->pages > INT32_MAX / c->page_size / c->kv_heads) return GS_ERR_UNSUPPORTED;
  return GS_OK;
}

gs_status check_batch(const gs_seq_batch* b, const gs_paged_cache* c) {
  if (!b || b->n < 0 || b->tokens < 0 || b->tokens >= INT32_MAX || b->max_new < 0 || b->table_width < 0)
    return GS_ERR_INVALID_ARG;
  if (b->n == 0 || b->tokens == 0) return GS_OK;
  if (!b->offsets_dev || !b->kv_lens_dev || !b->table_dev || b->table_width == 0) return GS_ERR_INVALID_ARG;
  if (!aligned(b->offsets_dev, 4) || !aligned(b->kv_lens_dev, 4) || !aligned(b->table_dev, 4)) return GS_ERR_INVALID_ARG;
  if (b->table_width > INT32_MAX / c->page_size) return GS_ERR_INVALID_ARG;
  return GS_OK;
}

}  // namespace

extern "C" {

gs_status gs_add_rms_norm(const void* x_dev, const void* residual_dev, const void* w_dev, int64_t T, int64_t n, float eps,
                          void* h_dev, void* y_dev, void* y8_dev, float* scales_dev, int32_t group, void* stream) {
  if (T < 0 || T > INT32_MAX || n < 1 || n > (1 << 24) || !(eps >= 0.f) || !std::isfinite(eps)) return GS_ERR_INVALID_ARG;
  if (y8_dev && group != 0 && group != 128) return GS_ERR_UNSUPPORTED;
  if (!y_dev && !y8_dev) return GS_ERR_INVALID_ARG;
  if (T == 0) return GS_OK;
  if (!x_dev || !w_dev || !aligned(x_dev, 16) || !aligned(residual_dev, 16) || !aligned(w_dev, 16) || !aligned(h_dev, 16) ||
      !aligned(y_dev, 16) || !aligned(y8_dev, 16) || !aligned(scales_dev, 4) || (y8_dev && !scales_dev))
    return GS_ERR_INVALID_ARG;
  // outputs: h may be x or the residual, y may be x; nothing else overlaps
  const size_t wide = (size_t)T * (size_t)n * 2, row = (size_t)n * 2;
  const size_t n8 = (size_t)T * (size_t)n, nsc = y8_dev ? (size_t)T * (group ? (size_t)(n + group - 1) / group : 1) * 4 : 0;
  if ((h_dev != x_dev && overlap(h_dev, wide, x_dev, wide)) || (h_dev != residual_dev && overlap(h_dev, wide, residual_dev, wide)) ||
      (y_dev != x_dev && overlap(y_dev, wide, x_dev, wide)) || overlap(y_dev, wide, residual_dev, wide) ||
      overlap(y_dev, wide, h_dev, wide) || overlap(h_dev, wide, w_dev, row) || overlap(y_dev, wide, w_dev, row))
    return GS_ERR_INVALID_ARG;
  const void* others[5] = {x_dev, residual_dev, h_dev, y_dev, w_dev};
  for (int i = 0; i < 5 && y8_dev; ++i)
    if (overlap(y8_dev, n8, others[i], i == 4 ? row : wide) || overlap(scales_dev, nsc, others[i], i == 4 ? row : wide))
      return GS_ERR_INVALID_ARG;
  if (y8_dev && overlap(y8_dev, n8, scales_dev, nsc)) return GS_ERR_INVALID_ARG;
  return launch_add_rms_norm(x_dev, residual_dev, w_dev, T, n, eps, h_dev, y_dev, y8_dev, y8_dev ? scales_dev : nullptr, group,
                             static_cast<cudaStream_t>(stream));
}

gs_status gs_adapters_batched(int32_t n, const gs_adapter_layer* layers, const int32_t* offsets_dev, const int32_t* ids_dev,
                              int32_t n_seqs, int64_t T, void* stream) {
  if (n < 0 || n > kMaxAdapterLayers || n_seqs < 0 || T < 0 || T >= INT32_MAX) return GS_ERR_INVALID_ARG;
  if (n == 0) return GS_OK;
  if (!layers) return GS_ERR_INVALID_ARG;
  for (int i = 0; i < n; ++i) {
    const gs_adapter_layer& L = layers[i];
    if (L.in < 8 || L.in % 8 != 0 || L.out < 1 || L.in > INT32_MAX || L.out > INT32_MAX || L.n_adapters < 1 || L.rank < 1)
      return GS_ERR_INVALID_ARG;
    if (L.rank % 8 != 0 || L.rank > kMaxRank) return GS_ERR_UNSUPPORTED;
    if (L.in * L.rank > INT32_MAX || L.out * L.rank > INT32_MAX) return GS_ERR_UNSUPPORTED;
  }
  if (n_seqs == 0 || T == 0) return GS_OK;
  if (!offsets_dev || !ids_dev || !aligned(offsets_dev, 4) || !aligned(ids_dev, 4)) return GS_ERR_INVALID_ARG;
  for (int i = 0; i < n; ++i) {
    const gs_adapter_layer& L = layers[i];
    if (!L.x_dev || !L.base_dev || !L.out_dev || !L.A_dev || !L.B_dev || !L.scale_dev) return GS_ERR_INVALID_ARG;
    if (!aligned(L.x_dev, 16) || !aligned(L.base_dev, 16) || !aligned(L.out_dev, 16) || !aligned(L.A_dev, 16) ||
        !aligned(L.B_dev, 16) || !aligned(L.scale_dev, 4))
      return GS_ERR_INVALID_ARG;
    const size_t bytes = (size_t)T * (size_t)L.out * 2;
    if (L.out_dev != L.base_dev && overlap(L.out_dev, bytes, L.base_dev, bytes)) return GS_ERR_INVALID_ARG;
    for (int j = 0; j < n; ++j) {
      if (overlap(L.out_dev, bytes, layers[j].x_dev, (size_t)T * (size_t)layers[j].in * 2)) return GS_ERR_INVALID_ARG;
      if (j != i && (overlap(L.out_dev, bytes, layers[j].out_dev, (size_t)T * (size_t)layers[j].out * 2) ||
                     overlap(L.out_dev, bytes, layers[j].base_dev, (size_t)T * (size_t)layers[j].out * 2)))
        return GS_ERR_INVALID_ARG;
    }
  }
  return launch_adapters(layers, n, offsets_dev, ids_dev, n_seqs, T, static_cast<cudaStream_t>(stream));
}

gs_status gs_cache_append(const gs_paged_cache* cache, const gs_seq_batch* batch, const void* q_dev, int64_t q_stride,
                          int32_t q_heads, const void* k_dev, int64_t k_stride, const void* v_dev, int64_t v_stride,
                          const float* cos_dev, const float* sin_dev, int64_t n_pos, void* q_out_dev, void* stream) {
  gs_status st = check_cache(cache);
  if (st != GS_OK || (st = check_batch(batch, cache)) != GS_OK) return st;
  const int64_t D = cache->head_dim, kv_row = cache->kv_heads * D;
  if (q_heads <= 0 || q_heads > (1 << 20) || n_pos < 1) return GS_ERR_INVALID_ARG;
  if (q_stride < q_heads * D || k_stride < kv_row || v_stride < kv_row || q_stride % 8 || k_stride % 8 || v_stride % 8)
    return GS_ERR_INVALID_ARG;
  if (batch->tokens == 0) return GS_OK;
  if (batch->n == 0) return GS_ERR_INVALID_ARG;   // tokens of no sequence
  if (!q_dev || !k_dev || !v_dev || !cos_dev || !sin_dev || !q_out_dev || !aligned(q_dev, 16) || !aligned(k_dev, 16) ||
      !aligned(v_dev, 16) || !aligned(cos_dev, 16) || !aligned(sin_dev, 16) || !aligned(q_out_dev, 16))
    return GS_ERR_INVALID_ARG;
  // q_out may be q itself, densely stored; otherwise the outputs overlap no input
  const size_t T = (size_t)batch->tokens, out_b = T * (size_t)(q_heads * D) * 2;
  const size_t qb = ((T - 1) * (size_t)q_stride + (size_t)(q_heads * D)) * 2, kb = ((T - 1) * (size_t)k_stride + (size_t)kv_row) * 2,
               vb = ((T - 1) * (size_t)v_stride + (size_t)kv_row) * 2;
  const size_t cb = (size_t)cache->pages * (size_t)(cache->page_size * kv_row) * 2;
  if (!(q_out_dev == q_dev && q_stride == q_heads * D) && overlap(q_out_dev, out_b, q_dev, qb)) return GS_ERR_INVALID_ARG;
  if (overlap(q_out_dev, out_b, k_dev, kb) || overlap(q_out_dev, out_b, v_dev, vb)) return GS_ERR_INVALID_ARG;
  const void* pages[2] = {cache->k_dev, cache->v_dev};
  for (const void* p : pages)
    if (overlap(p, cb, q_dev, qb) || overlap(p, cb, k_dev, kb) || overlap(p, cb, v_dev, vb) || overlap(p, cb, q_out_dev, out_b))
      return GS_ERR_INVALID_ARG;
  if (overlap(pages[0], cb, pages[1], cb)) return GS_ERR_INVALID_ARG;
  return launch_cache_append(*cache, *batch, q_dev, q_stride, q_heads, k_dev, k_stride, v_dev, v_stride, cos_dev, sin_dev, n_pos,
                             q_out_dev, static_cast<cudaStream_t>(stream));
}

static gs_status check_attention(const gs_paged_cache* cache, const gs_seq_batch* batch, int32_t q_heads) {
  gs_status st = check_cache(cache);
  if (st != GS_OK || (st = check_batch(batch, cache)) != GS_OK) return st;
  if (q_heads <= 0 || q_heads % cache->kv_heads != 0) return GS_ERR_INVALID_ARG;
  if (q_heads / cache->kv_heads > 64 || !attention_units_fit(*cache, *batch, q_heads)) return GS_ERR_UNSUPPORTED;
  return GS_OK;
}

gs_status gs_paged_attention_workspace(const gs_paged_cache* cache, const gs_seq_batch* batch, int32_t q_heads, size_t* bytes) {
  const gs_status st = check_attention(cache, batch, q_heads);
  if (st != GS_OK) return st;
  if (!bytes) return GS_ERR_INVALID_ARG;
  *bytes = attention_workspace_bytes(*cache, *batch, q_heads);
  return GS_OK;
}

gs_status gs_paged_attention(const gs_paged_cache* cache, const gs_seq_batch* batch, const void* q_dev, int64_t q_stride,
                             int32_t q_heads, float scale, void* out_dev, void* workspace_dev, size_t workspace_bytes,
                             void* stream) {
  const gs_status st = check_attention(cache, batch, q_heads);
  if (st != GS_OK) return st;
  const int64_t row = (int64_t)q_heads * cache->head_dim;
  if (q_stride < row || q_stride % 8 != 0 || !std::isfinite(scale)) return GS_ERR_INVALID_ARG;
  if (batch->tokens == 0) return GS_OK;
  if (batch->n == 0) return GS_ERR_INVALID_ARG;
  if (!q_dev || !out_dev || !aligned(q_dev, 16) || !aligned(out_dev, 16)) return GS_ERR_INVALID_ARG;
  const size_t need = attention_workspace_bytes(*cache, *batch, q_heads);
  if (workspace_bytes < need || (need && (!workspace_dev || !aligned(workspace_dev, 16)))) return GS_ERR_INVALID_ARG;
  const size_t T = (size_t)batch->tokens, ob = T * (size_t)row * 2, qb = ((T - 1) * (size_t)q_stride + (size_t)row) * 2;
  const size_t cb = (size_t)cache->pages * (size_t)cache->page_size * (size_t)cache->kv_heads * (size_t)cache->head_dim * 2;
  if (overlap(out_dev, ob, q_dev, qb) || overlap(out_dev, ob, cache->k_dev, cb) || overlap(out_dev, ob, cache->v_dev, cb) ||
      overlap(workspace_dev, need, out_dev, ob) || overlap(workspace_dev, need, q_dev, qb) ||
      overlap(workspace_dev, need, cache->k_dev, cb) || overlap(workspace_dev, need, cache->v_dev, cb))
    return GS_ERR_INVALID_ARG;
  return launch_paged_attention(*cache, *batch, q_dev, q_stride, q_heads, scale, out_dev, workspace_dev,
                                static_cast<cudaStream_t>(stream));
}

}  // extern "C"
