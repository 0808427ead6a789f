// The operators around a block's projections: norm, adapters, cache and attention.
#pragma once

#include "gs_common.cuh"

namespace gs {

constexpr int kMaxRank = 128;         // low-rank adapters
constexpr int kMaxAdapterLayers = 8;  // layers of one gs_adapters_batched call

// norm.cu
gs_status launch_add_rms_norm(const void* x, const void* res, const void* w, int64_t T, int64_t n, float eps, void* h,
                              void* y, void* y8, float* scales, int32_t group, cudaStream_t s);
// adapters.cu
gs_status launch_adapters(const gs_adapter_layer* layers, int n, const int32_t* offsets, const int32_t* ids, int32_t n_seqs,
                          int64_t T, cudaStream_t s);
// append.cu
gs_status launch_cache_append(const gs_paged_cache& c, const gs_seq_batch& b, const void* q, int64_t q_stride, int32_t q_heads,
                              const void* k, int64_t k_stride, const void* v, int64_t v_stride, const float* cos_t,
                              const float* sin_t, int64_t n_pos, void* q_out, cudaStream_t s);
// attention.cu
bool attention_units_fit(const gs_paged_cache& c, const gs_seq_batch& b, int32_t q_heads);   // work is counted in 32 bits
size_t attention_workspace_bytes(const gs_paged_cache& c, const gs_seq_batch& b, int32_t q_heads);
gs_status launch_paged_attention(const gs_paged_cache& c, const gs_seq_batch& b, const void* q, int64_t q_stride,
                                 int32_t q_heads, float scale, void* out, void* ws, cudaStream_t s);

inline int sm_count() {
  static const int n = []() {
    int dev = 0, v = 0;
    if (cudaGetDevice(&dev) != cudaSuccess ||
        cudaDeviceGetAttribute(&v, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || v <= 0)
      v = 148;
    return v;
  }();
  return n;
}

// These kernels are short and follow one another: each may be set up while the launch before it
// drains, and begins by waiting for that one's end (start_of_work, by every thread, before
// anything is read or written).  Us in a graph, plain / so: append of 16 tokens 2.5 / 2.1,
// attention of one token 7.7 / 7.3, norm of 1 x 4096 1.9 / 1.75.
template <class P>
gs_status launch_behind(void (*kernel)(P), dim3 grid, unsigned threads, size_t smem, cudaStream_t s, const P& params) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cudaLaunchAttribute overlap;
  overlap.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  overlap.val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = &overlap;
  cfg.numAttrs = 1;
  const cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, params);
  note_launch();
  return e == cudaSuccess ? GS_OK : GS_ERR_CUDA;
}
__device__ __forceinline__ void start_of_work() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

// Number of entries i in [1, n] of a non-decreasing list with at[i] <= v, by a whole
// block (any barrier-synchronised block size).  n is at least 1.
__device__ __forceinline__ int block_count_le(const int32_t* __restrict__ at, int n, int v) {
  int c = 0;
  for (int i0 = 0; i0 < n; i0 += (int)blockDim.x) {
    const int i = i0 + (int)threadIdx.x;
    c += __syncthreads_count(i < n && __ldg(at + 1 + i) <= v);
  }
  return c;
}

__device__ __forceinline__ float bf16_lo(uint32_t v) { return __uint_as_float(v << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t v) { return __uint_as_float(v & 0xFFFF0000u); }
// {lo, hi} rounded to nearest even
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}

}  // namespace gs
