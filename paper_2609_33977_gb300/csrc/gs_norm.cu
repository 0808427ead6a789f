// RMS norm of a block's residual stream, with the residual's addition:
//     h = x + r,   y = h * rsqrt(mean(h^2) + eps) * w
// y is formed from the float32 sum h (not from the bf16 h that is stored for the
// next block), and rounded once: to bf16, or per group of columns to e4m3 with
// scale = max(max|y| / 448, 2^-126), q = y / scale.
//
// HBM-bound: 8 bytes per element in bf16 (x, r, h, y) and 4 operations.  One block
// per row keeps the row in registers (8 elements = one 16-byte vector per thread
// and step), so x and r are read once; sums are float32.  Rows whose length is no
// multiple of 8, or above 32768, take k_norm_any, which reads them again per pass
// (512 x 16384: 36 us against 12.2).  2047 x 5120 takes 13.7 us, 6.1 TB/s, in 8 bits 14.4
// (5.1 TB/s); one row of 4096 takes 1.4 us, a launch.
#include "gs_block.cuh"

#include <cfloat>

namespace gs {
namespace {

constexpr float kE4m3Max = 448.f;
constexpr float kScaleMin = 1.17549435e-38f;   // 2^-126, the least number of full precision

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
  return v;
}
__device__ __forceinline__ float warp_max(float v, int width = 32) {
  for (int d = width / 2; d > 0; d >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, d));
  return v;
}
// over the block, in a fixed order; red: 32 floats of shared memory, free afterwards
template <bool kMax>
__device__ __forceinline__ float block_reduce(float v, float* red) {
  v = kMax ? warp_max(v) : warp_sum(v);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, n = (blockDim.x + 31) >> 5;
  __syncthreads();
  if (lane == 0) red[warp] = v;
  __syncthreads();
  v = lane < n ? red[lane] : 0.f;
  return kMax ? warp_max(v) : warp_sum(v);
}

// A mean square (eps in it) that float32 squares do not give: out of their range, or of magnitudes that they lose.
__device__ __forceinline__ bool off_range(float ms) { return !(ms >= 0x1p-100f && ms <= FLT_MAX); }
// Such a row is scaled first, by the power of two that brings the larger of its largest magnitude and eps' root near 1
// (1: an infinite or empty row).  Rows of 1e20, say, whose squares are infinite, would be zeros otherwise.
__device__ __forceinline__ float row_scale(float amax, float eps) {
  const float top = fmaxf(amax, sqrtf(eps));
  if (!(top > 0.f) || isinf(top)) return 1.f;
  return __uint_as_float((uint32_t)max(1, 254 - (int)(__float_as_uint(top) >> 23)) << 23);
}

// four e4m3 codes, the first in the low byte (NaN stays NaN; the scale keeps the rest within 448)
__device__ __forceinline__ uint32_t pack_e4m3(float a, float b, float c, float d) {
  uint16_t lo, hi;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(lo) : "f"(b), "f"(a));
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(hi) : "f"(d), "f"(c));
  return (uint32_t)lo | ((uint32_t)hi << 16);
}
__device__ __forceinline__ float group_scale(float amax) { return fmaxf(amax / kE4m3Max, kScaleMin); }

// y / scale, rounded to nearest: the product with the rounded reciprocal, corrected once by its exact remainder
// (Markstein, IBM J. Res. Dev. 34, 1990).  Values near the middle of two codes need it: the product alone takes some to
// the other code.  Both are scaled where the remainder would fall below the least float32.  (Us of the product alone /
// so / one division an element: 777 x 3584  5.3 / 5.6 / 6.7, 2047 x 5120  14.3 / 14.9 / 17.6.)
struct Quotient {
  float up, scale, inv;
  __device__ __forceinline__ explicit Quotient(float sc) {
    up = sc < 1.f / (1ull << 62) ? (float)(1ull << 62) : 1.f;
    inv = 1.f / (sc * up);
    scale = isinf(sc) ? 0.f : sc * up;   // of an infinite scale finite y are zero, and infinite ones NaN
  }
  __device__ __forceinline__ float operator()(float y) const {
    y *= up;
    const float q = y * inv;
    return fmaf(fmaf(-q, scale, y), inv, q);
  }
};

struct NormParams {
  const uint16_t* x;
  const uint16_t* res;   // may be null
  const uint16_t* w;
  uint16_t* h;           // may be null
  uint16_t* y;           // may be null
  uint8_t* y8;           // may be null
  float* scales;         // [T][ceil(n / group)], with y8
  int64_t T;
  int32_t n, group;      // group 0: the whole row
  float eps;
};

// V vectors of 8 elements per thread; vector i of the row belongs to thread i % blockDim.x.
// Up to 1024 threads, so 64 registers at most; 56 with two vectors, or an SM holds four rows of 3584 instead of five
// (777 of them: 5.1 us, 4.6 so).
template <int V>
__global__ void __maxnreg__(V == 2 ? 56 : 64) k_norm(const NormParams P) {
  __shared__ float red[32];
  start_of_work();
  const int nv = P.n >> 3;
  const int64_t row = blockIdx.x;
  const uint4* xr = reinterpret_cast<const uint4*>(P.x + row * P.n);
  const uint4* rr = reinterpret_cast<const uint4*>(P.res + row * P.n);
  const uint4 zero = make_uint4(0u, 0u, 0u, 0u);
  uint4 a[V], b[V], w[V];
#pragma unroll
  for (int v = 0; v < V; ++v) {
    const int i = (int)threadIdx.x + v * (int)blockDim.x;
    a[v] = i < nv ? __ldcs(xr + i) : zero;
    b[v] = i < nv && P.res ? __ldcs(rr + i) : zero;
    w[v] = i < nv ? __ldg(reinterpret_cast<const uint4*>(P.w) + i) : zero;
  }
  float h[V][8];
  float ss = 0.f;
#pragma unroll
  for (int v = 0; v < V; ++v) {
    const uint32_t ax[4] = {a[v].x, a[v].y, a[v].z, a[v].w}, bx[4] = {b[v].x, b[v].y, b[v].z, b[v].w};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      h[v][2 * e] = P.res ? bf16_lo(ax[e]) + bf16_lo(bx[e]) : bf16_lo(ax[e]);
      h[v][2 * e + 1] = P.res ? bf16_hi(ax[e]) + bf16_hi(bx[e]) : bf16_hi(ax[e]);
      ss = fmaf(h[v][2 * e], h[v][2 * e], ss);
      ss = fmaf(h[v][2 * e + 1], h[v][2 * e + 1], ss);
    }
    const int i = (int)threadIdx.x + v * (int)blockDim.x;
    if (P.h && i < nv)
      reinterpret_cast<uint4*>(P.h + row * P.n)[i] =
          make_uint4(pack_bf16(h[v][0], h[v][1]), pack_bf16(h[v][2], h[v][3]), pack_bf16(h[v][4], h[v][5]),
                     pack_bf16(h[v][6], h[v][7]));
  }
  float ms = block_reduce<false>(ss, red) / (float)P.n + P.eps, amax = 0.f;
  if (off_range(ms)) {   // the same for the whole block
#pragma unroll
    for (int v = 0; v < V; ++v)
#pragma unroll
      for (int e = 0; e < 8; ++e) amax = fmaxf(amax, fabsf(h[v][e]));
    const float s = row_scale(block_reduce<true>(amax, red), P.eps);
    ss = amax = 0.f;
#pragma unroll
    for (int v = 0; v < V; ++v)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        h[v][e] *= s;
        ss = fmaf(h[v][e], h[v][e], ss);
      }
    ms = block_reduce<false>(ss, red) / (float)P.n + P.eps * s * s;
  }
  const float inv = rsqrtf(ms);
#pragma unroll
  for (int v = 0; v < V; ++v) {
    const uint32_t wx[4] = {w[v].x, w[v].y, w[v].z, w[v].w};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      h[v][2 * e] *= inv * bf16_lo(wx[e]);
      h[v][2 * e + 1] *= inv * bf16_hi(wx[e]);
    }
    const int i = (int)threadIdx.x + v * (int)blockDim.x;
    if (P.y && i < nv)
      reinterpret_cast<uint4*>(P.y + row * P.n)[i] =
          make_uint4(pack_bf16(h[v][0], h[v][1]), pack_bf16(h[v][2], h[v][3]), pack_bf16(h[v][4], h[v][5]),
                     pack_bf16(h[v][6], h[v][7]));
#pragma unroll
    for (int e = 0; e < 8; ++e) amax = fmaxf(amax, fabsf(h[v][e]));
  }
  if (!P.y8) return;
  float sc = 0.f;
  if (P.group == 0) {
    sc = group_scale(block_reduce<true>(amax, red));
    if (threadIdx.x == 0) P.scales[row] = sc;
  }
  const int ng = P.group ? (P.n + P.group - 1) / P.group : 1;
#pragma unroll
  for (int v = 0; v < V; ++v) {
    const int i = (int)threadIdx.x + v * (int)blockDim.x;
    if (P.group) {   // 128 columns: 16 neighbouring threads
      float m = 0.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) m = fmaxf(m, fabsf(h[v][e]));
      sc = group_scale(warp_max(m, 16));
      if (i < nv && (i & 15) == 0) P.scales[row * ng + (i >> 4)] = sc;
    }
    const Quotient by(sc);
    if (i < nv)
      reinterpret_cast<uint2*>(P.y8 + row * P.n)[i] =
          make_uint2(pack_e4m3(by(h[v][0]), by(h[v][1]), by(h[v][2]), by(h[v][3])),
                     pack_e4m3(by(h[v][4]), by(h[v][5]), by(h[v][6]), by(h[v][7])));
  }
}

// Any row length: one element per thread and step, the row read again for each pass.
__global__ void __launch_bounds__(256) k_norm_any(const NormParams P) {
  __shared__ float red[32];
  start_of_work();
  const int64_t row = blockIdx.x;
  const uint16_t* x = P.x + row * P.n;
  const uint16_t* r = P.res ? P.res + row * P.n : nullptr;
  const auto at = [&](int i) {
    const float a = bf16_lo(x[i]);
    return r ? a + bf16_lo(r[i]) : a;
  };
  float ss = 0.f;
  for (int i = threadIdx.x; i < P.n; i += 256) {
    const float h = at(i);
    ss = fmaf(h, h, ss);
  }
  float ms = block_reduce<false>(ss, red) / (float)P.n + P.eps, s = 1.f;
  if (off_range(ms)) {
    float amax = 0.f;
    for (int i = threadIdx.x; i < P.n; i += 256) amax = fmaxf(amax, fabsf(at(i)));
    s = row_scale(block_reduce<true>(amax, red), P.eps);
    ss = 0.f;
    for (int i = threadIdx.x; i < P.n; i += 256) {
      const float h = at(i) * s;
      ss = fmaf(h, h, ss);
    }
    ms = block_reduce<false>(ss, red) / (float)P.n + P.eps * s * s;
  }
  const float inv = rsqrtf(ms);
  const auto out = [&](int i) { return at(i) * s * (inv * bf16_lo(P.w[i])); };
  if (P.y8) {
    const int width = P.group ? P.group : P.n, ng = (P.n + width - 1) / width;
    for (int g = 0; g < ng; ++g) {
      const int end = min(P.n, (g + 1) * width);
      float amax = 0.f;
      for (int i = g * width + (int)threadIdx.x; i < end; i += 256) amax = fmaxf(amax, fabsf(out(i)));
      const float sc = group_scale(block_reduce<true>(amax, red));
      const Quotient by(sc);
      if (threadIdx.x == 0) P.scales[row * ng + g] = sc;
      for (int i = g * width + (int)threadIdx.x; i < end; i += 256)
        P.y8[row * P.n + i] = (uint8_t)pack_e4m3(by(out(i)), 0.f, 0.f, 0.f);
    }
  }
  // h may be the residual's own buffer and y the input's: every pass above is over
  __syncthreads();
  for (int i = threadIdx.x; i < P.n; i += 256) {
    const float h = at(i), y = h * s * (inv * bf16_lo(P.w[i]));
    if (P.h) P.h[row * P.n + i] = (uint16_t)pack_bf16(h, 0.f);
    if (P.y) P.y[row * P.n + i] = (uint16_t)pack_bf16(y, 0.f);
  }
}

}  // namespace

gs_status launch_add_rms_norm(const void* x, const void* res, const void* w, int64_t T, int64_t n, float eps, void* h,
                              void* y, void* y8, float* scales, int32_t group, cudaStream_t s) {
  NormParams P;
  P.x = static_cast<const uint16_t*>(x);
  P.res = static_cast<const uint16_t*>(res);
  P.w = static_cast<const uint16_t*>(w);
  P.h = static_cast<uint16_t*>(h);
  P.y = static_cast<uint16_t*>(y);
  P.y8 = static_cast<uint8_t*>(y8);
  P.scales = scales;
  P.T = T;
  P.n = (int32_t)n;
  P.group = group;
  P.eps = eps;
  const int64_t nv = n / 8;
  // Vectors a thread, us at 2 / 4 (three sets of buffers, partly in L2): 2048 x 1024  3.1 / 3.5, 777 x 3584 in 8 bits  5.0 / 5.1, 1 x 8192  2.5 / 2.7,
  // 16 x 5120  2.2 / 2.5; 2047 x 5120  12.0 / 11.2, 1024 x 8192  11.0 / 9.9, 2048 x 11008  36.6 / 29.6.
  // (One a thread: 12.2, 11.7 and 36.6 for the last three, and 2 % more than two at 1 x 4096 to 777 x 3584.)
  if (n % 8 == 0 && nv <= 4096) {
    const int v = nv <= 512 || (nv <= 2048 && T <= sm_count()) ? 2 : 4;
    const unsigned threads = (unsigned)(((nv + v - 1) / v + 31) / 32 * 32);
    return launch_behind(v == 2 ? k_norm<2> : k_norm<4>, dim3((unsigned)T), threads, 0, s, P);
  }
  return launch_behind(k_norm_any, dim3((unsigned)T), 256, 0, s, P);
}

}  // namespace gs
