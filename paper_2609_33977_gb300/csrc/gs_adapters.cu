// Low-rank adapters of many requests beside a shared projection:
//     out[t] = base[t] + s_a B_a (A_a x[t]),   a = the adapter of token t's request.
//
// HBM-bound: x, base and out move once (2 r FLOP per element of x and out), A and B
// once per adapter, all of it in one launch for up to 8 layers.  A tile of M tokens
// of one request belongs to a cluster of CL CTAs: CTA c contracts its part of the
// inputs, the partial A x [M][r] are summed over the cluster through distributed
// shared memory in a fixed order, and CTA c then forms its part of the outputs.
// CL is the largest of 8, 4, 2 with which all tiles are resident (ad_cluster).  M is 16
// where requests are short (a decode step has one token each) and 32 where they are
// long, so that A and B come from L2 half as often (launch_adapters).
//
// Products are m16n8k16 with float32 sums.  A contraction may take its index in any
// order, so a lane takes 8 consecutive elements of its row as one 16-byte load and
// feeds them to two MMAs; no operand goes through shared memory.  A x enters the
// second product as hi + lo bf16 (two MMAs), so that its only rounding to 16 bits
// is the output's.  Loads are unconditional, at clamped addresses: one that depends on
// a branch waits for the one before it.
//
// q, k and v of 16 sequences with an adapter each (4096x4096, rank 16): 6.9 us, 10.1 with the
// operands in HBM; 9 MB, so the way of a tile through two products and two cluster barriers,
// not the bytes.  2048 tokens through 4096x11008, rank 32: 27 us, 3.0 TB/s: the loads of one block of inputs wait for
// the products of the one before, and two CTAs an SM do not hide all of it.
#include "gs_block.cuh"

#include <cooperative_groups.h>

namespace gs {
namespace {
namespace cg = cooperative_groups;

constexpr int kAdThreads = 256, kAdWarps = kAdThreads / 32;

struct AdLayer {
  const uint16_t* x;      // [T][in]
  const uint16_t* base;   // [T][out]
  uint16_t* out;          // [T][out]
  const uint16_t* A;      // [n_adapters][rank][in]
  const uint16_t* B;      // [n_adapters][out][rank]
  const float* scale;     // [n_adapters]
  int32_t in, out_n, n_adapters, rank;
};
struct AdParams {
  AdLayer layer[kMaxAdapterLayers];
  const int32_t* offsets;
  const int32_t* ids;
  int64_t T;
  int32_t n_seqs;
};

__device__ __forceinline__ void mma16816(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                         uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// Elements of the rank that a lane feeds to one step of the second product: 8 (two
// MMAs) for ranks in whole 32s, 4 (one MMA) in whole 16s, else 2 (half an MMA).
__host__ __device__ constexpr int rank_elems(int rank) { return rank % 32 == 0 ? 8 : rank % 16 == 0 ? 4 : 2; }

// Columns [col, col + 8) of a lane's 2 mt rows, some of whose sums t [mt][4][4] an infinite element of B made infinite or
// NaN: hi and lo are two terms of one product, which may cancel then, or lo is 0.  Such sums are formed again in float32.
__device__ __noinline__ void store_odd(const AdLayer& L, const float* t, const float* sax, const uint16_t* B, int64_t t0,
                                       int nt, int rank, int col, int mt) {
  const int g = (int)(threadIdx.x & 31) >> 2;
#pragma unroll 1
  for (int i = 0; i < 16 * mt; ++i) {
    const int r = 16 * (i >> 4) + 8 * ((i >> 1) & 1) + g, o = col + 2 * ((i >> 2) & 3) + (i & 1);
    if (r >= nt || o >= L.out_n) continue;
    float s = t[i];
    if (!isfinite(s)) {
      s = 0.f;
#pragma unroll 1
      for (int k = 0; k < rank; ++k) s = fmaf(sax[r * rank + k], bf16_lo(__ldg(B + (int64_t)o * rank + k)), s);
    }
    const int64_t at = (t0 + r) * L.out_n + o;
    L.out[at] = (uint16_t)pack_bf16(bf16_lo(L.base[at]) + s, 0.f);
  }
}

// out columns [32 blk, 32 blk + 32) of the tile: lane (g, q) of a warp ends with
// columns 8 q .. 8 q + 7 of rows g and g + 8 of each 16 tokens.
// v: [m][step][hi, lo][lane] fragments of s A x, sax: its [rows][rank] in float32.
template <int MT, int E>
__device__ __forceinline__ void expand(const AdLayer& L, const uint4* v, const float* sax, const uint16_t* B, int64_t t0, int nt, int rank,
                                       int b0, int b1, int warp, int lane) {
  const int g = lane >> 2, q = lane & 3;
  const int steps = rank / (4 * E);
  const bool vec = (L.out_n & 7) == 0;
  // With one row of tiles and a short contraction two blocks are under way together: a load may not pass the stores
  // before it (the base may be the output), and the loads' wait is all there is.  Us at one / two: q, k, v of 16 tokens,
  // rank 16  7.7 / 7.4;  4096x11008, rank 32, 8 x 48 tokens  9.8 / 10.1;  rank 64, 16 tokens  14.0 / 15.0.
  constexpr int kB = MT == 1 && E <= 4 ? 2 : 1;
  constexpr int kMmas = E == 8 ? 2 : 1;
  for (int blk = b0 + warp; blk < b1; blk += kB * kAdWarps) {
    uint4 base[kB][MT][2];
    float acc[kB][MT][4][4];
#pragma unroll
    for (int b = 0; b < kB; ++b) {
      const int col = 32 * (blk + b * kAdWarps) + 8 * q;
#pragma unroll
      for (int m = 0; m < MT; ++m) {
#pragma unroll
        for (int h = 0; h < 2; ++h)
          if (vec)   // rows and columns past the last: values that nobody uses
            base[b][m][h] = *reinterpret_cast<const uint4*>(L.base + (t0 + min(16 * m + 8 * h + g, nt - 1)) * L.out_n + min(col, L.out_n - 8));
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[b][m][j][e] = 0.f;
      }
    }
    for (int s = 0; s < steps; ++s) {
      uint32_t w[kB][4][4];
#pragma unroll
      for (int b = 0; b < kB; ++b)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int o = 32 * (blk + b * kAdWarps) + 8 * (g >> 1) + 2 * j + (g & 1);   // this lane's row of B in MMA j
          const uint16_t* src = B + (int64_t)min(o, L.out_n - 1) * rank + s * 4 * E + q * E;
          w[b][j][0] = w[b][j][1] = w[b][j][2] = w[b][j][3] = 0u;
          if constexpr (E == 8) {
            const uint4 c = __ldg(reinterpret_cast<const uint4*>(src));
            w[b][j][0] = c.x;
            w[b][j][1] = c.y;
            w[b][j][2] = c.z;
            w[b][j][3] = c.w;
          } else if constexpr (E == 4) {
            const uint2 c = __ldg(reinterpret_cast<const uint2*>(src));
            w[b][j][0] = c.x;
            w[b][j][1] = c.y;
          } else {
            w[b][j][0] = __ldg(reinterpret_cast<const uint32_t*>(src));
          }
        }
#pragma unroll
      for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int p = 0; p < kMmas; ++p)
#pragma unroll
          for (int part = 0; part < 2; ++part) {
            const uint4 f = v[(((m * steps + s) * kMmas + p) * 2 + part) * 32 + lane];
#pragma unroll
            for (int b = 0; b < kB; ++b)
#pragma unroll
              for (int j = 0; j < 4; ++j) mma16816(acc[b][m][j], f.x, f.y, f.z, f.w, w[b][j][2 * p], w[b][j][2 * p + 1]);
          }
    }
#pragma unroll
    for (int b = 0; b < kB; ++b) {
      const int col = 32 * (blk + b * kAdWarps) + 8 * q;
      if (blk + b * kAdWarps >= b1) break;   // not this CTA's
      // an infinite element of B shows in every row of its column: hi times it is infinite, or NaN where hi is 0
      float odd[2] = {0.f, 0.f};
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int e = 0; e < 2; ++e) odd[e] = fmaf(acc[b][0][j][e], 0.f, odd[e]);
      if (odd[0] + odd[1] != 0.f) {
        float t[MT * 16];
#pragma unroll
        for (int i = 0; i < MT * 16; ++i) t[i] = acc[b][i >> 4][(i >> 2) & 3][i & 3];
        store_odd(L, t, sax, B, t0, nt, rank, col, MT);
        continue;
      }
#pragma unroll
      for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int r = 16 * m + 8 * h + g;
          if (r >= nt || col >= L.out_n) continue;
          uint16_t* dst = L.out + (t0 + r) * L.out_n + col;
          if (vec) {
            const uint32_t bw[4] = {base[b][m][h].x, base[b][m][h].y, base[b][m][h].z, base[b][m][h].w};
            uint32_t o[4];
#pragma unroll
            for (int j = 0; j < 4; ++j)
              o[j] = pack_bf16(bf16_lo(bw[j]) + acc[b][m][j][2 * h], bf16_hi(bw[j]) + acc[b][m][j][2 * h + 1]);
            *reinterpret_cast<uint4*>(dst) = make_uint4(o[0], o[1], o[2], o[3]);
          } else {
            const uint16_t* src = L.base + (t0 + r) * L.out_n + col;
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
              for (int e = 0; e < 2; ++e)
                if (col + 2 * j + e < L.out_n)
                  dst[2 * j + e] = (uint16_t)pack_bf16(bf16_lo(src[2 * j + e]) + acc[b][m][j][2 * h + e], 0.f);
          }
        }
    }
    __syncwarp();   // lanes may come from store_odd
  }
}

// CTAs of an SM: two where the partial sums (4 NT MT registers) leave room for it (2048 tokens of rank 16: 21 us; three,
// with fewer registers, 30; one of 512 threads 22)
constexpr int ad_per_sm(int NT, int MT) { return NT * MT <= 8 ? 2 : 1; }

// NT: n-tiles of 8 ranks held (rank <= 8 NT); MT: m-tiles of 16 tokens; CL: CTAs of a cluster
template <int NT, int MT, int CL>
__global__ void __launch_bounds__(kAdThreads, ad_per_sm(NT, MT)) __cluster_dims__(CL, 1, 1) k_adapters(const __grid_constant__ AdParams P) {
  extern __shared__ __align__(16) uint8_t ad_smem[];
  constexpr int M = 16 * MT;
  cg::cluster_group cluster = cg::this_cluster();
  start_of_work();
  const int c = (int)cluster.block_rank();
  const int u = (int)(blockIdx.x / CL);
  const AdLayer& L = P.layer[blockIdx.y];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, q = lane & 3;

  // Unit u is tile u - f(r) of request r, where f(r) = floor(offsets[r] / M) + r is the
  // request's first unit: f(r + 1) - f(r) is never below its ceil(len / M) tiles.
  int r = -1;
  for (int i0 = 0; i0 < P.n_seqs; i0 += kAdThreads) {
    const int i = i0 + (int)threadIdx.x;
    r += __syncthreads_count(i < P.n_seqs && __ldg(P.offsets + i) / M + i <= u);
  }
  if (r < 0) return;
  const int64_t first = max(0, __ldg(P.offsets + r)), end = min((int64_t)__ldg(P.offsets + r + 1), P.T);
  const int64_t t0 = first + (int64_t)(u - (int)(first / M) - r) * M;
  if (t0 < first || t0 >= end) return;   // the same for the whole cluster
  const int nt = (int)min((int64_t)M, end - t0);
  const int id = __ldg(P.ids + r);
  const int nb = (L.out_n + 31) / 32;
  const int b0 = c * nb / CL, b1 = (c + 1) * nb / CL;
  if (id < 0 || id >= L.n_adapters) {   // no adapter
    if (L.out != L.base) {
      const int64_t c0 = 32 * (int64_t)b0, n = min((int64_t)32 * b1, (int64_t)L.out_n) - c0;
      if ((L.out_n & 7) == 0) {
        const int64_t n8 = n / 8;
        for (int64_t i = threadIdx.x; i < n8 * nt; i += kAdThreads) {
          const int64_t at = (t0 + i / n8) * L.out_n + c0 + 8 * (i % n8);
          *reinterpret_cast<uint4*>(L.out + at) = *reinterpret_cast<const uint4*>(L.base + at);
        }
      } else if (n > 0) {
        for (int64_t i = threadIdx.x; i < n * nt; i += kAdThreads) {
          const int64_t at = (t0 + i / n) * L.out_n + c0 + i % n;
          L.out[at] = L.base[at];
        }
      }
    }
    return;
  }
  const int rank = L.rank, nrt = rank / 8;
  const uint16_t* A = L.A + (int64_t)id * rank * L.in;
  const uint16_t* B = L.B + (int64_t)id * rank * L.out_n;

  // ---- A x over this CTA's inputs: blocks of 32, taken by the warps in turn
  float acc[MT][NT][4];
#pragma unroll
  for (int m = 0; m < MT; ++m)
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[m][j][e] = 0.f;
  const int nk = (L.in + 31) / 32;
  const int k1 = (c + 1) * nk / CL;
  const uint4 zero = make_uint4(0u, 0u, 0u, 0u);
#pragma unroll 2
  for (int kb = c * nk / CL + warp; kb < k1; kb += kAdWarps) {
    const int k = min(32 * kb + 8 * q, L.in - 8);
    uint4 xa[MT][2], wa[NT];
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
      for (int h = 0; h < 2; ++h)
        xa[m][h] = __ldg(reinterpret_cast<const uint4*>(L.x + (t0 + min(16 * m + 8 * h + g, nt - 1)) * L.in + k));
#pragma unroll
    for (int j = 0; j < NT; ++j) wa[j] = __ldg(reinterpret_cast<const uint4*>(A + (int64_t)min(8 * j + g, rank - 1) * L.in + k));
    if (32 * kb + 32 > L.in && 32 * kb + 8 * q >= L.in) {   // the last block's lanes past the inputs
#pragma unroll
      for (int m = 0; m < MT; ++m) xa[m][0] = xa[m][1] = zero;
#pragma unroll
      for (int j = 0; j < NT; ++j) wa[j] = zero;
    }
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
      for (int j = 0; j < NT; ++j) {
        if (j >= nrt) break;
        mma16816(acc[m][j], xa[m][0].x, xa[m][1].x, xa[m][0].y, xa[m][1].y, wa[j].x, wa[j].y);
        mma16816(acc[m][j], xa[m][0].z, xa[m][1].z, xa[m][0].w, xa[m][1].w, wa[j].z, wa[j].w);
      }
  }
  // ---- sums over the warps, then over the cluster, each in a fixed order
  float* part = reinterpret_cast<float*>(ad_smem);   // [warps][M][rank]
  float* mine = part + (size_t)kAdWarps * M * rank;  // [M][rank] of this CTA
  float* sum = mine + (size_t)M * rank;              // [M][rank] of the cluster
  const int n = M * rank;
#pragma unroll
  for (int m = 0; m < MT; ++m)
#pragma unroll
    for (int j = 0; j < NT; ++j) {
      if (j >= nrt) break;
#pragma unroll
      for (int h = 0; h < 2; ++h)
        *reinterpret_cast<float2*>(part + (size_t)warp * n + (16 * m + 8 * h + g) * rank + 8 * j + 2 * q) =
            make_float2(acc[m][j][2 * h], acc[m][j][2 * h + 1]);
    }
  __syncthreads();
  for (int i = threadIdx.x; i < n; i += kAdThreads) {
    float s = 0.f;
#pragma unroll
    for (int w = 0; w < kAdWarps; ++w) s += part[(size_t)w * n + i];
    mine[i] = s;
  }
  cluster.sync();
  const float scale = __ldg(L.scale + id);
  {
    // CTA c sums its part of the elements and gives them to every CTA
    const int per = n / CL;   // n is a multiple of 128
    for (int i = c * per + (int)threadIdx.x; i < (c + 1) * per; i += kAdThreads) {
      float s = 0.f;
#pragma unroll
      for (int w = 0; w < CL; ++w) s += cluster.map_shared_rank(mine, w)[i];
      s *= scale;
#pragma unroll
      for (int w = 0; w < CL; ++w) cluster.map_shared_rank(sum, w)[i] = s;
    }
  }
  cluster.sync();
  // ---- s A x as hi + lo fragments of the second product (over the warps' partial sums)
  uint4* frag = reinterpret_cast<uint4*>(ad_smem);
  const int E = rank_elems(rank), steps = rank / (4 * E), mmas = E == 8 ? 2 : 1;
  for (int i = threadIdx.x; i < MT * steps * mmas * 32; i += kAdThreads) {
    const int ln = i & 31, p = (i >> 5) % mmas, s = (i >> 5) / mmas % steps, m = (i >> 5) / mmas / steps;
    uint32_t hi[4], lo[4];
#pragma unroll
    for (int f = 0; f < 4; ++f) {   // a0: row g, a1: row g + 8 of the first two elements; a2, a3: of the next two
      const int row = 16 * m + 8 * (f & 1) + (ln >> 2), e = 4 * p + 2 * (f >> 1);
      float v0 = 0.f, v1 = 0.f;
      if (e < E) {
        const float* src = sum + row * rank + s * 4 * E + (ln & 3) * E + e;
        v0 = src[0];
        v1 = src[1];
      }
      hi[f] = pack_bf16(v0, v1);
      // an infinity has no remainder
      const float h0 = bf16_lo(hi[f]), h1 = bf16_hi(hi[f]);
      lo[f] = pack_bf16(isinf(h0) ? 0.f : v0 - h0, isinf(h1) ? 0.f : v1 - h1);
    }
    uint4* dst = frag + (((m * steps + s) * mmas + p) * 2) * 32 + ln;
    dst[0] = make_uint4(hi[0], hi[1], hi[2], hi[3]);
    dst[32] = make_uint4(lo[0], lo[1], lo[2], lo[3]);
  }
  __syncthreads();
  if (E == 8) expand<MT, 8>(L, frag, sum, B, t0, nt, rank, b0, b1, warp, lane);
  else if (E == 4) expand<MT, 4>(L, frag, sum, B, t0, nt, rank, b0, b1, warp, lane);
  else expand<MT, 2>(L, frag, sum, B, t0, nt, rank, b0, b1, warp, lane);
}

template <int NT, int MT, int CL>
gs_status ad_launch(const AdParams& P, int n, int rank, cudaStream_t s) {
  constexpr int M = 16 * MT;
  // partial sums of the warps, this CTA's and the cluster's; the fragments (4 bytes an
  // element and part, padded to whole MMAs for odd multiples of 8) overlay the first
  const size_t smem = (size_t)(kAdWarps + 2) * M * rank * 4;
  constexpr size_t kMost = (size_t)(kAdWarps + 2) * M * (8 * NT) * 4;
  static const cudaError_t attr =
      cudaFuncSetAttribute(k_adapters<NT, MT, CL>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kMost);
  if (attr != cudaSuccess) return GS_ERR_CUDA;
  const int64_t units = P.T / M + P.n_seqs;
  if (units * CL > INT32_MAX) return GS_ERR_UNSUPPORTED;
  return launch_behind(k_adapters<NT, MT, CL>, dim3((unsigned)(units * CL), (unsigned)n), kAdThreads, smem, s, P);
}

// The largest cluster with which all tiles are resident at once: more CTAs a tile shorten
// it as long as they do not queue (us at 8 / 4 / 2: 51 tiles of rank 16  10.7 / 7.8 / 9.7,
// 70 tiles of rank 32  34 / 29 / 44, 17 tiles of rank 64  15 / 23 / 41).
template <int NT, int MT>
gs_status ad_cluster(const AdParams& P, int n, int rank, cudaStream_t s) {
  const int64_t tiles = (P.T / (16 * MT) + P.n_seqs) * n, room = (int64_t)sm_count() * ad_per_sm(NT, MT);
  if (tiles * 8 <= room) return ad_launch<NT, MT, 8>(P, n, rank, s);
  return tiles * 4 <= room ? ad_launch<NT, MT, 4>(P, n, rank, s) : ad_launch<NT, MT, 2>(P, n, rank, s);
}

}  // namespace

gs_status launch_adapters(const gs_adapter_layer* layers, int n, const int32_t* offsets, const int32_t* ids, int32_t n_seqs,
                          int64_t T, cudaStream_t s) {
  AdParams P;
  P.offsets = offsets;
  P.ids = ids;
  P.T = T;
  P.n_seqs = n_seqs;
  int rank = 0;
  for (int i = 0; i < n; ++i) {
    AdLayer& L = P.layer[i];
    L.x = static_cast<const uint16_t*>(layers[i].x_dev);
    L.base = static_cast<const uint16_t*>(layers[i].base_dev);
    L.out = static_cast<uint16_t*>(layers[i].out_dev);
    L.A = static_cast<const uint16_t*>(layers[i].A_dev);
    L.B = static_cast<const uint16_t*>(layers[i].B_dev);
    L.scale = layers[i].scale_dev;
    L.in = (int32_t)layers[i].in;
    L.out_n = (int32_t)layers[i].out;
    L.n_adapters = layers[i].n_adapters;
    L.rank = layers[i].rank;
    rank = rank > L.rank ? rank : L.rank;
  }
  // 32 tokens a tile where the mean request has at least 64 (us at 16 / 32 a tile; 4096x11008 but where said otherwise):
  //   rank 16 and 32    6 requests of 2048 tokens  29.5 / 21.2 and 34.9 / 26.8,  12 x 64 (4096x4096, rank 16)  11.7 / 10.6
  //   below, rank 32    16 x 48 tokens  19.7 / 24.1,  8 x 48  13.1 / 15.9,  8 x 32  12.9 / 14.6
  //   rank 128          2048 tokens  101 / 77;  rank 64: 41.4 / 50.1, its sums leave no second CTA an SM: always 16
  // (64 a tile: 34 at rank 16, 53 at 32, 79 at 64.)
  const bool longer = T >= (int64_t)64 * n_seqs;
  if (rank <= 16) return longer ? ad_cluster<2, 2>(P, n, rank, s) : ad_cluster<2, 1>(P, n, rank, s);
  if (rank <= 32) return longer ? ad_cluster<4, 2>(P, n, rank, s) : ad_cluster<4, 1>(P, n, rank, s);
  if (rank <= 64) return ad_cluster<8, 1>(P, n, rank, s);
  return longer ? ad_cluster<16, 2>(P, n, rank, s) : ad_cluster<16, 1>(P, n, rank, s);
}

}  // namespace gs
