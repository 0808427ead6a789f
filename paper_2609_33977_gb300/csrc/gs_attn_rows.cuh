// What the two kernels for few rows share: their most rows, the room of a row of a part, and loads of fragments.
// A part is [rows][D], then [rows][kPartPad] with maximum and sum (over 8 bits the numerators' maximum too), the rest zeros:
// a 32-byte sector that is written in part costs whoever reads it a fill from HBM.
#pragma once

#include "gs_attn.cuh"

namespace gs {

constexpr int kMost = 32;      // rows
constexpr int kPartPad = 8;    // floats of a row of a part beside the output's

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
}  // namespace gs
