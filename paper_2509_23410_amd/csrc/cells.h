// Cells of a paged cache and rows of products: loads of four values as fp32, stores of four values rounded once.
#pragma once
#include "seqs.h"

namespace patch {

typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));

struct Four { float x[4]; };

__device__ __forceinline__ float bf16_lo(uint32_t u) { return __uint_as_float(u << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t u) { return __uint_as_float(u & 0xFFFF0000u); }

// element i (a multiple of 4) of a row of fp32 or bf16
__device__ __forceinline__ Four load4(const uint8_t* row, int i, int f32) {
    Four r;
    if (f32) {
        const ep_f32x4 v = *reinterpret_cast<const PATCH_EP_GLOBAL ep_f32x4*>(as_global(row) + 4 * i);
        r = {{v[0], v[1], v[2], v[3]}};
    } else {
        const u32x2_t v = *reinterpret_cast<const PATCH_EP_GLOBAL u32x2_t*>(as_global(row) + 2 * i);
        r = {{bf16_lo(v[0]), bf16_hi(v[0]), bf16_lo(v[1]), bf16_hi(v[1])}};
    }
    return r;
}

__device__ __forceinline__ u32x2_t pack_bf16(const Four& v) { return u32x2_t{bf16_pair(v.x[0], v.x[1]), bf16_pair(v.x[2], v.x[3])}; }

// e4m3 (the one with no infinities), nearest, ties to even; what is beyond 448 becomes 448, a NaN stays one
__device__ __forceinline__ float e4m3_range(float x) { return x > 448.f ? 448.f : x < -448.f ? -448.f : x; }
__device__ __forceinline__ uint32_t pack_e4m3(const Four& v, float scale) {
    int u = 0;
    u = __builtin_amdgcn_cvt_pk_fp8_f32(e4m3_range(v.x[0] / scale), e4m3_range(v.x[1] / scale), u, false);
    u = __builtin_amdgcn_cvt_pk_fp8_f32(e4m3_range(v.x[2] / scale), e4m3_range(v.x[3] / scale), u, true);
    return (uint32_t)u;
}

}  // namespace patch
