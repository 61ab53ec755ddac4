// What the attention kernels of both directions share: tile geometry, stores of a lane's head-dim elements, reductions over the
// lanes of a query (internal).
#pragma once

#include "common.h"
#include "mfma_lds.h"

namespace ragged {

constexpr int kHeadDim = 64;
constexpr int kBN = 64;                 // rows per tile of one operand
constexpr int kTileBytes = kBN * kHeadDim * 2;   // one tile of one operand: 8 KB
constexpr float kLog2e = 1.4426950408889634f;
constexpr int kMaxGridYZ = 65535;       // HIP's limit on the second and third grid dimension

// Store 16 consecutive head-dim elements of one output row.
__device__ __forceinline__ void store16(_Float16* dst, const float (&v)[16]) {
    f16x8 a, b;
#pragma unroll
    for (int e = 0; e < 8; ++e) { a[e] = (_Float16)v[e]; b[e] = (_Float16)v[8 + e]; }
    reinterpret_cast<uint4*>(dst)[0] = __builtin_bit_cast(uint4, a);
    reinterpret_cast<uint4*>(dst)[1] = __builtin_bit_cast(uint4, b);
}
__device__ __forceinline__ void store16(__bf16* dst, const float (&v)[16]) {
    bf16x8 a, b;
#pragma unroll
    for (int e = 0; e < 8; ++e) { a[e] = (__bf16)v[e]; b[e] = (__bf16)v[8 + e]; }
    reinterpret_cast<uint4*>(dst)[0] = __builtin_bit_cast(uint4, a);
    reinterpret_cast<uint4*>(dst)[1] = __builtin_bit_cast(uint4, b);
}
__device__ __forceinline__ void store16(float* dst, const float (&v)[16]) {
#pragma unroll
    for (int e = 0; e < 4; ++e)
        reinterpret_cast<float4*>(dst)[e] = make_float4(v[4 * e], v[4 * e + 1], v[4 * e + 2], v[4 * e + 3]);
}

// Store 4 consecutive head-dim elements of one output row.
__device__ __forceinline__ void store4(_Float16* dst, const float (&v)[4]) {
    typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));
    const f16x4 a = {(_Float16)v[0], (_Float16)v[1], (_Float16)v[2], (_Float16)v[3]};
    *reinterpret_cast<uint2*>(dst) = __builtin_bit_cast(uint2, a);
}
__device__ __forceinline__ void store4(__bf16* dst, const float (&v)[4]) {
    typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
    const bf16x4 a = {(__bf16)v[0], (__bf16)v[1], (__bf16)v[2], (__bf16)v[3]};
    *reinterpret_cast<uint2*>(dst) = __builtin_bit_cast(uint2, a);
}
__device__ __forceinline__ void store4(float* dst, const float (&v)[4]) {
    *reinterpret_cast<float4*>(dst) = make_float4(v[0], v[1], v[2], v[3]);
}

// Reductions over the four lanes that share a query (l, l^16, l^32, l^48) with the gfx950 lane-swap
// instructions (pure VALU, no LDS round trip).  permlane32_swap(a, b) returns {a.lo|b.lo, a.hi|b.hi}
// (32-lane halves); permlane16_swap(a, b) returns {a.row0,b.row0,a.row2,b.row2} and
// {a.row1,b.row1,a.row3,b.row3} (16-lane rows).  With b a copy of a, combining the two results
// reduces across the halves, then across the rows.  The copy is made through an opaque move so the
// two operands can never be folded into one register (the instruction swaps its operands in place).
__device__ __forceinline__ unsigned opaque_copy(unsigned x) {
    unsigned y;
    asm volatile("v_mov_b32 %0, %1" : "=v"(y) : "v"(x));
    return y;
}
__device__ __forceinline__ float as_f32(unsigned u) { return __builtin_bit_cast(float, u); }
__device__ __forceinline__ unsigned as_u32(float f) { return __builtin_bit_cast(unsigned, f); }
__device__ __forceinline__ float quad_max(float x) {
    const auto a = __builtin_amdgcn_permlane32_swap(as_u32(x), opaque_copy(as_u32(x)), false, false);
    const unsigned a0 = a[0], a1 = a[1];
    x = fmaxf(as_f32(a0), as_f32(a1));
    const auto b = __builtin_amdgcn_permlane16_swap(as_u32(x), opaque_copy(as_u32(x)), false, false);
    const unsigned b0 = b[0], b1 = b[1];
    return fmaxf(as_f32(b0), as_f32(b1));
}
__device__ __forceinline__ float quad_sum(float x) {
    const auto a = __builtin_amdgcn_permlane32_swap(as_u32(x), opaque_copy(as_u32(x)), false, false);
    const unsigned a0 = a[0], a1 = a[1];
    x = as_f32(a0) + as_f32(a1);
    const auto b = __builtin_amdgcn_permlane16_swap(as_u32(x), opaque_copy(as_u32(x)), false, false);
    const unsigned b0 = b[0], b1 = b[1];
    return as_f32(b0) + as_f32(b1);
}

}  // namespace ragged
