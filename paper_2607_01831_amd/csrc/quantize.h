// Arithmetic of the uniform 8-bit codec shared by its kernels (gfx950): group
// parameters, codes, the 4 + 4 split, and the rounding of a read-back value.
// The fp32 arithmetic that decides a code is spelled out operation by
// operation (sub, mul, round-half-even, clamp; one IEEE division per group)
// so that every code is the one the definition gives, whichever kernel
// computes it.
#pragma once

#include <float.h>
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace lynx {

__device__ __forceinline__ float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }

// Eight BF16 values held in a uint4 -> floats.
__device__ __forceinline__ void unpack8(const uint4 &u, float *x) {
    x[0] = bf16_lo(u.x); x[1] = bf16_hi(u.x);
    x[2] = bf16_lo(u.y); x[3] = bf16_hi(u.y);
    x[4] = bf16_lo(u.z); x[5] = bf16_hi(u.z);
    x[6] = bf16_lo(u.w); x[7] = bf16_hi(u.w);
}

// Group statistics from the group's min and max: zero, scale, inverse range.
__device__ __forceinline__ void group_params(float mn, float mx, float &zero, float &scale,
                                             float &inv) {
    if (mn == 0.0f) mn = 0.0f;  // -0 -> +0
    if (mx == 0.0f) mx = 0.0f;
    const float range = mx - mn;
    const float r = 255.0f / range;  // correctly rounded IEEE division
    if (!(range > 0.0f) || !(range <= FLT_MAX) || !(r <= FLT_MAX)) {
        scale = 0.0f;
        inv = 0.0f;
    } else {
        scale = range / 255.0f;
        inv = r;
    }
    zero = mn;
}

// (Min / max and the cross-lane reductions come from lane_ops.h; non-finite
// inputs give unspecified codes.)

// Eight values -> eight codes clamp(rint((x - zero) * inv), 0, 255), then
// the anchor word (nibble j = code_j >> 4) and the residual word (nibble j =
// code_j & 15).  v_cvt_pk_u8_f32 rounds half to even and saturates to
// [0, 255] (NaN -> 0), which is exactly the clamp-of-rint of the definition.
__device__ __forceinline__ void quantize_split8(const float *x, const float *zero, const float *inv,
                                                uint32_t &anc, uint32_t &res) {
    uint32_t w[2] = {0u, 0u};
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const float y = (x[j] - zero[j]) * inv[j];
        w[j >> 2] = __builtin_amdgcn_cvt_pk_u8_f32(y, (uint32_t)(j & 3), w[j >> 2]);
    }
    // bytes (c0, c1, c2, c3) -> nibble pairs c0 | c1 << 4 in byte 0, c2 | c3 << 4 in byte 2
    const uint32_t a0 = (w[0] >> 4) & 0x0F0F0F0Fu, a1 = (w[1] >> 4) & 0x0F0F0F0Fu;
    const uint32_t r0 = w[0] & 0x0F0F0F0Fu, r1 = w[1] & 0x0F0F0F0Fu;
    anc = __builtin_amdgcn_perm(a1 | (a1 >> 4), a0 | (a0 >> 4), 0x06040200u);
    res = __builtin_amdgcn_perm(r1 | (r1 >> 4), r0 | (r0 >> 4), 0x06040200u);
}

typedef unsigned int u32v4 __attribute__((ext_vector_type(4)));

// Eight values -> eight codes (bytes 0..7 of the result), as quantize_split8.
__device__ __forceinline__ uint64_t quantize8(const float *x, const float *zero, const float *inv) {
    uint32_t w[2] = {0u, 0u};
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const float y = (x[j] - zero[j]) * inv[j];
        w[j >> 2] = __builtin_amdgcn_cvt_pk_u8_f32(y, (uint32_t)(j & 3), w[j >> 2]);
    }
    return (uint64_t)w[0] | ((uint64_t)w[1] << 32);
}

__device__ __forceinline__ uint32_t f32_to_bf16_bits(float f) {
    const uint32_t u = __float_as_uint(f);
    if ((u & 0x7F800000u) == 0x7F800000u && (u & 0x007FFFFFu)) return (u >> 16) | 0x40u;
    return (u + 0x7FFFu + ((u >> 16) & 1u)) >> 16;
}

}  // namespace lynx
