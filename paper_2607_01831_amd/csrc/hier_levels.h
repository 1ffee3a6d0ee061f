// The levels of the hierarchical codec's codes (Alg. 1; hier.hip), shared by the
// kernels that read them.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "lynx_internal.h"

namespace lynx {

// The signed code of an anchor nibble qa alone (FULL 0), or with the correction
// nibble qr: its sign, and the place on the transform's axis in units of one code.
// Biased: code 16 V, or 16 V - Q_res; centred: the bucket's centre 16 V + 7.5, or
// 16 V + 8 + Q_res; 4-bit: V.
struct SignedCode {
    float code;
    bool negative;
};
template <int FULL>
__device__ __forceinline__ SignedCode signed_code(int variant, uint32_t qa, uint32_t qr) {
    const bool neg = qa >= 8;
    const int V = neg ? 15 - (int)qa : (int)qa;  // sign-aware: -V - 1 in two's complement
    const int r = qr >= 8 ? (int)qr - 16 : (int)qr;
    if (variant == kHBiased) return {(float)min(max(16 * V - (FULL ? r : 0), 0), 127), neg};
    if (variant == kHCentred) return {FULL ? (float)(16 * V + 8 + r) : 16.0f * V + 7.5f, neg};
    return {(float)V, neg};
}

// The signed level as fp16: expm1(code / M log1p(alpha)) / alpha, 0 .. 1, rounded to
// nearest (2^-11 of itself; by 2^-25 below 2^-14).  log1p_alpha is rounded
// from double on the host; a tiny alpha takes the first two terms of the series,
// where expm1's argument would be a denormal.
template <int FULL>
__device__ __forceinline__ _Float16 signed_level_f16(float alpha, float log1p_alpha, int variant, uint32_t qa,
                                                     uint32_t qr) {
    const SignedCode c = signed_code<FULL>(variant, qa, qr);
    const float x = c.code / (variant == kHInt4 ? 7.0f : 127.0f);
    const float lv = alpha < 1e-4f ? fmaf(0.5f * alpha * x, x - 1.0f, x) : expm1f(x * log1p_alpha) / alpha;
    return (_Float16)(c.negative ? -lv : lv);
}

}  // namespace lynx
