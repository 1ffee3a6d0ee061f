// The hierarchical codec's codes (Alg. 1; hier.hip) as matrix operands: the levels'
// table, the maps of a chunk, the scales of operands (hier_attn.hip).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "f16_ops.h"
#include "lane_ops.h"
#include "lynx_internal.h"
#include "split_merge.h"

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
// nearest (2^-11 of itself, or by 2^-25 below 2^-14: the smallest codes of an alpha of
// 1000 and more).  log1p_alpha is rounded from double on the host; a tiny alpha takes
// the first two terms of the series, where expm1's argument would be a denormal.
template <int FULL>
__device__ __forceinline__ _Float16 signed_level_f16(float alpha, float log1p_alpha, int variant, uint32_t qa,
                                                     uint32_t qr) {
    const SignedCode c = signed_code<FULL>(variant, qa, qr);
    const float x = c.code / (variant == kHInt4 ? 7.0f : 127.0f);
    const float lv = alpha < 1e-4f ? fmaf(0.5f * alpha * x, x - 1.0f, x) : expm1f(x * log1p_alpha) / alpha;
    return (_Float16)(c.negative ? -lv : lv);
}

// ---- the table of levels ----
// 64 copies of 256 entries by plane byte, entry e of lane l at 256 e + 4 l, so a
// lookup's address is the plane byte over the lane's byte, one v_perm, and every lane
// reads a bank of its own.  The entry of a byte of two nibbles is the pair of their
// levels, of a byte of one code its level twice.
constexpr int kTableBytes = 256 * 256;
constexpr int kHierChunk = 32;   // tokens of a codec chunk
constexpr int kHierPage = 256;   // tokens of a codec page

// Made by a workgroup of 256; a barrier stands between this and the first lookup.
template <int FULL>
__device__ __forceinline__ void fill_table(const HierArgs &a, uint8_t *table) {
    const int byte = threadIdx.x;
    uint32_t entry;
    if (FULL) {
        const uint32_t x =
            __builtin_bit_cast(uint16_t, signed_level_f16<1>(a.alpha, a.log1p_alpha, a.variant, byte >> 4, byte & 15));
        entry = x | x << 16;
    } else {
        entry = __builtin_bit_cast(uint16_t, signed_level_f16<0>(a.alpha, a.log1p_alpha, a.variant, byte & 15, 0)) |
                (uint32_t)__builtin_bit_cast(uint16_t, signed_level_f16<0>(a.alpha, a.log1p_alpha, a.variant, byte >> 4, 0)) << 16;
    }
    // rows of 64 copies, 16 bytes a lane; a wavefront's rows are its lanes' entries
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
        const int from = 4 * r + (lane >> 4);
        const uint32_t x = __shfl(entry, from);
        *reinterpret_cast<uint4 *>(table + (size_t)(byte - lane + from) * 256 + 16 * (lane & 15)) = make_uint4(x, x, x, x);
    }
}
// The entry of byte `by` of a word of the planes; lane4: the lane's byte.
__device__ __forceinline__ uint32_t look_up(const uint8_t *table, uint32_t word, int by, uint32_t lane4) {
    return *reinterpret_cast<const uint32_t *>(table + __builtin_amdgcn_perm(word, lane4, 0x0c0c0400u + ((uint32_t)by << 8)));
}

// ---- operands ----
__device__ __forceinline__ uint32_t pk_fma(uint32_t a, uint32_t b, uint32_t c) {
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_fma(__builtin_bit_cast(f16x2_t, a),
                                                                  __builtin_bit_cast(f16x2_t, b),
                                                                  __builtin_bit_cast(f16x2_t, c)));
}
__device__ __forceinline__ uint32_t low16s(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x05040100u); }
__device__ __forceinline__ uint32_t high16s(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x07060302u); }
// Largest of a non-negative value over the wavefront, uniform; a NaN may be lost.
__device__ __forceinline__ float wave_max(float v) { return row_max<64>(v); }
// The largest |b| + |m| of the scaled K and V, and the largest |q|: products up to
// 2^24, sums in fp32.
constexpr int kKvTop = 14, kQTop = 10;
// A softmax weight is exp2(score - reference + kPTop); the reference moves when a
// score passes it by kSlack, so weights stay below 2^(kPTop + kSlack) < 65504.
constexpr int kPTop = 7, kSlack = 8;
// The exponent e with x < 2^e (x >= 0), kept where 2^(kKvTop - e) is a normal float.
constexpr int kLeast = -112;
__device__ __forceinline__ int exponent_of(float x) { return max((int)(__float_as_uint(x) >> 23) - 126, kLeast); }

// The maps x = level b + m of two channels, K's and V's, from their scalars: sigma,
// mu, gscale, gmin of K, then of V.
struct Maps {
    float2 kb, km, vb, vm;
    float k_top, v_top;  // the larger |b| + |m| of the two
};
__device__ __forceinline__ Maps maps_of(const float2 *s) {
    Maps r;
    r.kb = make_float2(s[0].x * s[2].x, s[0].y * s[2].y);
    r.km = make_float2(fmaf(s[1].x, s[2].x, s[3].x), fmaf(s[1].y, s[2].y, s[3].y));
    r.vb = make_float2(s[4].x * s[6].x, s[4].y * s[6].y);
    r.vm = make_float2(fmaf(s[5].x, s[6].x, s[7].x), fmaf(s[5].y, s[6].y, s[7].y));
    r.k_top = fmaxf(fabsf(r.kb.x) + fabsf(r.km.x), fabsf(r.kb.y) + fabsf(r.km.y));
    r.v_top = fmaxf(fabsf(r.vb.x) + fabsf(r.vm.x), fabsf(r.vb.y) + fabsf(r.vm.y));
    return r;
}
// A wavefront's stage of them, [128] fp16 each: K's b, m, V's b, m.
constexpr int kStageBytes = 1024;
__device__ __forceinline__ void stage_maps(const Maps &x, int e_k, int e_v, int lane, uint8_t *stage) {
    const float sk = ldexpf(1.0f, kKvTop - e_k), sv = ldexpf(1.0f, kKvTop - e_v);
    uint32_t *st = reinterpret_cast<uint32_t *>(stage) + lane;
    st[0] = pack_f16_rne(x.kb.x * sk, x.kb.y * sk);
    st[64] = pack_f16_rne(x.km.x * sk, x.km.y * sk);
    st[128] = pack_f16_rne(x.vb.x * sv, x.vb.y * sv);
    st[192] = pack_f16_rne(x.vm.x * sv, x.vm.y * sv);
}

}  // namespace lynx
