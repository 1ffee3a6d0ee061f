// Norms of the query and key heads with the position rotation in the same pass
// (gfx950): from the rows of the projections to the rows that attention, the
// verification and the append read.
//
// What it computes, per token and head of 128 dims: y = x rsqrt(mean(x^2) + eps) w
// (Q and K, each with its own weights, or y = x), then pairs of the first `rotary`
// dims turned by the angle position * inv_freq[i]; V is moved as it is.  fp32
// throughout, rounded to BF16 once.
//
// It is bound by memory: every byte is read once and written once.  16 lanes hold a
// head, 8 dims (16 bytes) each, so the mean is four DPP additions.  The angles are
// a token's, not a head's: a workgroup computes the cosines and sines of its tokens
// once, a pair a thread, and the lanes keep those of their 8 dims for all of a
// token's heads.  The angle is taken in turns in double precision and reduced there
// (a position of 2^31 turns by 1e-7 of a turn too much at most), its sine and
// cosine in fp32.
#include "lane_ops.h"
#include "lynx_internal.h"

namespace lynx {
namespace {

constexpr int kThreads = 256;
constexpr int kHeads = kThreads / 16;  // heads that a workgroup holds at once

__device__ __forceinline__ float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }
typedef float f32x2_t __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t pack2(float a, float b) {
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2_t){a, b}, bf16x2_t));
}
__device__ __forceinline__ void unpack8(const uint4 &u, float *x) {
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[2 * i] = bf16_lo(w[i]);
        x[2 * i + 1] = bf16_hi(w[i]);
    }
}

// Where the other half of a lane's pairs is: in the lane itself (neighbouring
// dims), or rotary / 2 dims away, a whole number of lanes: 8 of 16, or any.
enum Pairs { kNeighbours, kHalves64, kHalves };

__device__ __forceinline__ uint32_t swap_halves(uint32_t v) {  // with lane ^ 8 of the row of 16
    return (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x128, 0xF, 0xF, false);  // row_ror:8
}
template <Pairs PAIRS>
__device__ __forceinline__ uint4 partner(const uint4 &u, int from) {
    if (PAIRS == kNeighbours)
        return make_uint4(u.x << 16 | u.x >> 16, u.y << 16 | u.y >> 16, u.z << 16 | u.z >> 16, u.w << 16 | u.w >> 16);
    if (PAIRS == kHalves64) return make_uint4(swap_halves(u.x), swap_halves(u.y), swap_halves(u.z), swap_halves(u.w));
    return make_uint4(__shfl(u.x, from), __shfl(u.y, from), __shfl(u.z, from), __shfl(u.w, from));
}

// Workgroup: TOKENS tokens, all their heads (gridDim.y 1) or every gridDim.y-th
// group of 16.  The heads of a token: Q, K, V.
template <Pairs PAIRS, int TOKENS>
__global__ __launch_bounds__(kThreads) void rope_kernel(RopeArgs a) {
    // by dim: cosine, and sine with the sign that its partner enters with
    __shared__ __attribute__((aligned(16))) float s_cos[TOKENS][kHeadDim], s_sin[TOKENS][kHeadDim];
    const int tid = threadIdx.x, lane = tid & 63, c = tid & 15;
    const int n0 = blockIdx.x * TOKENS;
    const int half = a.rotary / 2;
    for (int i = tid; i < TOKENS * (kHeadDim / 2); i += kThreads) {
        const int tok = i / (kHeadDim / 2), p = i % (kHeadDim / 2);
        float co = 1.0f, si = 0.0f;
        int d0 = 2 * p, d1 = 2 * p + 1;  // the pair's dims; those past `rotary` stay as they are
        if (p < half) {
            const int pos = a.positions[min(n0 + tok, a.n_tokens - 1)];
            double turns = (double)pos * ((double)a.inv_freq[p] * 0.15915494309189535);
            turns -= rint(turns);
            sincospif(2.0f * (float)turns, &si, &co);
            co *= a.scale;
            si *= a.scale;
            if (PAIRS != kNeighbours) {
                d0 = p;
                d1 = p + half;
            }
        }
        s_cos[tok][d0] = co;
        s_cos[tok][d1] = co;
        s_sin[tok][d0] = -si;
        s_sin[tok][d1] = si;
    }
    // the lane that holds the partners of this lane's dims
    int from = lane;
    if (PAIRS == kHalves && 8 * c < a.rotary) from = 8 * c < half ? lane + half / 8 : lane - half / 8;
    float wq[8], wk[8], pq[8], pk[8];  // weights of the lane's dims and of their partners
    {
        const uint4 one = make_uint4(0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u);
        const uint4 q = a.q_weight ? reinterpret_cast<const uint4 *>(a.q_weight)[c] : one;
        const uint4 k = a.k_weight ? reinterpret_cast<const uint4 *>(a.k_weight)[c] : one;
        unpack8(q, wq);
        unpack8(k, wk);
        unpack8(partner<PAIRS>(q, from), pq);
        unpack8(partner<PAIRS>(k, from), pk);
    }
    __syncthreads();
    const int heads = a.Hq + a.Hkv + (a.v ? a.Hkv : 0);
#pragma unroll 1
    for (int tok = 0; tok < TOKENS; ++tok) {
        const int n = n0 + tok;
        if (n >= a.n_tokens) break;
        const int pos = a.positions[n];
        const int64_t row = a.rows ? a.rows[n] : n;
        if (pos < 0 || row < 0 || row >= a.n_rows) continue;
        float co[8], si[8];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const float4 x = reinterpret_cast<const float4 *>(s_cos[tok])[2 * c + i];
            const float4 y = reinterpret_cast<const float4 *>(s_sin[tok])[2 * c + i];
            co[4 * i] = x.x; co[4 * i + 1] = x.y; co[4 * i + 2] = x.z; co[4 * i + 3] = x.w;
            si[4 * i] = y.x; si[4 * i + 1] = y.y; si[4 * i + 2] = y.z; si[4 * i + 3] = y.w;
        }
        for (int h0 = kHeads * blockIdx.y; h0 < heads; h0 += kHeads * gridDim.y) {
            const int h = h0 + (tid >> 4);
            const bool is_q = h < a.Hq, is_v = h >= a.Hq + a.Hkv;
            const int own = is_q ? h : is_v ? h - a.Hq - a.Hkv : h - a.Hq;
            const uint16_t *src = is_q ? a.q + (size_t)n * a.q_stride : is_v ? a.v + (size_t)n * a.v_stride : a.k + (size_t)n * a.k_stride;
            uint16_t *dst = is_q ? a.q_out + (size_t)row * a.Hq * kHeadDim : (is_v ? a.v_out : a.k_out) + (size_t)row * a.Hkv * kHeadDim;
            const bool live = h < heads;
            const uint4 u = live ? reinterpret_cast<const uint4 *>(src + (size_t)own * kHeadDim)[c] : make_uint4(0u, 0u, 0u, 0u);
            const uint4 pu = partner<PAIRS>(u, from);
            float x[8], p[8];
            unpack8(u, x);
            unpack8(pu, p);
            float ss = 0.0f;
#pragma unroll
            for (int i = 0; i < 8; ++i) ss = fmaf(x[i], x[i], ss);
            ss = row16_sum(ss);
            const bool normed = is_q ? a.q_weight != nullptr : a.k_weight != nullptr;
            const float r = normed ? 1.0f / sqrtf(ss * (1.0f / kHeadDim) + a.eps) : 1.0f;
            uint32_t o[4];
#pragma unroll
            for (int i = 0; i < 8; i += 2) {
                float y[2];
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const float xw = x[i + k] * r * (is_q ? wq[i + k] : wk[i + k]);
                    const float pw = p[i + k] * r * (is_q ? pq[i + k] : pk[i + k]);
                    // (a dim past `rotary` is its own partner's no one: cosine 1, no product with an infinity)
                    y[k] = 8 * c < a.rotary ? fmaf(pw, si[i + k], xw * co[i + k]) : xw;
                }
                o[i / 2] = pack2(y[0], y[1]);
            }
            if (live)
                reinterpret_cast<uint4 *>(dst + (size_t)own * kHeadDim)[c] = is_v ? u : make_uint4(o[0], o[1], o[2], o[3]);
        }
    }
}

template <Pairs PAIRS>
void launch_pairs(const RopeArgs &a, hipStream_t stream) {
    const int heads = a.Hq + a.Hkv + (a.v ? a.Hkv : 0), groups = (heads + kHeads - 1) / kHeads;
    if (a.n_tokens >= 2048)
        hipLaunchKernelGGL((rope_kernel<PAIRS, 4>), dim3((a.n_tokens + 3) / 4), dim3(kThreads), 0, stream, a);
    else
        hipLaunchKernelGGL((rope_kernel<PAIRS, 1>), dim3(a.n_tokens, groups), dim3(kThreads), 0, stream, a);
}

}  // namespace

hipError_t launch_rope(const RopeArgs &a, hipStream_t stream) {
    if (a.n_tokens <= 0) return hipSuccess;
    if (a.pairs)
        launch_pairs<kNeighbours>(a, stream);
    else if (a.rotary == kHeadDim)
        launch_pairs<kHalves64>(a, stream);
    else
        launch_pairs<kHalves>(a, stream);
    return hipGetLastError();
}

}  // namespace lynx
