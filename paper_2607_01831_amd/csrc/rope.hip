// Norms of the query and key heads with the position rotation in the same pass
// (gfx950): from the rows of the projections to the rows that attention, the
// verification and the append read.
//
// What it computes, per token and head of 128 dims: y = x rsqrt(mean(x^2) + eps) w
// (Q and K, each with its own weights, or y = x), then pairs of the first `rotary`
// dims turned by the angle position * inv_freq[i]; V is moved as it is.  fp32
// throughout, rounded to BF16 once.
//
// It is bound by memory: every byte is read once and written once (16384 tokens of
// 32 + 8 + 8 heads 73.7 us, 403 MB, 5.5 TB/s; a large copy 5.1); a call of few tokens
// by one launch's latency, 4.0 us with the host's.  16 lanes hold a head, 8 dims (16
// bytes) each, so the mean is four DPP additions, and a pair's other half comes from
// its lane by one more, normed.  A workgroup takes 16 heads of a token: 64 threads
// compute the token's cosines and sines while the heads' rows are on their way.
// Tokens two and four to a workgroup need fewer angles and were slower: before pairs
// were exchanged normed (each lane then made its partners' too), 2048 tokens took 12.9
// us, so 15.1 and 15.4; 16384 79.4, so 78.0 and 79.3; now 12.6 and 75.3.
// The angle is taken in turns in double precision and reduced there (a position of
// 2^31 turns by 1e-7 of a turn too much at most), its sine and cosine in fp32.
#include "lane_ops.h"
#include "lynx_internal.h"

namespace lynx {
namespace {

constexpr int kThreads = 256;
constexpr int kHeads = kThreads / 16;  // heads that a workgroup takes
constexpr int kGridTokens = 65535;     // tokens along the grid's second axis

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

template <Pairs PAIRS>
__device__ __forceinline__ float partner(const float *x, int i, int from) {
    if (PAIRS == kNeighbours) return x[i ^ 1];
    if (PAIRS == kHalves64)  // lane ^ 8 of the row of 16: row_ror:8
        return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(x[i]), 0x128, 0xF, 0xF, false));
    return __shfl(x[i], from);
}
// Where dim d's cosine and sine are: so that the 16 lanes of a head read 256 bytes in a
// row, twice.
__device__ __forceinline__ int place(int d) { return ((d & 4) << 4) | ((d >> 3) << 2) | (d & 3); }

// Workgroup (heads / 16, tokens, tokens / 65535): 16 heads of a token, which has its Q,
// K and V heads in that order.
template <Pairs PAIRS>
__global__ __launch_bounds__(kThreads) void rope_kernel(RopeArgs a) {
    // by dim: cosine, and sine with the sign that its partner enters with
    __shared__ __attribute__((aligned(16))) float s_cos[kHeadDim], s_sin[kHeadDim];
    const int tid = threadIdx.x, lane = tid & 63, c = tid & 15;
    const int64_t n = (int64_t)blockIdx.z * kGridTokens + blockIdx.y;
    if (n >= a.n_tokens) return;
    const int pos = a.positions[n];
    const int64_t row = a.rows ? a.rows[n] : n;
    const int half = a.rotary / 2;
    const int h = kHeads * (int)blockIdx.x + (tid >> 4);
    const bool live = h < a.Hq + a.Hkv + (a.v ? a.Hkv : 0), is_q = h < a.Hq, is_v = h >= a.Hq + a.Hkv;
    const int own = is_q ? h : is_v ? h - a.Hq - a.Hkv : h - a.Hq;
    const int64_t stride = is_q ? a.q_stride : is_v ? a.v_stride : a.k_stride;
    const uint16_t *src = (is_q ? a.q : is_v ? a.v : a.k) + (size_t)own * kHeadDim;
    const uint4 u = live ? reinterpret_cast<const uint4 *>(src + n * stride)[c] : make_uint4(0u, 0u, 0u, 0u);
    const uint16_t *weight = is_q ? a.q_weight : a.k_weight;
    const uint4 wu = weight ? reinterpret_cast<const uint4 *>(weight)[c] : make_uint4(0u, 0u, 0u, 0u);
    if (tid < kHeadDim / 2) {
        float co = 1.0f, si = 0.0f;
        int d0 = 2 * tid, d1 = 2 * tid + 1;  // the pair's dims; those past `rotary` stay as they are
        if (tid < half) {
            double turns = (double)pos * ((double)a.inv_freq[tid] * 0.15915494309189535);
            turns -= rint(turns);
            sincospif(2.0f * (float)turns, &si, &co);
            co *= a.scale;
            si *= a.scale;
            if (PAIRS != kNeighbours) {
                d0 = tid;
                d1 = tid + half;
            }
        }
        s_cos[place(d0)] = co;
        s_cos[place(d1)] = co;
        s_sin[place(d0)] = -si;
        s_sin[place(d1)] = si;
    }
    // the lane that holds the partners of this lane's dims
    int from = lane;
    if (PAIRS == kHalves && 8 * c < a.rotary) from = 8 * c < half ? lane + half / 8 : lane - half / 8;
    __syncthreads();
    if (pos < 0 || row < 0 || row >= a.n_rows) return;  // (here, so that no load waits for it)
    float x[8], w[8];
    unpack8(u, x);
    if (weight) {
        unpack8(wu, w);
        float ss = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) ss = fmaf(x[i], x[i], ss);
        const float r = rsqrtf(row16_sum(ss) * (1.0f / kHeadDim) + a.eps);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = x[i] * r * w[i];
    }
    uint32_t o[4];
#pragma unroll
    for (int i = 0; i < 8; i += 4) {
        const float4 co4 = reinterpret_cast<const float4 *>(s_cos)[4 * i + c];
        const float4 si4 = reinterpret_cast<const float4 *>(s_sin)[4 * i + c];
        const float co[4] = {co4.x, co4.y, co4.z, co4.w}, si[4] = {si4.x, si4.y, si4.z, si4.w};
        float y[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            y[k] = fmaf(partner<PAIRS>(x, i + k, from), si[k], x[i + k] * co[k]);
            // (a dim past `rotary` has no partner: no product of 0 with an infinity)
            if (PAIRS != kHalves64 && 8 * c >= a.rotary) y[k] = x[i + k];
        }
        o[i / 2] = pack2(y[0], y[1]);
        o[i / 2 + 1] = pack2(y[2], y[3]);
    }
    if (live) {
        uint16_t *dst = is_q ? a.q_out + (size_t)row * a.Hq * kHeadDim : (is_v ? a.v_out : a.k_out) + (size_t)row * a.Hkv * kHeadDim;
        reinterpret_cast<uint4 *>(dst + (size_t)own * kHeadDim)[c] = is_v ? u : make_uint4(o[0], o[1], o[2], o[3]);
    }
}

template <Pairs PAIRS>
void launch_pairs(const RopeArgs &a, hipStream_t stream) {
    const int heads = a.Hq + a.Hkv + (a.v ? a.Hkv : 0);
    const dim3 grid((heads + kHeads - 1) / kHeads, a.n_tokens < kGridTokens ? a.n_tokens : kGridTokens,
                    (unsigned)(((int64_t)a.n_tokens + kGridTokens - 1) / kGridTokens));
    hipLaunchKernelGGL((rope_kernel<PAIRS>), grid, dim3(kThreads), 0, stream, a);
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
