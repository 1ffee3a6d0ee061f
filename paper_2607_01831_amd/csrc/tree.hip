// Verification attention of a token tree (gfx950): the merge of the context's
// partials and the tree's own tokens.
//
// What it computes (Sec. 4.3, with the drafts a tree instead of a chain): node
// i of the tree attends the whole context and, among the nodes, its ancestors
// and itself.  The context part is the verification kernel's (verify.hip),
// which knows nothing of the tree; its partials (max, sum, output) of a row
// meet here with one more partial over the nodes, whose mask is the row's set
// of ancestors, one bit a node.
#include "lane_ops.h"
#include "lynx_internal.h"
#include "split_merge.h"
#include "work_list.h"

#include <math.h>

#include <type_traits>

namespace lynx {
namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr int kThreads = 256;

typedef short bf16x8_t __attribute__((ext_vector_type(8)));

__device__ __forceinline__ float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }
// Either half of a word of two BF16 is an infinity or a NaN.
__device__ __forceinline__ bool not_finite(uint32_t w) {
    return (w & 0x7f80u) == 0x7f80u || (w & 0x7f800000u) == 0x7f800000u;
}

// The ancestors of every node and the node itself, a bit each, in the node's
// lane (n <= 64); 0 for a node that is not there: one whose parent is not one
// of -1 .. i - 1, or any node below such a one.  Pointer doubling: after round
// r a lane holds its 2^r nearest ancestors and the one above them, so six
// rounds reach the root of any tree of 64.
__device__ __forceinline__ uint64_t ancestors(const int32_t *parents, int n) {
    const int lane = threadIdx.x & 63;
    int up = lane < n ? parents[lane] : -2;
    bool there = up >= -1 && up < lane;
    uint64_t mask = 1ull << lane;
    if (!there) up = -1;
#pragma unroll
    for (int r = 0; r < 6; ++r) {
        const int from = max(up, 0);
        const uint64_t m = __shfl(mask, from);
        const int next = __shfl(up, from);
        const bool ok = __shfl((int)there, from);
        if (up >= 0) {
            mask |= m;
            there = there && ok;
            up = next;
        }
    }
    return there ? mask : 0ull;
}

// A 64-bit value of one lane, in scalar registers (the lane number is uniform).
__device__ __forceinline__ uint64_t lane64(uint64_t v, int lane) {
    return (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)v, lane) |
           (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(v >> 32), lane) << 32;
}

// One workgroup per (ROWS rows, kv head, sequence): the rows' partials over the
// context, then the nodes that any of the rows sees (a row's ancestors are few,
// and the rows of a workgroup, neighbours in the tree, share most of them).
// Scores: wavefront w takes 16 of those nodes against the rows on the matrix
// cores (K and the queries are BF16, so the products are exact and the sums
// fp32).  Weights times values: thread (row r, dims 8 d8 .. + 7), fp32, the
// values staged in LDS once for all rows.  Where ROWS < 16 the threads of a row
// stand in 16 / ROWS groups, which share its partials.
// FIND: how the row's partials are found (see attn_combine_rows_kernel).
template <int ROWS, int FIND>
__global__ __launch_bounds__(kThreads) void tree_combine_kernel(TreeArgs a) {
    if (FIND == 1) __builtin_assume(a.B > 1 && a.B <= 64);
    constexpr int kPer = kThreads / ROWS;  // threads per row
    constexpr int kGroups = kPer / 16;     // groups of 16 threads per row
    constexpr int kBatch = 4;              // partials loaded together
    constexpr int kMost = 64;
    const int h = blockIdx.y, b = blockIdx.z;
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
    const int d8 = tid & 15, r = tid / kPer, grp = (tid % kPer) / 16;
    const int Hkv = a.geo.Hkv;
    const int row0 = blockIdx.x * ROWS;
    const bool row_live = row0 + r < a.rows_total;
    const int gr = min(row0 + r, a.rows_total - 1);
    __shared__ __attribute__((aligned(16))) uint4 s_v[kMost][16];  // values of the nodes seen
    __shared__ __attribute__((aligned(16))) float s_p[16][kMost + 4];  // scores (log2 units), then weights
    __shared__ int s_node[kMost];                                   // the nodes seen
    __shared__ float s_ml[ROWS][kGroups][2];
    __shared__ __attribute__((aligned(16))) float s_acc[kGroups > 1 ? ROWS : 1][kGroups > 1 ? kGroups - 1 : 1][kHeadDim];

    const int own = a.seq_lens[FIND == 0 ? b : min(lane, a.B - 1)];
    const uint64_t masks = ancestors(a.parents + (size_t)b * a.n, a.n);
    auto query_row = [&](int row) { return ((size_t)b * a.n + row / a.G) * a.Hq + (size_t)h * a.G + row % a.G; };
    // the queries, as the matrix cores' operand: row lane % 16, dims 8 kg + 32 kk
    const int kg = lane >> 4;
    const int qr = min(row0 + (lane & 15), a.rows_total - 1);
    uint4 qf[4];
#pragma unroll
    for (int kk = 0; kk < 4; ++kk)
        qf[kk] = *reinterpret_cast<const uint4 *>(a.q + query_row(qr) * kHeadDim + 8 * kg + 32 * kk);

    // ---- the row's partials: `live` of them from number seg0 on ----
    int live, seg0;
    if (FIND == 0) {
        live = min(a.max_live, WorkList<kWorkUnit, false>::units(max(0, min(own, a.max_seq_len))));
        seg0 = b * a.direct;
    } else {
        const WorkList<kWorkUnit, false> list(a.seq_lens, a.B, a.max_seq_len, a.workers, own);
        list.partials(b, seg0, live);
    }
    const size_t base = ((size_t)h * a.rows_total + gr) * a.n_seg + seg0;
    const float4 *o4 = reinterpret_cast<const float4 *>(a.ws_o + base * kHeadDim) + 2 * d8;
    float4 pv[kBatch][2];
    float2 ml[kBatch];
    auto load_batch = [&](int s0) {
#pragma unroll
        for (int k = 0; k < kBatch; ++k) {
            const int s = min(s0 + kGroups * k, live - 1);
            pv[k][0] = o4[(size_t)s * (kHeadDim / 4)];
            pv[k][1] = o4[(size_t)s * (kHeadDim / 4) + 1];
            ml[k] = a.ws_ml[base + s];
        }
    };
    load_batch(grp);

    // ---- the nodes that any of the rows sees ----
    uint64_t seen = 0;
    const int last = (min(row0 + ROWS, a.rows_total) - 1) / a.G;
    for (int i = row0 / a.G; i <= last; ++i) seen |= lane64(masks, i);
    const int n_seen = __popcll(seen);
    if (w == 0 && (seen >> lane & 1)) s_node[__popcll(seen & ((1ull << lane) - 1))] = lane;
    __syncthreads();
    const size_t t0 = ((size_t)b * a.n * Hkv + h) * kHeadDim;
    const size_t step = (size_t)Hkv * kHeadDim;
    if (16 * w < n_seen) {  // uniform in the wavefront
        const uint16_t *k = a.k_new + t0 + s_node[min(16 * w + (lane & 15), n_seen - 1)] * step + 8 * kg;
        f32x4_t s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int kk = 0; kk < 4; ++kk)
            s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                __builtin_bit_cast(__attribute__((__vector_size__(16))) __bf16, *reinterpret_cast<const uint4 *>(k + 32 * kk)),
                __builtin_bit_cast(__attribute__((__vector_size__(16))) __bf16, qf[kk]), s, 0, 0, 0);
        // lane (row lane % 16, kg) has the products with nodes 16 w + 4 kg ..
        const uint64_t mask = __shfl(masks, qr / a.G);
        const float sm = kLog2e * rsqrtf((float)kHeadDim);
        float x[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int j = 16 * w + 4 * kg + i;
            x[i] = j < n_seen && (mask >> s_node[min(j, kMost - 1)] & 1) ? s[i] * sm : -INFINITY;
        }
        *reinterpret_cast<float4 *>(&s_p[lane & 15][16 * w + 4 * kg]) = make_float4(x[0], x[1], x[2], x[3]);
    }
    bool odd = false;  // a value that is no number: it may not meet a weight of 0
    for (int j = tid / 16; j < n_seen; j += kThreads / 16) {
        const uint4 v = *reinterpret_cast<const uint4 *>(a.v_new + t0 + s_node[j] * step + 8 * d8);
        odd |= not_finite(v.x) || not_finite(v.y) || not_finite(v.z) || not_finite(v.w);
        s_v[j][d8] = v;
    }

    // ---- merge the partials ----
    float M = -INFINITY, L = 0.0f, acc[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    for (int s0 = grp; s0 < live; s0 += kGroups * kBatch) {
        if (s0 != grp) load_batch(s0);
        float mb = M;
#pragma unroll
        for (int k = 0; k < kBatch; ++k) {
            if (s0 + kGroups * k >= live) ml[k] = make_float2(-INFINITY, 0.0f);
            mb = fmaxf(mb, ml[k].x);
        }
        const float sc = M == -INFINITY ? 0.0f : exp2f(M - mb);
        L *= sc;
#pragma unroll
        for (int e = 0; e < 8; ++e) acc[e] *= sc;
#pragma unroll
        for (int k = 0; k < kBatch; ++k) {
            const float f = ml[k].x == -INFINITY ? 0.0f : exp2f(ml[k].x - mb);
            L = fmaf(ml[k].y, f, L);  // a NaN sum (bad block id) stays NaN
            // a partial of weight 0 may hold no output at all
            const float4 x = f != 0.0f ? pv[k][0] : make_float4(0.f, 0.f, 0.f, 0.f);
            const float4 y = f != 0.0f ? pv[k][1] : make_float4(0.f, 0.f, 0.f, 0.f);
            const float v[8] = {x.x, x.y, x.z, x.w, y.x, y.y, y.z, y.w};
#pragma unroll
            for (int e = 0; e < 8; ++e) acc[e] = fmaf(v[e], f, acc[e]);
        }
        M = mb;
    }
    if (kGroups > 1 && d8 == 0) {
        s_ml[r][grp][0] = M;
        s_ml[r][grp][1] = L;
    }
    if (kGroups > 1 && grp > 0)
        for (int e = 0; e < 8; ++e) s_acc[r][grp - 1][8 * d8 + e] = acc[e];
    odd = __syncthreads_or(odd);

    // ---- the row's weights over the nodes: its first 16 threads, node 16 i + d8
    // each; 0 for a node that the row does not see ----
    if (grp == 0) {
        if (kGroups > 1) {
            float Mg = M;
#pragma unroll
            for (int g = 1; g < kGroups; ++g) Mg = fmaxf(Mg, s_ml[r][g][0]);
            const float f0 = M == -INFINITY ? 0.0f : exp2f(M - Mg);
            L *= f0;
#pragma unroll
            for (int e = 0; e < 8; ++e) acc[e] *= f0;
#pragma unroll
            for (int g = 1; g < kGroups; ++g) {
                const float f = s_ml[r][g][0] == -INFINITY ? 0.0f : exp2f(s_ml[r][g][0] - Mg);
                L = fmaf(s_ml[r][g][1], f, L);
#pragma unroll
                for (int e = 0; e < 8; ++e) acc[e] = fmaf(s_acc[r][g - 1][8 * d8 + e], f, acc[e]);
            }
            M = Mg;
        }
        float t[4], top = M;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            t[i] = 16 * i + d8 < n_seen ? s_p[r][16 * i + d8] : -INFINITY;
            top = fmaxf(top, t[i]);
        }
        top = row16_max(top);
        const float sc = M == -INFINITY ? 0.0f : exp2f(M - top);
        float sum = 0.0f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float p = t[i] == -INFINITY ? 0.0f : exp2f(t[i] - top);
            sum += p;
            if (16 * i + d8 < n_seen) s_p[r][16 * i + d8] = p;
        }
        L = fmaf(L, sc, row16_sum(sum));
#pragma unroll
        for (int e = 0; e < 8; ++e) acc[e] *= sc;
    }
    __syncthreads();
    // a node that is not there sees nothing
    const bool there = __shfl(masks, gr / a.G) != 0;
    if (grp != 0) return;
    auto add_values = [&](auto careful) {
        for (int j = 0; j < n_seen; ++j) {
            const float p = s_p[r][j];
            uint4 v = s_v[j][d8];
            if (careful && p == 0.0f) v = make_uint4(0u, 0u, 0u, 0u);
            const uint32_t x[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                acc[2 * e] = fmaf(p, bf16_lo(x[e]), acc[2 * e]);
                acc[2 * e + 1] = fmaf(p, bf16_hi(x[e]), acc[2 * e + 1]);
            }
        }
    };
    if (odd)
        add_values(std::true_type{});
    else
        add_values(std::false_type{});
    if (!row_live) return;
    // 0 where the row has no weight; a NaN sum marks a bad block id
    const float inv = !there ? 0.0f : isnan(L) ? NAN : L > 0.0f ? 1.0f / L : 0.0f;
    uint32_t o[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const float x = there ? acc[2 * e] * inv : 0.0f, y = there ? acc[2 * e + 1] * inv : 0.0f;
        o[e] = f32_to_bf16_rne(x) | (uint32_t)f32_to_bf16_rne(y) << 16;
    }
    *reinterpret_cast<uint4 *>(a.out + query_row(gr) * kHeadDim + 8 * d8) = make_uint4(o[0], o[1], o[2], o[3]);
}

template <int ROWS>
void launch_rows(const TreeArgs &a, hipStream_t stream) {
    const dim3 grid((a.rows_total + ROWS - 1) / ROWS, a.geo.Hkv, a.B);
    if (a.direct || a.B == 1)
        hipLaunchKernelGGL((tree_combine_kernel<ROWS, 0>), grid, dim3(kThreads), 0, stream, a);
    else if (a.B <= 64)
        hipLaunchKernelGGL((tree_combine_kernel<ROWS, 1>), grid, dim3(kThreads), 0, stream, a);
    else
        hipLaunchKernelGGL((tree_combine_kernel<ROWS, 2>), grid, dim3(kThreads), 0, stream, a);
}

}  // namespace

hipError_t launch_tree_combine(const TreeArgs &a, int rows, hipStream_t stream) {
    if (rows == 4)
        launch_rows<4>(a, stream);
    else
        launch_rows<16>(a, stream);
    return hipGetLastError();
}

}  // namespace lynx
