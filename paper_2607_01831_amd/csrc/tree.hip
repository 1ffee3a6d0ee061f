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

namespace lynx {
namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr int kThreads = 128;

__device__ __forceinline__ float bf16_f(uint16_t v) { return __uint_as_float((uint32_t)v << 16); }

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

// One workgroup per (row, kv head, sequence), a thread per dim.
__global__ __launch_bounds__(kThreads) void tree_combine_kernel(TreeArgs a) {
    const int gr = blockIdx.x, h = blockIdx.y, b = blockIdx.z, d = threadIdx.x;
    const int node = gr / a.G;
    const size_t qrow = ((size_t)b * a.n + node) * a.Hq + (size_t)h * a.G + gr % a.G;
    const uint64_t masks = ancestors(a.parents + (size_t)b * a.n, a.n);
    const uint64_t mask = __shfl(masks, node);
    __shared__ float s_t[64];
    const float sm = kLog2e * rsqrtf((float)kHeadDim);

    using List = WorkList<kWorkUnit, false>;
    int live = 0, seg0 = b * a.direct;
    if (!a.direct && a.B > 1)
        List(a.seq_lens, a.B, a.max_seq_len, a.workers).partials(b, seg0, live);
    else
        live = min(a.max_live, List::units(max(0, min(a.seq_lens[b], a.max_seq_len))));
    const size_t base = ((size_t)h * a.rows_total + gr) * a.n_seg + seg0;
    float M = -INFINITY, L = 0.0f, acc = 0.0f;
    for (int s = 0; s < live; ++s) {
        const float2 ml = a.ws_ml[base + s];
        if (ml.x == -INFINITY && !isnan(ml.y)) continue;
        const float m = fmaxf(M, ml.x);
        const float e0 = M == -INFINITY ? 0.0f : exp2f(M - m), e1 = exp2f(ml.x - m);
        L = fmaf(ml.y, e1, L * e0);
        acc = fmaf(a.ws_o[(base + s) * kHeadDim + d], e1, acc * e0);
        M = m;
    }
    const size_t t0 = ((size_t)b * a.n * a.geo.Hkv + h) * kHeadDim;
    const size_t step = (size_t)a.geo.Hkv * kHeadDim;
    if (d < 64) {
        float s = -INFINITY;
        if (mask >> d & 1) {
            s = 0.0f;
            for (int e = 0; e < kHeadDim; ++e)
                s = fmaf(bf16_f(a.q[qrow * kHeadDim + e]), bf16_f(a.k_new[t0 + d * step + e]), s);
            s *= sm;
        }
        s_t[d] = s;
    }
    __syncthreads();
    for (int j = 0; j < a.n; ++j) {
        if (!(mask >> j & 1)) continue;
        const float s = s_t[j], m = fmaxf(M, s);
        const float e0 = M == -INFINITY ? 0.0f : exp2f(M - m), e1 = exp2f(s - m);
        L = fmaf(L, e0, e1);
        acc = fmaf(bf16_f(a.v_new[t0 + j * step + d]), e1, acc * e0);
        M = m;
    }
    float o = isnan(L) ? NAN : (L > 0.0f ? acc / L : 0.0f);
    if (mask == 0) o = 0.0f;  // the node is not there
    a.out[qrow * kHeadDim + d] = f32_to_bf16_rne(o);
}

}  // namespace

hipError_t launch_tree_combine(const TreeArgs &a, hipStream_t stream) {
    hipLaunchKernelGGL(tree_combine_kernel, dim3(a.rows_total, a.geo.Hkv, a.B), dim3(kThreads), 0, stream, a);
    return hipGetLastError();
}

}  // namespace lynx
