// Acceptance of a tree of drafted tokens (gfx950): Sec. 4.3's rule (keep the
// agreeing prefix, correct the first divergence) with the drafts a tree.
//
// Row 0 of a sequence holds the target model's scores for the token after the
// context, row j + 1 those for the token after node j.  Every row has one
// choice: its highest score (the lowest index among equal ones), or a draw
// from its probabilities with the row's own uniform.  From the root on, the
// walk steps to the child of the current node whose token is the current row's
// choice (the first such child) and ends where there is none, and that choice
// is the next token.  With drawn choices the emitted tokens are distributed as
// the target model's whatever the tree, because every one of them is a draw
// from the target's own row.
//
// The draw is exact, by integer weights (see lynx_spec_accept_sample in
// lynx.h): w_v = floor(p_v 2^40), S their sum, t = floor(S U / 2^32), the
// token the first whose inclusive prefix exceeds t.
#include "lane_ops.h"
#include "lynx_internal.h"

#include <limits.h>
#include <math.h>

namespace lynx {
namespace {

constexpr int kThreads = 256;
constexpr int kChunk = 4096;  // vocabulary entries per workgroup of the first pass

__device__ __forceinline__ bool better(float v, int i, float bv, int bi) { return v > bv || (v == bv && i < bi); }

__device__ __forceinline__ uint64_t weight(float r) {
    r = r > 0.0f ? r : 0.0f;  // NaN and negatives count 0
    r = r < 1.0f ? r : 1.0f;
    return (uint64_t)(r * 1099511627776.0f);  // 2^40: exact scaling, then truncation
}

__device__ __forceinline__ uint32_t uniform32(float u) {
    const float s = u * 4294967296.0f;
    if (!(s > 0.0f)) return 0u;
    if (s >= 4294967296.0f) return 0xFFFFFFFFu;
    return (uint32_t)s;
}

// The best (score, index) of a chunk of a row; an index of INT_MAX where it has
// no score above NaN.
__global__ __launch_bounds__(kThreads) void tree_argmax_kernel(TreeAcceptArgs a) {
    const int c = blockIdx.x, row = blockIdx.y, b = blockIdx.z, tid = threadIdx.x;
    const float *x = a.scores + ((size_t)b * (a.n + 1) + row) * a.vocab;
    const int hi = min(a.vocab, (c + 1) * kChunk);
    float bv = -INFINITY;
    int bi = INT_MAX;
    for (int e = c * kChunk + tid; e < hi; e += kThreads)
        if (better(x[e], e, bv, bi)) {
            bv = x[e];
            bi = e;
        }
    __shared__ float s_v[kThreads];
    __shared__ int s_i[kThreads];
    s_v[tid] = bv;
    s_i[tid] = bi;
    __syncthreads();
    for (int off = kThreads / 2; off > 0; off >>= 1) {
        if (tid < off && better(s_v[tid + off], s_i[tid + off], s_v[tid], s_i[tid])) {
            s_v[tid] = s_v[tid + off];
            s_i[tid] = s_i[tid + off];
        }
        __syncthreads();
    }
    if (tid == 0) {
        const size_t p = ((size_t)b * (a.n + 1) + row) * a.chunks + c;
        a.part[2 * p] = __float_as_uint(s_v[0]);
        a.part[2 * p + 1] = (uint32_t)s_i[0];
    }
}

// The sum of a chunk's weights.
__global__ __launch_bounds__(kThreads) void tree_sum_kernel(TreeAcceptArgs a) {
    const int c = blockIdx.x, row = blockIdx.y, b = blockIdx.z, tid = threadIdx.x;
    const float *x = a.scores + ((size_t)b * (a.n + 1) + row) * a.vocab;
    const int hi = min(a.vocab, (c + 1) * kChunk);
    uint64_t s = 0;
    for (int e = c * kChunk + tid; e < hi; e += kThreads) s += weight(x[e]);
    __shared__ uint64_t s_s[kThreads];
    s_s[tid] = s;
    __syncthreads();
    for (int off = kThreads / 2; off > 0; off >>= 1) {
        if (tid < off) s_s[tid] += s_s[tid + off];
        __syncthreads();
    }
    if (tid == 0) reinterpret_cast<uint64_t *>(a.part)[((size_t)b * (a.n + 1) + row) * a.chunks + c] = s_s[0];
}

// One wavefront per row: its choice.
template <bool SAMPLE>
__global__ __launch_bounds__(64) void tree_choice_kernel(TreeAcceptArgs a) {
    const int row = blockIdx.x, b = blockIdx.y, lane = threadIdx.x;
    const size_t r = (size_t)b * (a.n + 1) + row;
    int choice = -1;
    if (SAMPLE) {
        const uint64_t *part = reinterpret_cast<const uint64_t *>(a.part) + r * a.chunks;
        uint64_t S = 0;
        for (int c = 0; c < a.chunks; ++c) S += part[c];
        if (S > 0) {
            const uint32_t U = uniform32(a.uniforms[r]);
            uint64_t t = (S >> 32) * U + (((S & 0xFFFFFFFFull) * U) >> 32);
            int c = 0;
            while (t >= part[c]) t -= part[c++];  // t < S: ends inside the row
            const float *x = a.scores + r * a.vocab;
            // 64 entries at a time
            for (int e0 = c * kChunk;; e0 += 64) {
                const uint64_t w = e0 + lane < a.vocab ? weight(x[e0 + lane]) : 0;
                uint64_t upto = w;
                for (int off = 1; off < 64; off <<= 1) {
                    const uint64_t y = __shfl_up(upto, off);
                    if (lane >= off) upto += y;
                }
                const uint64_t past = __ballot(upto > t);
                if (past) {
                    choice = e0 + __ffsll((long long)past) - 1;
                    break;
                }
                t -= __shfl(upto, 63);
            }
        }
    } else {
        float bv = -INFINITY;
        int bi = INT_MAX;
        for (int c = 0; c < a.chunks; ++c) {
            const float v = __uint_as_float(a.part[2 * (r * a.chunks + c)]);
            const int i = (int)a.part[2 * (r * a.chunks + c) + 1];
            if (better(v, i, bv, bi)) {
                bv = v;
                bi = i;
            }
        }
        if (bi != INT_MAX) choice = bi;
    }
    if (lane == 0) a.choice[r] = choice;
}

// One wavefront per sequence walks the tree, a node in each lane.
__global__ __launch_bounds__(64) void tree_walk_kernel(TreeAcceptArgs a) {
    const int b = blockIdx.x, lane = threadIdx.x;
    const bool in = lane < a.n;
    const int up = in ? a.parents[(size_t)b * a.n + lane] : -2;
    const int token = in ? a.tokens[(size_t)b * a.n + lane] : -1;
    const bool there = up >= -1 && up < lane && token >= 0 && token < a.vocab;
    const int want = there ? a.choice[(size_t)b * (a.n + 1) + up + 1] : -1;
    const bool agrees = there && want == token;
    int at = -1, kept = 0, mine = -1;
    for (;;) {
        const uint64_t next = __ballot(agrees && up == at);
        if (!next) break;
        at = __ffsll((long long)next) - 1;  // nodes go up along a path: ends
        if (lane == kept) mine = at;
        ++kept;
    }
    if (in) a.path[(size_t)b * a.n + lane] = mine;
    if (lane == 0) {
        a.accepted[b] = kept;
        a.next_token[b] = a.choice[(size_t)b * (a.n + 1) + at + 1];
    }
    // the workspace is left zero
    __syncthreads();
    const size_t r0 = (size_t)b * (a.n + 1);
    for (int i = lane; i <= a.n; i += 64) a.choice[r0 + i] = 0;
    for (int i = lane; i < (a.n + 1) * a.chunks; i += 64)
        reinterpret_cast<uint64_t *>(a.part)[r0 * a.chunks + i] = 0;
}

}  // namespace

static int chunks_of(int vocab) { return (vocab + kChunk - 1) / kChunk; }

// Per row 16 bytes of state and 8 a chunk, per sequence 16 bytes.
size_t spec_tree_workspace(int B, int n, int vocab) {
    return (size_t)B * ((size_t)(n + 1) * (16 + 8 * (size_t)chunks_of(vocab)) + 16);
}

hipError_t launch_spec_accept_tree(TreeAcceptArgs a, int B, void *workspace, hipStream_t stream) {
    a.chunks = chunks_of(a.vocab);
    const size_t rows = (size_t)B * (a.n + 1);
    a.part = reinterpret_cast<uint32_t *>(workspace);
    a.choice = reinterpret_cast<int32_t *>(a.part + 2 * rows * a.chunks);
    const dim3 grid(a.chunks, a.n + 1, B);
    if (a.uniforms) {
        hipLaunchKernelGGL(tree_sum_kernel, grid, dim3(kThreads), 0, stream, a);
        hipLaunchKernelGGL(tree_choice_kernel<true>, dim3(a.n + 1, B), dim3(64), 0, stream, a);
    } else {
        hipLaunchKernelGGL(tree_argmax_kernel, grid, dim3(kThreads), 0, stream, a);
        hipLaunchKernelGGL(tree_choice_kernel<false>, dim3(a.n + 1, B), dim3(64), 0, stream, a);
    }
    hipLaunchKernelGGL(tree_walk_kernel, dim3(B), dim3(64), 0, stream, a);
    return hipGetLastError();
}

}  // namespace lynx
