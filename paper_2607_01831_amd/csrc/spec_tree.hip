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
//
// What bounds it: the rows along the path are all that decides, a few of the
// n + 1, but which ones they are is known a row at a time.  So there are two
// kernels:
//  * tree_rows_kernel reads every row at once: bandwidth for the rows that are
//    not needed, but no waiting;
//  * tree_path_kernel follows the path, a workgroup per (vocabulary chunk,
//    sequence): each publishes its chunk's best score (or sum of weights) of
//    the row, waits until all chunks are in, and goes on to the child that they
//    decide: a few microseconds a row, and nothing else is read (drawn, besides,
//    a row that the draw's chunk makes likely to be the next).
// 16 sequences of 63 nodes and 128256 entries, 4 kept (525 MB in all rows, 41 MB
// on the paths): 93.6 us (5.6 TB/s) and 19.7 us, 3.4 us a row after the first.
// A wait in tree_path_kernel is bounded: a workgroup that has waited too long
// (the others are not running, another kernel holds the device) reads its chunk
// of every row and leaves; whoever leaves last walks the tree from what has been
// published, so the result is the same.
#include "lane_ops.h"
#include "lynx_internal.h"

#include <limits.h>
#include <math.h>


namespace lynx {
namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;

__device__ __forceinline__ bool better(float v, int i, float bv, int bi) { return v > bv || (v == bv && i < bi); }

// floor(p 2^40) of p clamped to [0, 1] (a NaN counts 0), as its upper part times
// 2^20 and its lower 20 bits: every step is exact, and the parts of 64 entries
// sum in 32 bits.
__device__ __forceinline__ void weight_parts(float p, uint32_t &upper, uint32_t &lower) {
    const float s = fminf(fmaxf(p, 0.0f), 1.0f) * 1048576.0f;  // 2^20
    const uint32_t u = (uint32_t)s;
    upper += u;
    lower += (uint32_t)((s - (float)u) * 1048576.0f);
}
__device__ __forceinline__ uint64_t weight(float p) {
    uint32_t upper = 0, lower = 0;
    weight_parts(p, upper, lower);
    return ((uint64_t)upper << 20) + lower;
}

__device__ __forceinline__ uint32_t uniform32(float u) {
    const float s = u * 4294967296.0f;
    if (!(s > 0.0f)) return 0u;
    if (s >= 4294967296.0f) return 0xFFFFFFFFu;
    return (uint32_t)s;
}

// One word per chunk of a row says what the chunk holds, 0 while it is not in:
// greedy, (score, index) as a number that is larger for a higher score and,
// among equal ones, for a lower index, or 1 for NaNs alone; drawn, the sum of
// the weights, times 2, plus 1.
__device__ __forceinline__ uint64_t key_of(float v, int i) {
    const uint32_t u = __float_as_uint(v + 0.0f);  // -0 is +0
    return (uint64_t)(u >> 31 ? ~u : u | 0x80000000u) << 32 | (uint32_t)~i;
}
__device__ __forceinline__ int index_of(uint64_t key) { return key >> 32 ? (int)~(uint32_t)key : -1; }

// State of a row, a cache line apart: chunks that are in, and its choice + 2.
struct RowState {
    unsigned count;
    int choice;
    unsigned arrived;  // (of state n + 1: the sequence's arrivals)
    unsigned pad[13];
};
static_assert(sizeof(RowState) == kTreeStateBytes, "state size");

template <typename T>
__device__ __forceinline__ T agent_load(const T *p) {
    return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
template <typename T>
__device__ __forceinline__ void agent_store(T *p, T v) {
    __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ unsigned agent_add(unsigned *p) {
    return __hip_atomic_fetch_add(p, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
// This thread's memory operations so far are done, for every other workgroup of
// the device too where they were agent_store or agent_add.
__device__ __forceinline__ void settled() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }

__device__ __forceinline__ uint64_t wave_max(uint64_t v) {
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) {
        const uint64_t o = __shfl_xor(v, off);
        v = o > v ? o : v;
    }
    return v;
}
__device__ __forceinline__ uint64_t wave_sum(uint64_t v) {
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) v += __shfl_xor(v, off);
    return v;
}
__device__ __forceinline__ uint64_t wave_scan(uint64_t v) {  // inclusive
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
        const uint64_t o = __shfl_up(v, off);
        if (lane >= off) v += o;
    }
    return v;
}
// The exclusive prefix of x over the workgroup's threads, and the total.
__device__ __forceinline__ uint64_t block_scan(uint64_t x, uint64_t *s_wave, uint64_t &total) {
    const int w = threadIdx.x >> 6;
    const uint64_t upto = wave_scan(x);
    __syncthreads();
    if ((threadIdx.x & 63) == 63) s_wave[w] = upto;
    __syncthreads();
    uint64_t before = upto - x;
    total = 0;
    for (int j = 0; j < kWaves; ++j) {
        if (j < w) before += s_wave[j];
        total += s_wave[j];
    }
    return before;
}

// A thread's PER entries of a chunk of 256 PER: entry j is
// lo + 1024 (j / 4) + 4 tid + j % 4 where rows are 16-byte aligned (vec4),
// lo + 256 j + tid otherwise; entries past the row are NaN.
template <int PER>
__device__ __forceinline__ void load_chunk(const float *row, int lo, int V, bool vec4, float (&x)[PER]) {
    const int tid = threadIdx.x;
    if (vec4) {
#pragma unroll
        for (int j = 0; j < PER / 4; ++j) {
            const int e = lo + 4 * kThreads * j + 4 * tid;
            const float4 u = *reinterpret_cast<const float4 *>(row + min(e, V - 4));
            x[4 * j] = e < V ? u.x : NAN;
            x[4 * j + 1] = e < V ? u.y : NAN;
            x[4 * j + 2] = e < V ? u.z : NAN;
            x[4 * j + 3] = e < V ? u.w : NAN;
        }
    } else {
#pragma unroll
        for (int j = 0; j < PER; ++j) {
            const int e = lo + kThreads * j + tid;
            const float u = row[min(e, V - 1)];
            x[j] = e < V ? u : NAN;
        }
    }
}

// The word of a chunk, in thread 0.
template <bool SAMPLE, int PER>
__device__ __forceinline__ uint64_t chunk_word(const float (&x)[PER], int lo, bool vec4, uint64_t *s_wave) {
    const int tid = threadIdx.x;
    uint64_t v;
    if (SAMPLE) {
        uint32_t upper = 0, lower = 0;
#pragma unroll
        for (int j = 0; j < PER; ++j) weight_parts(x[j], upper, lower);
        v = wave_sum(((uint64_t)upper << 20) + lower);
    } else {
        float bv = -INFINITY;
#pragma unroll
        for (int j = 0; j < PER; ++j) bv = fmaxf(bv, x[j]);  // passes over NaN
        const float m = max_kg(row16_max(bv));
        int bi = INT_MAX;
#pragma unroll
        for (int j = PER - 1; j >= 0; --j)
            bi = x[j] == m ? (vec4 ? lo + 4 * kThreads * (j / 4) + 4 * tid + j % 4 : lo + kThreads * j + tid) : bi;
#pragma unroll
        for (int off = 32; off > 0; off >>= 1) bi = min(bi, __shfl_xor(bi, off));
        v = bi == INT_MAX ? 1 : key_of(m, bi);
    }
    if ((tid & 63) == 0) s_wave[tid >> 6] = v;
    __syncthreads();
    if (tid == 0) {
        for (int j = 1; j < kWaves; ++j) v = SAMPLE ? v + s_wave[j] : s_wave[j] > v ? s_wave[j] : v;
        if (SAMPLE) v = 2 * v + 1;
    }
    return v;
}

// t = floor(S U / 2^32), U = floor(u 2^32)
__device__ __forceinline__ uint64_t target(uint64_t S, float u) {
    const uint64_t U = uniform32(u);
    return (S >> 32) * U + (((S & 0xFFFFFFFFull) * U) >> 32);
}

// By one wavefront, a row's words (word `lane` in `first`): whether all are in.
__device__ __forceinline__ bool look(const uint64_t *words, int chunks, uint64_t &first) {
    const int lane = threadIdx.x & 63;
    first = lane < chunks ? agent_load(words + lane) : 1;
    bool all = first != 0;
    for (int c = 64 + lane; c < chunks; c += 64) all &= agent_load(words + c) != 0;
    return __all(all);
}
// All being in, the choice (greedy), or where the draw falls: the chunk, or -1
// where every weight is 0, and the target less the weights before the chunk.
__device__ __forceinline__ int best_index(const uint64_t *words, int chunks, uint64_t first) {
    uint64_t v = first;
    for (int c = 64 + (int)(threadIdx.x & 63); c < chunks; c += 64) {
        const uint64_t x = agent_load(words + c);
        v = x > v ? x : v;
    }
    return index_of(wave_max(v));
}
__device__ __forceinline__ int drawn_chunk(const uint64_t *words, int chunks, uint64_t first, float u, uint64_t &left) {
    const int lane = threadIdx.x & 63;
    uint64_t S = first >> 1;
    for (int c = 64 + lane; c < chunks; c += 64) S += agent_load(words + c) >> 1;
    S = wave_sum(S);
    if (S == 0) return -1;
    uint64_t t = target(S, u);  // below S: a chunk is found
    for (int c0 = 0;; c0 += 64) {
        const uint64_t x = (c0 == 0 ? first : c0 + lane < chunks ? agent_load(words + c0 + lane) : 0) >> 1;
        const uint64_t upto = wave_scan(x);
        const uint64_t past = __ballot(upto > t);
        if (past) {
            const int l = __ffsll((long long)past) - 1;
            left = t - __shfl(upto - x, l);
            return c0 + l;
        }
        t -= __shfl(upto, 63);
    }
}

// A chunk (held as load_chunk gives it) laid out for its draw: through LDS, so
// that thread tid has entries PER tid .. + PER - 1 and one scan does (16
// sequences, 50257 entries, 6 kept, along the path: 38 us, with a scan for every
// 256 entries 62 us).  The weights before the thread's entries, and theirs.
template <int PER>
__device__ __forceinline__ int entry_slot(int e) { return e + e / PER; }  // a thread's entries start in another bank
template <int PER>
__device__ __forceinline__ uint64_t lay_out(const float (&x)[PER], bool vec4, uint64_t *s_wave, float *s_x, uint64_t &sum) {
    const int tid = threadIdx.x;
#pragma unroll
    for (int j = 0; j < PER; ++j)
        s_x[entry_slot<PER>(vec4 ? 4 * kThreads * (j / 4) + 4 * tid + j % 4 : kThreads * j + tid)] = x[j];
    __syncthreads();
    uint32_t upper = 0, lower = 0;
#pragma unroll
    for (int j = 0; j < PER; ++j) weight_parts(s_x[entry_slot<PER>(PER * tid + j)], upper, lower);
    sum = ((uint64_t)upper << 20) + lower;
    uint64_t all;
    return block_scan(sum, s_wave, all);
}
// The entry at which the chunk's weights pass `left`, in the thread that has it;
// -1 in the others.
template <int PER>
__device__ __forceinline__ int drawn_entry(const float *s_x, int lo, uint64_t left, uint64_t before, uint64_t sum) {
    if (left < before || left - before >= sum) return -1;
    int at = PER - 1;
    uint64_t upto = before + sum;
#pragma unroll
    for (int j = PER - 1; j > 0; --j) {
        upto -= weight(s_x[entry_slot<PER>(PER * threadIdx.x + j)]);  // the weights of the entries before j
        if (upto > left) at = j - 1;
    }
    return lo + PER * threadIdx.x + at;
}

// The tree in a wavefront, a node in each lane.
struct Tree {
    int up, token;
    bool there;
    __device__ __forceinline__ Tree(const TreeAcceptArgs &a, int b) {
        const int lane = threadIdx.x & 63;
        const bool in = lane < a.n;
        up = in ? a.parents[(size_t)b * a.n + lane] : -2;
        token = in ? a.tokens[(size_t)b * a.n + lane] : -1;
        there = up >= -1 && up < lane && token >= 0 && token < a.vocab;
    }
    // The node that follows `at` (-1: the context) where the choice after it is
    // `choice`; -1 where none does.
    __device__ __forceinline__ int next(int at, int choice) const {
        return __ffsll((long long)__ballot(there && up == at && token == choice)) - 1;
    }
};

__device__ __forceinline__ void write_result(const TreeAcceptArgs &a, int b, int kept, int mine, int choice) {
    const int lane = threadIdx.x & 63;
    if (lane < a.n) a.path[(size_t)b * a.n + lane] = mine;
    if (lane == 0) {
        a.accepted[b] = kept;
        a.next_token[b] = choice;
    }
}

// Every row at once: workgroup (chunk, row, sequence).  The last chunk of a row
// to come in makes the row's choice, the last row of a sequence the walk.
template <bool SAMPLE, int PER>
__global__ __launch_bounds__(kThreads) void tree_rows_kernel(TreeAcceptArgs a) {
    const int c = blockIdx.x, row = blockIdx.y, b = blockIdx.z;
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
    const bool vec4 = a.vocab % 4 == 0;
    const int lo = c * PER * kThreads;
    const size_t r = (size_t)b * (a.n + 1) + row;
    RowState *state = reinterpret_cast<RowState *>(a.state) + (size_t)b * (a.n + 2);
    uint64_t *words = a.words + r * a.chunks;
    const float *x = a.scores + r * a.vocab;
    __shared__ uint64_t s_wave[kWaves], s_left;
    __shared__ int s_at, s_last, s_chunk;
    __shared__ float s_x[SAMPLE ? (PER + 1) * kThreads : 1];
    float v[PER];
    load_chunk(x, lo, a.vocab, vec4, v);
    const uint64_t word = chunk_word<SAMPLE>(v, lo, vec4, s_wave);
    if (tid == 0) {
        agent_store(words + c, word);
        settled();
        s_last = agent_add(&state[row].count) == (unsigned)(a.chunks - 1);
    }
    __syncthreads();
    if (!s_last) return;
    int choice;
    if (SAMPLE) {
        if (w == 0) {
            uint64_t left = 0, first;
            look(words, a.chunks, first);
            const int at = drawn_chunk(words, a.chunks, first, a.uniforms[r], left);
            if (lane == 0) {
                s_chunk = at;
                s_left = left;
            }
        }
        __syncthreads();
        choice = s_chunk;
        if (choice >= 0) {
            const int at = choice * PER * kThreads;
            load_chunk(x, at, a.vocab, vec4, v);
            uint64_t sum;
            const uint64_t before = lay_out(v, vec4, s_wave, s_x, sum);
            const int entry = drawn_entry<PER>(s_x, at, s_left, before, sum);
            if (entry >= 0) s_at = entry;
            __syncthreads();
            choice = s_at;
        }
    } else {
        choice = 0;
        if (w == 0) {
            uint64_t first;
            look(words, a.chunks, first);
            choice = best_index(words, a.chunks, first);
        }
    }
    settled();
    __syncthreads();  // the words have been read
    for (int i = tid; i < a.chunks; i += kThreads) agent_store(words + i, (uint64_t)0);
    if (w != 0) return;
    if (lane == 0) {
        agent_store(&state[row].count, 0u);
        agent_store(&state[row].choice, choice + 2);
    }
    settled();
    int last = 0;
    if (lane == 0) last = agent_add(&state[a.n + 1].arrived) == (unsigned)a.n;
    if (!__shfl(last, 0)) return;
    const Tree tree(a, b);
    const int after = agent_load(&state[tree.there ? tree.up + 1 : 0].choice) - 2;
    const bool edge = tree.there && after == tree.token;
    int at = -1, kept = 0, mine = -1;
    for (;;) {
        const uint64_t next = __ballot(edge && tree.up == at);
        if (!next) break;
        at = __ffsll((long long)next) - 1;  // nodes go up along a path: ends
        if (lane == kept) mine = at;
        ++kept;
    }
    write_result(a, b, kept, mine, agent_load(&state[at + 1].choice) - 2);
    settled();
    for (int i = lane; i <= a.n; i += 64) agent_store(&state[i].choice, 0);
    if (lane == 0) agent_store(&state[a.n + 1].arrived, 0u);
}

// The rows along the path: workgroup (chunk, sequence).
template <bool SAMPLE, int PER>
__global__ __launch_bounds__(kThreads) void tree_path_kernel(TreeAcceptArgs a) {
    const int c = blockIdx.x, b = blockIdx.y;
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
    const int V = a.vocab, n = a.n;
    const bool vec4 = V % 4 == 0;
    const int lo = c * PER * kThreads;
    const size_t r0 = (size_t)b * (n + 1);
    RowState *state = reinterpret_cast<RowState *>(a.state) + (size_t)b * (n + 2);
    __shared__ uint64_t s_wave[kWaves], s_left;
    __shared__ int s_at, s_row, s_draw, s_last;
    __shared__ float s_x[SAMPLE ? (PER + 1) * kThreads : 1];
    constexpr int kEnd = -1, kLate = -2;

    const Tree tree(a, b);
    int at = -1, kept = 0, mine = -1, choice = -1;
    uint64_t done = 0;  // rows above 0 that this workgroup has read, a bit per node
    // Ends when f() holds, or with false after so many looks.
    auto wait = [&](auto f) {
        for (int left = a.looks; left > 0; --left) {
            if (f()) return true;
            __builtin_amdgcn_s_sleep(1);
        }
        return false;
    };
    float v[PER];
    int row = 0, held = -1;  // held: the row whose chunk is in v already
    for (;;) {
        uint64_t *words = a.words + (r0 + row) * a.chunks;
        if (held != row) load_chunk(a.scores + (r0 + row) * V, lo, V, vec4, v);
        const uint64_t word = chunk_word<SAMPLE>(v, lo, vec4, s_wave);
        if (tid == 0) agent_store(words + c, word);
        const float uniform = SAMPLE ? a.uniforms[r0 + row] : 0.0f;
        uint64_t before = 0, sum = 0;
        if (SAMPLE) before = lay_out(v, vec4, s_wave, s_x, sum);  // in case the draw falls here, while the words come in
        bool in = false;                                         // (of the first wavefront)
        if (w == 0) {
            uint64_t left = 0, first = 0;
            in = wait([&] { return look(words, a.chunks, first); });
            int draw = -1;
            if (in) {
                if (SAMPLE)
                    draw = drawn_chunk(words, a.chunks, first, uniform, left);
                else
                    choice = best_index(words, a.chunks, first);
            }
            if (lane == 0) {
                s_draw = in ? draw : kLate;
                s_left = left;
            }
        }
        if (SAMPLE) {
            __syncthreads();
            const int draw = s_draw;
            if (draw == kLate) {
                row = kLate;
                break;
            }
            if (draw == c) {  // the draw falls into this chunk: the others wait for its entry
                const int entry = drawn_entry<PER>(s_x, lo, s_left, before, sum);
                if (entry >= 0) agent_store(&state[row].choice, entry + 2);
            }
            // while the entry comes in, the row that follows if it is the token of
            // the first child that lies in the drawn chunk (16 sequences of 128256
            // entries, 4 kept: 31.2 us, without 34.4)
            const int from = draw * PER * kThreads;
            const bool mine_may = tree.there && tree.up == row - 1 && tree.token - from >= 0 &&
                                  tree.token - from < PER * kThreads;
            const uint64_t may = draw >= 0 ? __ballot(mine_may) : 0ull;
            if (may) {
                held = __ffsll((long long)may);  // the child's number and 1
                load_chunk(a.scores + (r0 + held) * V, lo, V, vec4, v);
            }
            if (w == 0) {
                int got = 1;  // no weight at all: -1
                in = draw < 0 || wait([&] { return (got = agent_load(&state[row].choice)) != 0; });
                choice = got - 2;
            }
        }
        if (w == 0) {
            const int j = in ? tree.next(at, choice) : -1;
            if (j >= 0) {
                at = j;
                if (lane == kept) mine = j;
                ++kept;
                done |= 1ull << j;
            }
            if (lane == 0) s_row = !in ? kLate : j >= 0 ? j + 1 : kEnd;
        }
        __syncthreads();
        row = s_row;
        __syncthreads();
        if (row < 0) break;
    }
    const bool late = row == kLate;
    if (late) {
        // the others may never come while this workgroup is here: its chunk of
        // every other row, and away
        if (tid == 0) s_left = done;
        __syncthreads();
        const uint64_t read = s_left;
        for (int j = 0; j < n; ++j) {
            if (read >> j & 1) continue;
            load_chunk(a.scores + (r0 + j + 1) * V, lo, V, vec4, v);
            const uint64_t word = chunk_word<SAMPLE>(v, lo, vec4, s_wave);
            if (tid == 0) agent_store(a.words + (r0 + j + 1) * a.chunks + c, word);
            __syncthreads();
        }
    }

    settled();
    __syncthreads();
    if (tid == 0) s_last = agent_add(&state[n + 1].arrived) == (unsigned)(a.chunks - 1);
    __syncthreads();
    if (!s_last) return;
    if (late) {
        // every chunk of the rows on the path is in by now: the walk again
        at = -1;
        kept = 0;
        mine = -1;
        for (row = 0; row >= 0;) {
            const uint64_t *words = a.words + (r0 + row) * a.chunks;
            uint64_t left = 0, first;
            look(words, a.chunks, first);
            const int got = SAMPLE ? drawn_chunk(words, a.chunks, first, a.uniforms[r0 + row], left)
                                   : best_index(words, a.chunks, first);
            choice = got;
            if (SAMPLE && got >= 0) {
                load_chunk(a.scores + (r0 + row) * V, got * PER * kThreads, V, vec4, v);
                uint64_t sum;
                const uint64_t before = lay_out(v, vec4, s_wave, s_x, sum);
                const int entry = drawn_entry<PER>(s_x, got * PER * kThreads, left, before, sum);
                if (entry >= 0) s_at = entry;
                __syncthreads();
                choice = s_at;
                __syncthreads();  // every wavefront has it
            }
            const int j = tree.next(at, choice);  // every wavefront walks
            if (j >= 0) {
                at = j;
                if (lane == kept) mine = j;
                ++kept;
            }
            row = j >= 0 ? j + 1 : -1;
        }
    }
    if (w == 0) write_result(a, b, kept, mine, choice);
    __syncthreads();
    uint64_t *words = a.words + r0 * a.chunks;
    for (int i = tid; i < (n + 1) * a.chunks; i += kThreads) agent_store(words + i, (uint64_t)0);
    for (int i = tid; i <= n; i += kThreads) agent_store(&state[i].choice, 0);
    if (tid == 0) agent_store(&state[n + 1].arrived, 0u);
}

}  // namespace

constexpr int kRowsPer = 16;  // entries per thread of tree_rows_kernel
constexpr int kPathPer = 32;  // ... of tree_path_kernel

static int chunks_of(int vocab, int per) { return (vocab + per * kThreads - 1) / (per * kThreads); }

// [row states, and one for the sequence's arrivals][words]
size_t spec_tree_workspace(int B, int n, int vocab) {
    return (size_t)B * ((size_t)(n + 2) * kTreeStateBytes + (size_t)(n + 1) * 8 * chunks_of(vocab, kRowsPer));
}

// Which kernel: the rows at once while reading them all takes no longer than
// following a path of a few rows; entries in all rows, at once and along the path, us.
// Greedy, 4 kept: 13.3M 13.7 and 13.6, 16.2M 15.8 and 16.2, 16.4M 15.9 and 16.0 (16
// sequences: 15.8 and 15.2), 16.7M 16.3 and 14.3, 24.6M 20.3 and 18.1, 65.7M 43.2 and
// 17.1.  Drawn, where a row on the path waits for its draw too: 16.4M 20.3 and 28.6,
// 22.3M 24.3 and 29.1, 24.6M 25.6 and 28.9 (16 sequences: 31.1 and 29.1), 26.7M 27.8
// and 24.8, 65.7M 65.6 and 29.1.  What is kept is not known here, and a path as long
// as the tree is the other extreme: a chain of 63, all kept, 16 sequences, 224 us
// along it, 97 at once.  Chunks: 4096 entries where every row is read, 8192 along a
// path (16 sequences 20.2 us, by 4096 25.2, by 16384 26.7).
TreeAcceptWay spec_tree_way(int B, int n, int vocab, bool drawn) {
    const long long entries = (long long)B * (n + 1) * vocab;
    return TreeAcceptWay{entries <= (drawn ? 25000000ll : 16000000ll), 128};
}

hipError_t launch_spec_accept_tree(TreeAcceptArgs a, int B, TreeAcceptWay way, void *workspace, hipStream_t stream) {
    a.chunks = chunks_of(a.vocab, way.rows ? kRowsPer : kPathPer);
    a.looks = way.looks;
    a.state = workspace;
    a.words = reinterpret_cast<uint64_t *>(reinterpret_cast<char *>(workspace) + (size_t)B * (a.n + 2) * kTreeStateBytes);
    if (way.rows) {
        const dim3 grid(a.chunks, a.n + 1, B);
        if (a.uniforms)
            hipLaunchKernelGGL((tree_rows_kernel<true, kRowsPer>), grid, dim3(kThreads), 0, stream, a);
        else
            hipLaunchKernelGGL((tree_rows_kernel<false, kRowsPer>), grid, dim3(kThreads), 0, stream, a);
    } else {
        const dim3 grid(a.chunks, B);
        if (a.uniforms)
            hipLaunchKernelGGL((tree_path_kernel<true, kPathPer>), grid, dim3(kThreads), 0, stream, a);
        else
            hipLaunchKernelGGL((tree_path_kernel<false, kPathPer>), grid, dim3(kThreads), 0, stream, a);
    }
    return hipGetLastError();
}

}  // namespace lynx
