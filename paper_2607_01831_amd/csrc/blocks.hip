// The plan of a step on the device (gfx950): blocks for the new tokens of every
// sequence out of a stack of free ones, the block table's new entries, and of every
// new token its sequence, position, slot and row; and blocks given back.
//
// Sequence b holds len tokens in held = ceil(len / bt) blocks and asks for count
// more, need = ceil((len + count) / bt) - held blocks.  It is granted all of them
// where the blocks that it and the sequences before it need are on the stack and
// the tokens that they ask for have room.  So which block and which token number
// goes to whom follows from three prefix sums over the batch: the blocks asked, the
// tokens asked, the tokens granted.
//
// Bound by latency: the sums are a few reads and scans, and a token is four words.
// One launch: every workgroup computes the sums for itself (a batch's lengths are a
// few KB in the L2) and serves its share of the tokens; none waits for another.
// An entry of the table that this call writes is read from the stack by whoever
// needs it, an entry read from the table is never one that this call writes.  Only
// the stack's counter needs all to have read it before it moves: the last workgroup
// to arrive writes it.  The kernels take 3.0 and 1.9 us for one sequence, 3.8 and 3.6
// for 64 with 8 tokens each, 7.3 and 5.6 for 500 with 131072 rows (a call of the host
// 4.5).
#include "lane_ops.h"
#include "lynx_internal.h"
#include "split_merge.h"
#include "work_list.h"

namespace lynx {
namespace {

__device__ __forceinline__ int blocks_of(int tokens, int bt) { return (int)(((unsigned)tokens + bt - 1) / (unsigned)bt); }

// The sums over the workgroup's threads before this one's value, of `v`; `total` of all.
template <int THREADS>
__device__ __forceinline__ int scan_before(int v, int *s_wave, int &total) {
    const int upto = WorkList<kWorkUnit, false>::scan(v);
    const int w = threadIdx.x >> 6;
    __syncthreads();
    if ((threadIdx.x & 63) == 63) s_wave[w] = upto;
    __syncthreads();
    int before = 0;
    total = 0;
#pragma unroll
    for (int i = 0; i < THREADS / 64; ++i) {
        const int x = s_wave[i];
        before += i < w ? x : 0;
        total += x;
    }
    return before + upto - v;
}

struct Ask {
    int len, count, held, need;
};
__device__ __forceinline__ Ask ask_of(const BlocksArgs &a, int b) {
    Ask s;
    s.len = min(max(a.seq_lens[b], 0), a.capacity);
    s.count = min(min(max(a.counts[b], 0), a.n_src), a.capacity - s.len);
    s.held = blocks_of(s.len, a.bt);
    s.need = blocks_of(s.len + s.count, a.bt) - s.held;
    return s;
}

// The largest t with s[t] <= n, of a rising s[0 .. THREADS - 1] with s[0] <= n.
template <int THREADS>
__device__ __forceinline__ int find_last(const int *s, int n) {
    int t = 0;
#pragma unroll
    for (int step = THREADS / 2; step > 0; step >>= 1)
        if (s[t + step] <= n) t += step;
    return t;
}

// Once every workgroup has read the counter: write it.
template <int THREADS>
__device__ __forceinline__ void settle(int32_t *state, int value, int *flag) {
    if (gridDim.x == 1) {
        __syncthreads();
        if (threadIdx.x == 0) state[0] = value;
    } else if (last_to_arrive(reinterpret_cast<unsigned *>(state + 1), gridDim.x, flag) && threadIdx.x == 0) {
        state[0] = value;
    }
}

// Thread t answers for sequences t per .. t per + per - 1.
template <int THREADS>
__global__ __launch_bounds__(THREADS) void blocks_extend_kernel(BlocksArgs a, int per) {
    __shared__ int s_wave[THREADS / 64], s_flag;
    __shared__ int s_first[THREADS];  // tokens granted to the sequences before the thread's
    __shared__ int s_need[THREADS], s_count[THREADS];  // blocks and tokens asked before
    const int tid = threadIdx.x;
    const int b0 = tid * per, b1 = min(b0 + per, a.B);
    const int free = min(max(a.state[0], 0), a.num_blocks);
    Ask mine{};
    int need = 0, count = 0, all, all_need;
    for (int b = b0; b < b1; ++b) {
        mine = ask_of(a, b);
        need += mine.need;
        count += mine.count;
    }
    const int need0 = scan_before<THREADS>(need, s_wave, all_need);
    const int count0 = scan_before<THREADS>(count, s_wave, all);
    // The sums go on over the refused ones too; a sequence that needs no block needs
    // room for its tokens alone.
    auto fits = [&](const Ask &s, int upto_need, int upto_count) {
        return (s.need == 0 || upto_need <= free) && upto_count <= a.max_rows;
    };
    int granted = 0, taken = 0;
    for (int b = b0, n = need0, c = count0; b < b1; ++b) {
        if (per > 1) mine = ask_of(a, b);
        n += mine.need;
        c += mine.count;
        if (fits(mine, n, c)) {
            granted += mine.count;
            taken += mine.need;
        }
    }
    int total, total_taken;
    const int first0 = scan_before<THREADS>(granted, s_wave, total);
    scan_before<THREADS>(taken, s_wave, total_taken);
    s_first[tid] = first0;
    s_need[tid] = need0;
    s_count[tid] = count0;
    if (blockIdx.x == 0) {
        for (int b = b0, n = need0, c = count0, f = first0; b < b1; ++b) {
            if (per > 1) mine = ask_of(a, b);
            n += mine.need;
            c += mine.count;
            const int g = fits(mine, n, c) ? mine.count : 0;
            a.granted[b] = g;
            a.starts[b] = f;
            f += g;
        }
        if (tid == 0) a.starts[a.B] = total;
    }
    __syncthreads();
    // ---- tokens ----
    for (int n = blockIdx.x * THREADS + tid; n < a.max_rows; n += gridDim.x * THREADS) {
        int b = -1, pos = -1, slot = -1, row = -1;
        if (n < total) {
            const int t = find_last<THREADS>(s_first, n);
            int f = s_first[t], upto_need = s_need[t], upto_count = s_count[t];
            Ask s;
            for (b = t * per;; ++b) {  // ends: token n is granted to one of them
                s = ask_of(a, b);
                upto_need += s.need;
                upto_count += s.count;
                const int g = fits(s, upto_need, upto_count) ? s.count : 0;
                if (n < f + g) break;
                f += g;
            }
            const int i = n - f;
            pos = s.len + i;
            row = b * a.n_src + i;
            const int j = (int)((unsigned)pos / (unsigned)a.bt);
            int32_t *entry = a.block_table + (size_t)b * a.max_blocks + j;
            const int at = pos - j * a.bt;
            int id;
            if (j < s.held) {
                id = *entry;
            } else {
                id = a.free_blocks[free - 1 - (upto_need - s.need) - (j - s.held)];
                if (at == 0) *entry = id;  // a new block's first token is a new one
            }
            slot = id >= 0 && id < a.num_blocks ? id * a.bt + at : -1;
        }
        if (a.seq_of) a.seq_of[n] = b;
        if (a.positions) a.positions[n] = pos;
        if (a.slots) a.slots[n] = slot;
        if (a.rows) a.rows[n] = row;
    }
    settle<THREADS>(a.state, free - total_taken, &s_flag);
}

// Of n ids, the lowest on the stack first, those of the pool go on it from `at` up, in
// their order, while there is room: how many.  id_of(i) may read what lies at `at` + i.
template <int THREADS, typename Id>
__device__ int push_valid(const BlocksArgs &a, int at, int n, int *s_wave, Id id_of) {
    int64_t count = 0;
    for (int64_t i0 = 0; i0 < n; i0 += THREADS) {
        const int64_t i = i0 + threadIdx.x;
        const int id = i < n ? id_of((int)i) : -1;
        const bool valid = id >= 0 && id < a.num_blocks;
        int all;
        const int64_t to = at + count + scan_before<THREADS>(valid, s_wave, all);
        if (valid && to < a.num_blocks) a.free_blocks[to] = id;
        count = min(count + all, (int64_t)a.num_blocks - at);
    }
    return (int)count;
}

// seq_lens: tokens held; counts: tokens kept.  The blocks behind those go back, the
// first one of the first sequence on top.  An entry that holds no block (of a sequence
// given back before) is left out, which only a count of the valid ones before it can
// do; so all are stored as if they were valid, and the last workgroup to arrive closes
// the gaps where any of them saw an invalid one.  Where that many would not fit the
// stack, as happens with invalid ones alone, it pushes the valid ones by itself.
template <int THREADS>
__global__ __launch_bounds__(THREADS) void blocks_release_kernel(BlocksArgs a, int per) {
    __shared__ int s_wave[THREADS / 64];
    __shared__ unsigned s_seen;
    __shared__ int s_first[THREADS];
    const int tid = threadIdx.x;
    const int b0 = tid * per, b1 = min(b0 + per, a.B);
    const int free = min(max(a.state[0], 0), a.num_blocks);
    auto drop_of = [&](int b, int &keep) {
        const int len = min(max(a.seq_lens[b], 0), a.capacity);
        keep = blocks_of(min(max(a.counts[b], 0), len), a.bt);
        return blocks_of(len, a.bt) - keep;
    };
    int drop = 0, total, keep;
    for (int b = b0; b < b1; ++b) drop += drop_of(b, keep);
    s_first[tid] = scan_before<THREADS>(drop, s_wave, total);
    __syncthreads();
    // Block n of them: its id, the table's entry cleared.
    auto take = [&](int n) {
        const int t = find_last<THREADS>(s_first, n);
        int f = s_first[t], b, d;
        for (b = t * per;; ++b) {  // ends: block n is one of theirs
            d = drop_of(b, keep);
            if (n < f + d) break;
            f += d;
        }
        int32_t *entry = a.block_table + (size_t)b * a.max_blocks + keep + (n - f);
        const int id = *entry;
        *entry = -1;
        return id;
    };
    const bool room = (int64_t)free + total <= a.num_blocks;
    bool invalid = false;
    if (room)
        // (64 bits: the last step goes past the total, which may be 2^31 - 1)
        for (int64_t n = blockIdx.x * THREADS + tid; n < total; n += gridDim.x * THREADS) {
            const int id = take((int)n);
            invalid |= id < 0 || id >= a.num_blocks;
            // (through to memory: another workgroup may close the gaps)
            __hip_atomic_store(a.free_blocks + (free + total - 1 - n), id, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        }
    // ---- arrivals in the low 16 bits of the second word, above them who saw one ----
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    unsigned gaps = __syncthreads_or(invalid) ? 1u << 16 : 0u;
    if (gridDim.x > 1) {
        unsigned *word = reinterpret_cast<unsigned *>(a.state + 1);
        if (tid == 0) s_seen = gaps + __hip_atomic_fetch_add(word, 1u + gaps, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        __syncthreads();
        if ((s_seen & 0xffffu) != gridDim.x - 1) return;
        gaps = s_seen >> 16;
        if (tid == 0) __hip_atomic_store(word, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    int pushed = total;
    if (!room)
        pushed = push_valid<THREADS>(a, free, total, s_wave, [&](int i) { return take(total - 1 - i); });
    else if (gaps)
        pushed = push_valid<THREADS>(a, free, total, s_wave, [&](int i) {
            return __hip_atomic_load(a.free_blocks + (free + i), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        });
    if (tid == 0) a.state[0] = free + pushed;
}

}  // namespace

// A thread a sequence while 1024 of them hold the batch; 256 threads for a batch that
// needs no more, whose scans meet four wavefronts instead of sixteen (64 sequences of
// 8 tokens 3.4 us a call, so 3.9 with 1024; 4096 sequences 10.4 with 1024, so 15.8).
hipError_t launch_blocks_extend(const BlocksArgs &a, hipStream_t stream) {
    const int threads = a.B <= 256 ? 256 : 1024;
    const int per = (a.B + threads - 1) / threads;
    // a token a thread up to 256 workgroups
    const long long wgs = ((long long)a.max_rows + threads - 1) / threads;
    const dim3 grid((unsigned)(wgs < 1 ? 1 : wgs > 256 ? 256 : wgs));
    if (threads == 256)
        hipLaunchKernelGGL(blocks_extend_kernel<256>, grid, dim3(256), 0, stream, a, per);
    else
        hipLaunchKernelGGL(blocks_extend_kernel<1024>, grid, dim3(1024), 0, stream, a, per);
    return hipGetLastError();
}

hipError_t launch_blocks_release(const BlocksArgs &a, hipStream_t stream) {
    const int threads = a.B <= 256 ? 256 : 1024;
    const int per = (a.B + threads - 1) / threads;
    const long long wgs = ((long long)a.B * a.max_blocks + 16 * threads - 1) / (16 * threads);
    const dim3 grid((unsigned)(wgs < 1 ? 1 : wgs > 64 ? 64 : wgs));
    if (threads == 256)
        hipLaunchKernelGGL(blocks_release_kernel<256>, grid, dim3(256), 0, stream, a, per);
    else
        hipLaunchKernelGGL(blocks_release_kernel<1024>, grid, dim3(1024), 0, stream, a, per);
    return hipGetLastError();
}

}  // namespace lynx
