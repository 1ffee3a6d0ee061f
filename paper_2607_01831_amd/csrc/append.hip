// The cache written as tokens are kept, and read back (gfx950).
//
// A K group is 128 consecutive tokens of one channel, so its scale is known
// only when the group is whole.  Until then the group is open: its rows stay
// in BF16 too, in a ring of 256 rows per sequence (row t % 256 holds token t),
// and every append quantizes the whole open group again from them.  The cache
// is therefore at all times what lynx_kv_encode of the whole sequence gives,
// bit for bit, and the attention kernels need no case for an open group.  V
// groups are single tokens: only the new ones are quantized.
//
// What bounds it: a decode step's append moves at most 128 K rows of a head,
// so it is a chain of dependent loads (length, rows, group extrema, stores); a
// chunk of a prompt reads 4 bytes and writes 2 per element pair and is bound
// by memory: 4 x 4096 tokens of 8 heads 26.5 us into code planes (103 MB, 3.9 TB/s),
// 27.4 into anchors and residuals, 24.8 into anchors alone, 31.8 into all; one token
// of each of 16 sequences 7.1, and 7.7 into anchors and residuals; append_begin of
// those 5.5.
#include "lane_ops.h"
#include "lynx_internal.h"
#include "quantize.h"

namespace lynx {
namespace {

constexpr int kThreads = 256;
constexpr int kRing = kOpenRows;

// Row index of (kv head h, token t) of a sequence in a plane pool, or -1 where
// the block table names no valid block.
__device__ __forceinline__ long long pool_row(const Geometry &g, const int32_t *bt_row, int bt_shift, int h, int t) {
    const int bi = bt_shift >= 0 ? (t >> bt_shift) : t / g.bt;
    const int blk = bt_row[bi];
    if (blk < 0 || blk >= g.num_blocks) return -1;
    return ((long long)blk * g.Hkv + h) * g.bt + (t - bi * g.bt);
}

// Codes of 8 dims (8 m .. + 7) into every plane that the caller gave.
__device__ __forceinline__ void store_codes(const AppendArgs &a, int which, const float *x, const float *zero,
                                            const float *inv, long long row, int m) {
    const uint64_t c = quantize8(x, zero, inv);
    if (a.codes[which])
        __builtin_nontemporal_store(c, reinterpret_cast<uint64_t *>(a.codes[which] + row * kCodeRow + 8 * m));
    if (a.anc[which] || a.res[which]) {
        uint32_t an, rs;
        quantize_split8(x, zero, inv, an, rs);
        if (a.anc[which])
            __builtin_nontemporal_store(an, reinterpret_cast<uint32_t *>(a.anc[which] + row * kNibbleRow + 4 * m));
        if (a.res[which])
            __builtin_nontemporal_store(rs, reinterpret_cast<uint32_t *>(a.res[which] + row * kNibbleRow + 4 * m));
    }
}

__device__ __forceinline__ int opaque(int v) {
    asm volatile("" : "+v"(v));
    return v;
}

__device__ __forceinline__ uint4 load_once(const uint16_t *p) {
    const u32v4 x = __builtin_nontemporal_load(reinterpret_cast<const u32v4 *>(p));
    return make_uint4(x.x, x.y, x.z, x.w);
}

// Tokens appended to sequence b: the count, less what the cache has no room for
// and what follows the first entry of the path that names no row.
__device__ __forceinline__ int appended(const AppendArgs &a, int b, int T) {
    int n = min(max(0, min(a.counts[b], a.max_new)), a.capacity - T);
    if (a.path) {  // max_new <= 64: a lane per entry
        const int lane = threadIdx.x & 63;
        const int at = lane < n ? a.path[(size_t)b * a.max_new + lane] : 0;
        const uint64_t off = __ballot(at < 0 || at >= a.n_src);
        if (off) n = min(n, __ffsll((long long)off) - 1);
    }
    return n;
}

// One workgroup: the 128-token group u of the groups that sequence b's new
// tokens fall into (0 is the open one), of kv head h, of K (which 0) or V (1).
// Thread (tr = tid / 16, m = tid % 16) owns dims 8 m .. + 7 of the group's
// tokens tr, tr + 16, ..., so that a token's row is 16 lanes and every load and
// store of a wavefront covers whole rows; its 8 rows are all loaded before any
// is used, the new ones past the caches (each is read once).
__global__ __launch_bounds__(kThreads, 4) void append_kernel(AppendArgs a) {
    const int h = blockIdx.x >> 1, which = blockIdx.x & 1;
    const int u = blockIdx.y, b = blockIdx.z;
    const int tid = threadIdx.x, m = tid & 15, tr = tid >> 4, wave = tid >> 6;
    const int Hkv = a.geo.Hkv;
    const int T = min(max(a.seq_lens[b], 0), a.capacity);
    const int n_new = appended(a, b, T);
    const int end = T + n_new;
    const int g0 = T / kKGroup, g = g0 + u;
    const int t0 = g * kKGroup;
    if (n_new == 0 || t0 >= end) return;
    const int n = min(kKGroup, end - t0);  // tokens of the group
    const int n_old = max(0, T - t0);      // of them in the cache already

    const int32_t *bt_row = a.block_table + (size_t)b * a.geo.max_blocks;
    const uint16_t *src = which == 0 ? a.k_new : a.v_new;
    const size_t row_stride = (size_t)Hkv * kHeadDim;
    const uint16_t *fresh = src + (size_t)b * a.n_src * row_stride + (size_t)h * kHeadDim + 8 * m;
    uint16_t *ring = a.k_open + (size_t)b * kRing * row_stride + (size_t)h * kHeadDim + 8 * m;
    auto new_row = [&](int t) {  // the new row of token t >= T
        const int i = t - T;
        return fresh + (size_t)(a.path ? a.path[(size_t)b * a.max_new + i] : i) * row_stride;
    };

    // rows past the group's last repeat it; V's rows before the first new one
    // repeat that
    uint4 raw[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int tl = min(tr + 16 * i, n - 1);
        if (which == 0 && tl < n_old)
            raw[i] = *reinterpret_cast<const uint4 *>(ring + (size_t)((t0 + tl) % kRing) * row_stride);
        else
            raw[i] = load_once(new_row(t0 + max(tl, n_old)));
    }

    // what follows has its own row numbers: kept through the loads, the addresses
    // of all rows would be held in registers
    const int row0 = opaque(tr);
    if (which == 1) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int tl = row0 + 16 * i;
            float x[8];
            unpack8(raw[i], x);
            const float mn = row16_min(fmin3(fmin3(x[0], x[1], x[2]), fmin3(x[3], x[4], x[5]), fmin2(x[6], x[7])));
            const float mx = row16_max(fmax3(fmax3(x[0], x[1], x[2]), fmax3(x[3], x[4], x[5]), fmax2(x[6], x[7])));
            if (tl < n_old || tl >= n) continue;
            const int t = t0 + tl;
            float zero, scale, inv;
            group_params(mn, mx, zero, scale, inv);
            if (m == 0) {
                const size_t mi = ((size_t)b * Hkv + h) * a.geo.max_tokens + t;
                a.meta.v_scale[mi] = scale;
                a.meta.v_zero[mi] = zero;
            }
            const long long row = pool_row(a.geo, bt_row, a.bt_shift, h, t);
            if (row < 0) continue;
            const float z8[8] = {zero, zero, zero, zero, zero, zero, zero, zero};
            const float i8[8] = {inv, inv, inv, inv, inv, inv, inv, inv};
            store_codes(a, 1, x, z8, i8, row, m);
        }
        return;
    }

    __shared__ float s_min[4][kHeadDim], s_max[4][kHeadDim];
    __shared__ float s_zero[kHeadDim], s_inv[kHeadDim];
    // two tokens at a time: the whole window as floats would take 64 registers
    float kmin[8], kmax[8];
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
        float x[8], y[8];
        unpack8(raw[i], x);
        unpack8(raw[i + 1], y);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            kmin[j] = i == 0 ? fmin2(x[j], y[j]) : fmin3(kmin[j], x[j], y[j]);
            kmax[j] = i == 0 ? fmax2(x[j], y[j]) : fmax3(kmax[j], x[j], y[j]);
        }
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        kmin[j] = min_kg(kmin[j]);
        kmax[j] = max_kg(kmax[j]);
    }
    if ((tid & 63) < 16) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            s_min[wave][8 * m + j] = kmin[j];
            s_max[wave][8 * m + j] = kmax[j];
        }
    }
    __syncthreads();  // every row that this workgroup reads from the ring is in registers
    if (tid < kHeadDim) {
        const float mn = fmin2(fmin2(s_min[0][tid], s_min[1][tid]), fmin2(s_min[2][tid], s_min[3][tid]));
        const float mx = fmax2(fmax2(s_max[0][tid], s_max[1][tid]), fmax2(s_max[2][tid], s_max[3][tid]));
        float zero, scale, inv;
        group_params(mn, mx, zero, scale, inv);
        s_zero[tid] = zero;
        s_inv[tid] = inv;
        const size_t mi = (((size_t)b * Hkv + h) * a.geo.n_groups + g) * kHeadDim + tid;
        a.meta.k_scale[mi] = scale;
        a.meta.k_zero[mi] = zero;
    }
    __syncthreads();

    // ---- the ring: the rows of the last group begun, ge, and of the one before
    // it.  Group g's rows stand in the half g % 2, which the open group's
    // workgroup (u = 0) reads while the others run: a later group of the same
    // half is left to that workgroup, which has its rows by now. ----
    const int ge = end / kKGroup;
    const bool old_rows = T % kKGroup != 0;  // the open group has rows in the ring
    const bool keep = g >= ge - 1 && (u == 0 || !old_rows || ((g ^ g0) & 1));
    float kz[8], ki[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        kz[j] = s_zero[8 * m + j];
        ki[j] = s_inv[8 * m + j];
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int tl = row0 + 16 * i;
        if (tl >= n) continue;
        if (keep && tl >= n_old) *reinterpret_cast<uint4 *>(ring + (size_t)((t0 + tl) % kRing) * row_stride) = raw[i];
        const long long row = pool_row(a.geo, bt_row, a.bt_shift, h, t0 + tl);
        if (row < 0) continue;
        // (not the floats of the extrema: those would be held from there on)
        asm volatile("" : "+v"(raw[i].x), "+v"(raw[i].y), "+v"(raw[i].z), "+v"(raw[i].w));
        float x[8];
        unpack8(raw[i], x);
        store_codes(a, 0, x, kz, ki, row, m);
    }
    if (u != 0 || !old_rows) return;
    for (int later = max(g0 + 2, ge - 1); later <= ge; ++later) {
        if ((later ^ g0) & 1) continue;
        for (int t = later * kKGroup + tr; t < min(end, (later + 1) * kKGroup); t += 16)
            *reinterpret_cast<uint4 *>(ring + (size_t)(t % kRing) * row_stride) =
                *reinterpret_cast<const uint4 *>(new_row(t));
    }
}

// Two floats -> two BF16, rounded to nearest even, a in the low half.
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
    typedef float f32v2 __attribute__((ext_vector_type(2)));
    typedef __bf16 bf16v2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32v2){a, b}, bf16v2));
}

// Reads tokens back: x = fma(code, scale, zero), rounded to BF16 to nearest
// even.  Bound by memory: 132 bytes read and 256 written per row, and it is the
// writes that have to be whole: a token's rows of all kv heads stand side by
// side, so a workgroup takes HEADS heads of a few tokens and writes runs of 256
// HEADS bytes (a workgroup per head of 128 tokens, runs of 256 bytes: 161 us for
// 103K tokens of 8 heads in two sequences).  Thread (row tid / 16 of 16: token, head; dims
// 8 m .. + 7) keeps its head's K scales and zeros, and loads its PASSES tokens'
// codes before it uses any.  Codes and values go past the caches: those tokens 124 us
// (645 MB, 5.2 TB/s, a copy's rate), with cached loads 147, cached stores too 155;
// 2 x 65536 tokens 159 us (822 MB, 5.2 TB/s).
// RING: K alone, the open group and the one before it, into the ring; else
// tokens starts[b] .. + counts[b] - 1, to row t - starts[b] of the output.
template <bool RING, int HEADS, int PASSES>
__global__ __launch_bounds__(kThreads) void dequant_kernel(DequantArgs a) {
    constexpr int kStep = 16 / HEADS;        // tokens per pass
    constexpr int kTokens = kStep * PASSES;  // tokens per workgroup, inside one K group
    const int which = RING ? 0 : blockIdx.x & 1, h0 = (RING ? blockIdx.x : blockIdx.x >> 1) * HEADS;
    const int u = a.unit0 + blockIdx.y, b = blockIdx.z;
    const int tid = threadIdx.x, m = tid & 15, h = h0 + (tid >> 4) % HEADS, tr = (tid >> 4) / HEADS;
    const int Hkv = a.geo.Hkv;
    int first, end;
    if (RING) {
        end = min(max(a.starts[b], 0), a.capacity);  // the sequence's length
        first = max(0, end / kKGroup - 1) * kKGroup;
    } else {
        first = a.starts[b];
        if (first < 0 || first >= a.capacity) return;
        end = first + min(max(0, min(a.counts[b], a.max_n)), a.capacity - first);
    }
    const int t0 = first / kTokens * kTokens + u * kTokens;
    const int lo = max(first, t0), hi = min(end, t0 + kTokens);
    if (lo >= hi) return;
    const int32_t *bt_row = a.block_table + (size_t)b * a.geo.max_blocks;
    const uint8_t *codes = which == 0 ? a.k_codes : a.v_codes;
    const size_t vm = ((size_t)b * Hkv + h) * a.geo.max_tokens;
    uint2 c[PASSES];
    float2 sz[PASSES];
    bool live[PASSES], held[PASSES];  // written; in the pool
#pragma unroll
    for (int i = 0; i < PASSES; ++i) {
        const int at = t0 + tr + kStep * i, t = min(max(at, lo), hi - 1);  // rows outside the range repeat its nearest
        const long long row = pool_row(a.geo, bt_row, a.bt_shift, h, t);
        held[i] = row >= 0;
        live[i] = at == t && (RING || row >= 0);
        typedef unsigned int u32v2 __attribute__((ext_vector_type(2)));
        const u32v2 x = __builtin_nontemporal_load(
            reinterpret_cast<const u32v2 *>(codes + (row < 0 ? 0 : row) * kCodeRow + 8 * m));
        c[i] = make_uint2(x.x, x.y);
        if (which == 1) sz[i] = make_float2(a.meta.v_scale[vm + t], a.meta.v_zero[vm + t]);
    }
    float sc[8], zr[8];
    if (which == 0) {
        const size_t km = (((size_t)b * Hkv + h) * a.geo.n_groups + t0 / kKGroup) * kHeadDim + 8 * m;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            sc[j] = a.meta.k_scale[km + j];
            zr[j] = a.meta.k_zero[km + j];
        }
    }
    uint16_t *out = (which == 0 ? a.k_out : a.v_out) + (size_t)b * (RING ? kRing : a.max_n) * Hkv * kHeadDim;
#pragma unroll
    for (int i = 0; i < PASSES; ++i) {
        if (which == 1) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                sc[j] = sz[i].x;
                zr[j] = sz[i].y;
            }
        }
        u32v4 o;
#pragma unroll
        for (int j = 0; j < 8; j += 2) {
            const uint32_t w = (j < 4 ? c[i].x : c[i].y) >> (8 * (j & 3));
            o[j / 2] = pack_bf16(fmaf((float)(w & 0xFFu), sc[j], zr[j]), fmaf((float)((w >> 8) & 0xFFu), sc[j + 1], zr[j + 1]));
        }
        if (RING && !held[i]) o = u32v4{0u, 0u, 0u, 0u};  // (the rows of a group decide its scale)
        const int t = t0 + tr + kStep * i;
        const size_t to = RING ? (size_t)(t % kRing) : (size_t)(t - first);
        u32v4 *p = reinterpret_cast<u32v4 *>(out + (to * Hkv + h) * kHeadDim + 8 * m);
        if (live[i]) __builtin_nontemporal_store(o, p);
    }
}

template <bool RING, int HEADS>
void launch_dequant_heads(DequantArgs a, int B, int rows, hipStream_t stream) {
    constexpr int kPasses = 4;  // (8: 139 us for 103K tokens, 8.9 for 16 x 128; 4: 124 and 4.7)
    constexpr int kTokens = 16 / HEADS * kPasses;
    static_assert(kKGroup % kTokens == 0, "a workgroup stays in one K group");
    constexpr int kMostUnits = 65535;  // of a grid; more rows (524K at 8 heads) take a launch more
    const int units = (rows + 2 * kTokens - 2) / kTokens;
    for (a.unit0 = 0; a.unit0 < units; a.unit0 += kMostUnits)
        hipLaunchKernelGGL((dequant_kernel<RING, HEADS, kPasses>),
                           dim3((RING ? 1 : 2) * a.geo.Hkv / HEADS, min(kMostUnits, units - a.unit0), B),
                           dim3(kThreads), 0, stream, a);
}
template <bool RING>
hipError_t launch_dequant_any(const DequantArgs &a, int B, int rows, hipStream_t stream) {
    if (a.geo.Hkv % 8 == 0)
        launch_dequant_heads<RING, 8>(a, B, rows, stream);
    else if (a.geo.Hkv % 4 == 0)
        launch_dequant_heads<RING, 4>(a, B, rows, stream);
    else if (a.geo.Hkv % 2 == 0)
        launch_dequant_heads<RING, 2>(a, B, rows, stream);
    else
        launch_dequant_heads<RING, 1>(a, B, rows, stream);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_append(const AppendArgs &a, int B, hipStream_t stream) {
    // groups that max_new tokens can touch, whatever the length before
    const unsigned units = (unsigned)((a.max_new + 2 * kKGroup - 2) / kKGroup);
    hipLaunchKernelGGL(append_kernel, dim3(2 * a.geo.Hkv, units, B), dim3(kThreads), 0, stream, a);
    return hipGetLastError();
}

hipError_t launch_dequant(const DequantArgs &a, int B, hipStream_t stream) {
    return launch_dequant_any<false>(a, B, a.max_n, stream);
}

hipError_t launch_append_begin(const DequantArgs &a, int B, hipStream_t stream) {
    return launch_dequant_any<true>(a, B, kRing, stream);
}

}  // namespace lynx
