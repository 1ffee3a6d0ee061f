// Verification over the merged cache for many query rows a kv head (gfx950 MFMA,
// fp16 operands): the context part of a wide token tree.
//
// What it computes is verify.hip's: the partial (max, sum, output) of every row
// over a segment of the context.  There a wavefront folds the K scales into its
// own rows' queries, group by group, and unpacks K and V for itself, which costs
// as many vector instructions per (row, token) as the softmax does.  With 100 rows
// and more the keys are the smaller side: here the workgroup's 8 wavefronts share
// the tokens and split the rows, 32 each, so that a tile's K and V are
// reconstructed once for 256 rows (or 128), as fp16 in the matrix cores' operand
// order in LDS, and the queries are converted once.
//
// Operands:
//  * K' = (zero + code scale - c) 2^(14 - e_d), e_d the exponent of the largest |K| of
//    channel d in the segment (from the metadata), c a number inside the range of the
//    group: 0 at first, and from group to group moved to the range's end where it is
//    outside, so |K'| <= 2^15.  K' is computed in fp32 and rounded to fp16 once: a key is off by 2^-12
//    of its group's range at most, a sixteenth of a code's step (of itself where c is
//    0; and by 2^-39 of the channel's largest where it is a subnormal).  So neither
//    what the keys of a group have in common, which the softmax does not see, nor a
//    token far from the others takes bits from the rest.  sum_d q_d c_d, of exact
//    products (c has fp16's 11 bits), is added to the scores in fp32, where they
//    become weights; it is computed again where a c has moved (each time: 3 % more).
//  * the query is q_d 2^(e_d - E + 15), E the exponent of the row's largest product:
//    exact in fp16 (BF16 has 8 significant bits) down to 2^-32 of the largest.
//  * V' = (zero + code scale) 2^(15 - Ev), Ev the exponent of the segment's largest
//    |V|, rounded to fp16: off by 2^-12 of itself, and by 2^-40 of the largest where
//    it is a subnormal (the largest stands at fp16's upper end, 2^15, so that one
//    token's large values leave the others their bits).
//  * weights 2^8 p against a reference that follows the row's maximum once it is 2^7
//    behind, so up to 2^15, rounded to fp16: off by 2^-12 of themselves, or by 2^-33 of
//    the row's largest; l sums the rounded weights, so that an output is a mean by
//    them, in fp32.
//
// A step is a tile of 32 tokens for 256 rows, or, for half the rows, two tiles
// with a wavefront's two partners each on one (TS 2; they join at the end).  A
// tile costs a wavefront 34 MFMAs for its 32 rows (two of them sum the weights,
// as a column of ones behind the values).  Iteration j: copies of step j + 4 into
// LDS (asynchronous), what step j + 3 needs of its metadata, the scores of step
// j + 1 in turns with the weights of step j, the products with the values in turns
// with the conversion of step j + 2; one barrier.  2 x 64K tokens, 8 kv heads, with
// the merge: 512 rows 352 us (verify.hip's kernel 552), 128 rows 128 (169).  What
// bounds it: no unit alone.  By its counters (512 rows) a wavefront's tile has 34
// MFMAs, 124 other vector instructions and 29 of LDS, and of the 2950 cycles that it
// takes the matrix cores are busy 37%, the vector units 47%, LDS 34%; behind an
// MFMA's 16 cycles two vector instructions are free and each further one takes 5,
// 1650 cycles for a SIMD's two wavefronts, and the rest are the barrier and the waits
// around it.  Tried: fragments and codes read a step ahead of the barrier (347 and
// 170 us where 341 and 139 were: registers), four wavefronts of 32 rows twice on a CU
// (470), four of 64 rows (627), 128 rows by 16 a wavefront (152), two orders of the
// stretches for the wavefronts of a SIMD (444), conversions by v_fma_mix (357 for
// 350).
#include "f16_ops.h"
#include "lane_ops.h"
#include "lynx_internal.h"
#include "work_list.h"

#include <float.h>
#include <math.h>

namespace lynx {
namespace {

constexpr int kWaves = 8;
constexpr int kThreads = 64 * kWaves;
static_assert(kWideRows == 32 * kWaves, "two row tiles per wavefront");
constexpr int kTile = 32;  // tokens
constexpr float kLog2e = 1.4426950408889634f;
constexpr int kRawPlane = kTile * kCodeRow;         // 4 KB of codes
constexpr int kRawBytes = 2 * kRawPlane;
constexpr int kMetaSlots = 8;                       // steps that V metadata is kept of
constexpr int kFragBytes = 8 * 1024;                // a tile's 8 fragments of K, or of V
constexpr int kFragsV = 3;                          // V's buffers; K's are two
constexpr int kDepth = 4;                           // steps whose copies are in flight or not converted yet
constexpr int kUpper = 15;                          // fp16 operands reach up to 2^15
constexpr int kUpperK = kUpper - 1;                 // keys before c is taken off, which may be at the other end
constexpr float kSlack = 7.0f;                      // log2 units that the reference may lag behind
constexpr float kLift = kUpper - kSlack;            // ... that weights are held above it

// TS: tiles of a step, one for each TS-th of the wavefronts.
template <int LAYOUT, int TS>
__device__ __forceinline__ void wide_segment(const VerifyArgs &a, const Segment<kWorkUnit> &seg, int h, int chunk,
                                             const int tid) {
    const int Hkv = a.geo.Hkv;
    constexpr int kRows = kWideRows / TS;
    constexpr int kTilesPerGroup = kKGroup / kTile;
    static_assert(kTilesPerGroup % (2 * TS) == 0, "two steps stay in one K group");
    constexpr int kSteps = kTilesPerGroup / TS;  // per group
    const int lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6), col = lane & 15, kg = lane >> 4;
    const int b = seg.b, T = seg.T, g0 = seg.g0;
    const int ts = w / (kWaves / TS);                            // the wavefront's tile of a step
    const int row0 = chunk * kRows + 32 * (w % (kWaves / TS));  // its rows
    auto partial_index = [&](int r) { return ((size_t)h * a.rows_total + r) * a.n_seg + seg.number; };
    if (seg.n_groups == 0) {  // an empty sequence: (max, sum) = (-inf, 0)
        for (int r = chunk * kRows + tid; r < min(a.rows_total, (chunk + 1) * kRows); r += kThreads)
            a.ws_ml[partial_index(r)] = make_float2(-INFINITY, 0.0f);
        return;
    }
    const int first = g0 * kKGroup, end = min(T, first + seg.n_groups * kKGroup);
    const int n_steps = (end - first + kTile * TS - 1) / (kTile * TS);

    __shared__ __attribute__((aligned(16))) uint8_t s_raw[kDepth][TS][kRawBytes];
    __shared__ __attribute__((aligned(16))) uint8_t s_frag[2 + kFragsV][TS][kFragBytes];
    __shared__ __attribute__((aligned(16))) float s_vm[kMetaSlots][TS][2 * kTile];  // a tile's V scale | zero
    __shared__ __attribute__((aligned(16))) float s_km[3][2 * kHeadDim];  // K scale | zero of a group, three groups
    __shared__ int32_t s_ids[LAYOUT == 0 ? 1 : kWaves][2 * kDepth][TS][8];  // blocks of a step's rows
    __shared__ int s_e[kHeadDim];                                       // channel exponents
    // of two groups: scale and zero - c of the conversion, and c
    __shared__ __attribute__((aligned(16))) float s_kp[2][2][kHeadDim];
    __shared__ __attribute__((aligned(16))) _Float16 s_c[2][kHeadDim];
    __shared__ __attribute__((aligned(8))) int s_moved[2][2];  // by half the channels
    __shared__ float s_vmax[kWaves];
    float(*s_max)[kHeadDim] = reinterpret_cast<float(*)[kHeadDim]>(&s_frag[0][0][0]);  // (before there are fragments)
    auto frag_k = [&](int j) { return s_frag[j & 1]; };
    auto frag_v = [&](int j) { return s_frag[2 + j % kFragsV]; };

    const int32_t *bt_row = a.block_table + (size_t)b * a.geo.max_blocks;
    const size_t vmeta = ((size_t)b * Hkv + h) * a.geo.max_tokens;
    const size_t kmeta = ((size_t)b * Hkv + h) * a.geo.n_groups * kHeadDim;
    bool bad = false;

    // ---- copies ----
    // A row per 8 lanes; lane l fills physical chunk l % 8 of its row.
    const int crow = lane >> 3;
    auto block_of = [&](int t) { return a.bt_shift >= 0 ? t >> a.bt_shift : t / a.geo.bt; };
    auto place_in = [&](int t) { return a.bt_shift >= 0 ? t & (a.geo.bt - 1) : t % a.geo.bt; };
    // row numbers in 32 bits: 2^32 rows of codes would be 512 GB
    const uint32_t block_rows = (uint32_t)Hkv * a.geo.bt, head_rows = (uint32_t)h * a.geo.bt;
    auto token_of = [&](int j, int k) { return min(first + kTile * (TS * j + k) + 8 * (w & 3) + crow, T - 1); };
    // Every wavefront issues as many operations per step, so that it can wait for
    // the older ones: for each tile a copy of rows, one of metadata (of the next step:
    // K's where a group begins, by wavefront TS; else V's of tile w % TS, which may be
    // written more than once), and the block numbers of a later step.
    // Wavefront w copies rows 8 (w % 4) .. + 7 of K (w < 4) or V.
    constexpr int kOps = TS + (LAYOUT == 0 ? 1 : 2);
    auto copy_ids = [&](int j) {
        if (LAYOUT != 0 && lane < 8 * TS) {
            const int t = min(first + kTile * (TS * j + (lane >> 3)) + 8 * (w & 3) + (lane & 7), T - 1);
            lds_copy4(bt_row + block_of(t), lds_addr(&s_ids[LAYOUT == 0 ? 0 : w][j % (2 * kDepth)][0][0]));
        }
    };
    // logical chunk of the physical one that the lane fills, in bytes
    const uint32_t chunk_off = 16u * (uint32_t)((lane & 7) ^ crow ^ (w < 4 ? 0 : ((w & 3) >> 1) << 2));
    const int id0 = LAYOUT == 0 ? bt_row[0] : 0;
    if (LAYOUT == 0) bad = id0 < 0 || id0 >= a.geo.num_blocks;
    const size_t blk0 = ((size_t)(bad ? 0 : id0) * Hkv + h) * a.geo.bt;  // (LAYOUT 0) the sequence's first row
    const uint32_t km0 = lds_addr(&s_km[0][0]);
    const uint32_t raw0 = lds_addr(&s_raw[0][0][0]);
    auto raw_of = [&](int j, int k) { return raw0 + (uint32_t)((j % kDepth) * TS + k) * kRawBytes; };
    auto copy_km = [&](int g) {
        lds_copy16((lane < 32 ? a.meta.k_scale : a.meta.k_zero) + kmeta + (size_t)(g0 + g) * kHeadDim + 4 * (lane & 31),
                   km0 + (uint32_t)(g % 3) * 2 * kHeadDim * 4);
    };
    auto copy_vm = [&](int j) {
        const int tt = min(first + kTile * (TS * j + w % TS) + (lane & 31), T - 1);
        lds_copy4((lane < 32 ? a.meta.v_scale : a.meta.v_zero) + vmeta + tt, lds_addr(&s_vm[j % kMetaSlots][w % TS][0]));
    };
    auto issue = [&](int j, auto id_of) {
        if (j >= n_steps) return;
#pragma unroll
        for (int k = 0; k < TS; ++k) {
            const uint8_t *codes = w < 4 ? a.k_codes : a.v_codes;
            if (LAYOUT == 0) {  // rows side by side: the first one's address is the wavefront's
                const int t = min(first + kTile * (TS * j + k) + 8 * (w & 3), T - 1);
                lds_copy16(codes + (blk0 + t) * kCodeRow, (uint32_t)(min(crow, T - 1 - t) * kCodeRow) + chunk_off,
                           raw_of(j, k) + 1024u * w);
                continue;
            }
            const int t = token_of(j, k);
            int id = id_of(k);
            if (id < 0 || id >= a.geo.num_blocks) {
                bad = true;
                id = 0;
            }
            lds_copy16(codes + (size_t)((uint32_t)id * block_rows + head_rows + place_in(t)) * kCodeRow + chunk_off,
                       raw_of(j, k) + 1024u * w);
        }
        if (w == TS && (j + 1) % kSteps == 0 && j + 1 < n_steps)
            copy_km((j + 1) / kSteps);
        else
            copy_vm(j + 1);
        copy_ids(j + kDepth);
    };

    // ---- the exponents of the segment's channels and of its values ----
    {
        int ids[kDepth][TS];
#pragma unroll
        for (int j = 0; j < kDepth; ++j)
#pragma unroll
            for (int k = 0; k < TS; ++k) ids[j][k] = LAYOUT == 0 ? 0 : bt_row[block_of(token_of(j, k))];
#pragma unroll
        for (int j = 0; j < kDepth; ++j) issue(j, [&](int k) { return ids[j][k]; });
        if (w == TS) copy_km(0);
        copy_vm(0);
    }
    // the wavefront's queries: row col of each row tile, dims 8 kg + 32 kk
    uint4 qraw[2][4];
#pragma unroll
    for (int rt = 0; rt < 2; ++rt) {
        const int r = min(row0 + 16 * rt + col, a.rows_total - 1);
        const uint16_t *q = a.q + (((size_t)b * a.nq + r / a.G) * a.Hq + (size_t)h * a.G + r % a.G) * kHeadDim + 8 * kg;
#pragma unroll
        for (int kk = 0; kk < 4; ++kk) qraw[rt][kk] = *reinterpret_cast<const uint4 *>(q + 32 * kk);
    }
    {
        float4 m = make_float4(0.f, 0.f, 0.f, 0.f);
        const int d4 = tid & 31, gg = tid >> 5;  // 4 channels; groups gg, gg + 2 kWaves, ...
        // (several loads in flight; past the segment's end its last is read again)
        for (int g1 = gg; g1 < seg.n_groups; g1 += 4 * 2 * kWaves) {
            float4 s[4], z[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const size_t at = kmeta + (size_t)(g0 + min(g1 + 2 * kWaves * i, seg.n_groups - 1)) * kHeadDim;
                s[i] = reinterpret_cast<const float4 *>(a.meta.k_scale + at)[d4];
                z[i] = reinterpret_cast<const float4 *>(a.meta.k_zero + at)[d4];
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                m.x = fmax3_abs(m.x, z[i].x, fmaf(255.0f, s[i].x, z[i].x));
                m.y = fmax3_abs(m.y, z[i].y, fmaf(255.0f, s[i].y, z[i].y));
                m.z = fmax3_abs(m.z, z[i].z, fmaf(255.0f, s[i].z, z[i].z));
                m.w = fmax3_abs(m.w, z[i].w, fmaf(255.0f, s[i].w, z[i].w));
            }
        }
        reinterpret_cast<float4 *>(s_max[gg])[d4] = m;
        float v = 0.0f;
        for (int t1 = first + tid; t1 < end; t1 += 8 * kThreads) {
            float s[8], z[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const size_t at = vmeta + min(t1 + kThreads * i, end - 1);
                s[i] = a.meta.v_scale[at];
                z[i] = a.meta.v_zero[at];
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) v = fmax3_abs(v, z[i], fmaf(255.0f, s[i], z[i]));
        }
        v = max_kg(row16_max(v));
        if (lane == 0) s_vmax[w] = v;
        __syncthreads();
        if (tid < kHeadDim) {
            float x = s_max[0][tid];
#pragma unroll
            for (int i = 1; i < 2 * kWaves; ++i) x = fmax2(x, s_max[i][tid]);
            // a channel of zeros takes no part, whatever the queries hold there
            int e = x > 0.0f ? 0 : -10000;
            if (x > 0.0f && x <= FLT_MAX) frexpf(x, &e);
            s_e[tid] = e;
        }
    }
    int Ev = 0;
    {
        float v = s_vmax[0];
#pragma unroll
        for (int i = 1; i < kWaves; ++i) v = fmax2(v, s_vmax[i]);
        if (v > 0.0f && v <= FLT_MAX) frexpf(v, &Ev);
        Ev = min(max(Ev, kUpper + (int)kLift - 126), 126);  // 2^(Ev - kUpper - kLift) is a normal number
    }
    __syncthreads();

    // ---- the queries as operands ----
    u32x4_t qf[2][4];
    float sc[2];
#pragma unroll
    for (int rt = 0; rt < 2; ++rt) {
        uint32_t x[4][4];  // two queries each
#pragma unroll
        for (int kk = 0; kk < 4; ++kk) {
            x[kk][0] = qraw[rt][kk].x;
            x[kk][1] = qraw[rt][kk].y;
            x[kk][2] = qraw[rt][kk].z;
            x[kk][3] = qraw[rt][kk].w;
        }
        // the exponent of the row's largest product with a key (an upper bound where
        // the query is subnormal), from the exponents of both: the products
        // themselves may leave the range of fp32
        constexpr int kNone = -20000;
        int E = kNone;
#pragma unroll
        for (int kk = 0; kk < 4; ++kk)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int d = 32 * kk + 8 * kg + 2 * e;
                const int lo = (int)(x[kk][e] >> 7 & 0xFFu) + s_e[d], hi = (int)(x[kk][e] >> 23 & 0xFFu) + s_e[d + 1];
                E = max(E, max(x[kk][e] & 0x7FFFu ? lo : kNone, x[kk][e] & 0x7FFF0000u ? hi : kNone));
            }
        E = max(E, __shfl_xor(E, 16));
        E = max(E, __shfl_xor(E, 32)) - 126;
#pragma unroll
        for (int kk = 0; kk < 4; ++kk)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int d = 32 * kk + 8 * kg + 2 * e;
                qf[rt][kk][e] = pack_f16_rne(ldexpf(bf16_lo(x[kk][e]), s_e[d] - E + kUpper),
                                             ldexpf(bf16_hi(x[kk][e]), s_e[d + 1] - E + kUpper));
            }
        // positive and finite: times the -inf of a token past the context it must
        // not be a NaN
        sc[rt] = __builtin_amdgcn_fmed3f(ldexpf(kLog2e * rsqrtf((float)kHeadDim), E - kUpper - kUpperK), FLT_MIN, FLT_MAX);
    }

    // ---- conversion of a step into operand order ----
    // K: fragment 4 r + kk: lane (token 16 r + col, dims 32 kk + 8 kg .. + 7); V:
    // fragment c: lane (dim 16 c + col, tokens 16 (e / 4) + 4 kg + e % 4).  Wavefront
    // w makes fragment w of each.
    const int kk_own = w & 3;
    auto prepare = [&](int g) {  // a thread per channel
        if (w >= kHeadDim / 64) return;
        const float *km = s_km[g % 3];
        const int up = kUpperK - s_e[tid];
        const float scale = ldexpf(km[tid], up), zero = ldexpf(km[kHeadDim + tid], up);
        const float was = g > 0 ? (float)s_c[~g & 1][tid] : 0.0f;
        const _Float16 c = (_Float16)__builtin_amdgcn_fmed3f(was, zero, fmaf(255.0f, scale, zero));
        const bool moved = __any((float)c != was);
        if (lane == 0) s_moved[g & 1][w] = moved;
        s_kp[g & 1][0][tid] = scale;
        s_kp[g & 1][1][tid] = zero - (float)c;
        s_c[g & 1][tid] = c;
    };
    // The queries' products with the c of step j's group, as those with a tile whose
    // tokens are all c: what its scores are off by, times their scale.
    float off[2] = {0.0f, 0.0f};
    auto load_off = [&](int j) {
        f32x4_t x[2] = {};
#pragma unroll
        for (int kk = 0; kk < 4; ++kk) {
            const u32x4_t c = *reinterpret_cast<const u32x4_t *>(&s_c[(j / kSteps) & 1][32 * kk + 8 * kg]);
#pragma unroll
            for (int rt = 0; rt < 2; ++rt) x[rt] = mfma_f16(c, qf[rt][kk], x[rt]);
        }
#pragma unroll
        for (int rt = 0; rt < 2; ++rt) off[rt] = x[rt][0] * sc[rt];
    };
    const float down = ldexpf(1.0f, kUpper - Ev);
    auto prepare_v = [&](int j) {
        if (w < TS) s_vm[j % kMetaSlots][w][lane] *= down;
    };
    // (of a step past the last: what its slot holds, to where nothing reads)
    struct Raw {
        uint2 k;
        intx2_t v;
        float4 s[2], z[2], ks[2], kz[2];
    };
    auto load_raw = [&](int j, int k) {
        const int t = 16 * (w >> 2) + col, q = 2 * kk_own + (kg >> 1);
        const int tr = 16 * ((col >> 1) >> 2) + 4 * kg + ((col >> 1) & 3);
        const uint8_t *p = s_raw[j % kDepth][k];
        const float *vm = &s_vm[j % kMetaSlots][k][4 * kg];
        Raw r;
        r.k = *reinterpret_cast<const uint2 *>(p + t * kCodeRow + ((q ^ (t & 7)) * 16) + 8 * (kg & 1));
        r.v = __builtin_amdgcn_ds_read_tr8_b64_v2i32(
            (__attribute__((address_space(3))) intx2_t *)(p + kRawPlane + v_slot(tr, w) + 8 * (col & 1)));
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            r.s[i] = *reinterpret_cast<const float4 *>(vm + 16 * i);
            r.z[i] = *reinterpret_cast<const float4 *>(vm + kTile + 16 * i);
            const float *kp = &s_kp[(j / kSteps) & 1][0][32 * kk_own + 8 * kg + 4 * i];
            r.ks[i] = *reinterpret_cast<const float4 *>(kp);
            r.kz[i] = *reinterpret_cast<const float4 *>(kp + kHeadDim);
        }
        return r;
    };
    auto convert = [&](int j, int k, const Raw &raw) {
        u32x4_t o;
        const float ks[8] = {raw.ks[0].x, raw.ks[0].y, raw.ks[0].z, raw.ks[0].w, raw.ks[1].x, raw.ks[1].y, raw.ks[1].z, raw.ks[1].w};
        const float kz[8] = {raw.kz[0].x, raw.kz[0].y, raw.kz[0].z, raw.kz[0].w, raw.kz[1].x, raw.kz[1].y, raw.kz[1].z, raw.kz[1].w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const uint32_t x = (e < 2 ? raw.k.x : raw.k.y) >> (16 * (e & 1));
            o[e] = pack_f16_rne(fmaf((float)(x & 0xFFu), ks[2 * e], kz[2 * e]),
                                fmaf((float)((x >> 8) & 0xFFu), ks[2 * e + 1], kz[2 * e + 1]));
        }
        *reinterpret_cast<u32x4_t *>(frag_k(j)[k] + w * 1024 + 16 * lane) = o;
        const float4 *s = raw.s, *z = raw.z;
        const float vs[8] = {s[0].x, s[0].y, s[0].z, s[0].w, s[1].x, s[1].y, s[1].z, s[1].w};
        const float vz[8] = {z[0].x, z[0].y, z[0].z, z[0].w, z[1].x, z[1].y, z[1].z, z[1].w};
#pragma unroll
        for (int e = 0; e < 8; e += 2) {
            const uint32_t x = (uint32_t)raw.v[e >> 2] >> (8 * (e & 3));
            o[e / 2] = pack_f16_rne(fmaf((float)(x & 0xFFu), vs[e], vz[e]), fmaf((float)((x >> 8) & 0xFFu), vs[e + 1], vz[e + 1]));
        }
        *reinterpret_cast<u32x4_t *>(frag_v(j)[k] + w * 1024 + 16 * lane) = o;
    };

    wait_vmcnt<0>();
    __syncthreads();
    prepare(0);
    if (kSteps == 2) prepare(1);  // (step 2's, which iteration 0 converts)
    for (int j = 0; j < 3; ++j) prepare_v(j);
    __syncthreads();
    for (int j = 0; j < min(n_steps, 2); ++j)
        for (int k = 0; k < TS; ++k) convert(j, k, load_raw(j, k));
    // what is added to a score: kLift less the reference (FLT_MAX while no token has
    // been seen: a number, so that -inf and it are -inf)
    float lift[2] = {FLT_MAX, FLT_MAX};
    f32x4_t acc[2][8], l[2] = {};  // l: the sums of the weights, a ninth column of the values, all ones
    const u32x4_t ones = {0x3C003C00u, 0x3C003C00u, 0x3C003C00u, 0x3C003C00u};
#pragma unroll
    for (int rt = 0; rt < 2; ++rt)
#pragma unroll
        for (int c = 0; c < 8; ++c) acc[rt][c] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    // (a wavefront without rows computes its last one over: a branch around the
    // products cost the others more, 417 us against 361 where all have rows)
    const bool rows_live = row0 < a.rows_total;  // uniform in the wavefront
    __syncthreads();
    f32x4_t s[2][2];
    auto load_frags = [&](const uint8_t *frag, u32x4_t (&x)[8]) {
#pragma unroll
        for (int c = 0; c < 8; ++c) x[c] = *reinterpret_cast<const u32x4_t *>(frag + c * 1024 + 16 * lane);
    };
    auto scores = [&](const u32x4_t (&k)[8], f32x4_t (&x)[2][2]) {
#pragma unroll
        for (int r = 0; r < 2; ++r)
#pragma unroll
            for (int rt = 0; rt < 2; ++rt) x[rt][r] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int kk = 0; kk < 4; ++kk)
#pragma unroll
            for (int r = 0; r < 2; ++r)
#pragma unroll
                for (int rt = 0; rt < 2; ++rt) x[rt][r] = mfma_f16(k[4 * r + kk], qf[rt][kk], x[rt][r]);
    };
    u32x4_t kf[8], vf[8];
    load_frags(frag_k(0)[ts], kf);
    scores(kf, s);
    for (int j = 0; j < n_steps; ++j) {
        issue(j + kDepth, [&](int k) {
            return LAYOUT == 0 ? 0 : s_ids[LAYOUT == 0 ? 0 : w][(j + kDepth) % (2 * kDepth)][k][crow];
        });
        if ((j + 3) % kSteps == 0) prepare((j + 3) / kSteps);
        prepare_v(j + 3);
        if (j % kSteps == 0) {
            const int2 moved = *reinterpret_cast<const int2 *>(s_moved[(j / kSteps) & 1]);
            if (__builtin_amdgcn_readfirstlane(moved.x | moved.y)) load_off(j);
        }
        const int t0 = first + kTile * (TS * j + ts);
        if (t0 + kTile > end) {
#pragma unroll
            for (int r = 0; r < 2; ++r)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const bool in = t0 + 16 * r + 4 * kg + i < end;
#pragma unroll
                    for (int rt = 0; rt < 2; ++rt) s[rt][r][i] = in ? s[rt][r][i] : -INFINITY;
                }
        }
        float top[2];
#pragma unroll
        for (int rt = 0; rt < 2; ++rt) {
            const f32x4_t &x = s[rt][0], &y = s[rt][1];
            top[rt] = fmaf(fmax3(fmax3(x[0], x[1], x[2]), fmax3(x[3], y[0], y[1]), fmax2(y[2], y[3])), sc[rt], off[rt]);
        }
        if (__any(top[0] + lift[0] > kUpper || top[1] + lift[1] > kUpper)) {
#pragma unroll
            for (int rt = 0; rt < 2; ++rt) {
                const float next = fminf(kLift - max_kg(top[rt]), lift[rt]);
                const float alpha = __builtin_amdgcn_exp2f(next - lift[rt]);
                lift[rt] = next;
                float af[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) af[i] = __shfl(alpha, 4 * kg + i);
#pragma unroll
                for (int i = 0; i < 4; ++i) l[rt][i] *= af[i];
#pragma unroll
                for (int c = 0; c < 8; ++c)
#pragma unroll
                    for (int i = 0; i < 4; ++i) acc[rt][c][i] *= af[i];
            }
        }
        // Two stretches without branches, matrix and vector instructions in turns:
        // the scores of the next step with this one's weights ...
        load_frags(frag_k(j + 1)[ts], kf);
        __builtin_amdgcn_sched_barrier(0);
        load_frags(frag_v(j)[ts], vf);
        f32x4_t ahead[2][2];
        scores(kf, ahead);
        u32x4_t pa[2];
#pragma unroll
        for (int rt = 0; rt < 2; ++rt) {
            const f32x4_t &x = s[rt][0], &y = s[rt][1];
            const float c0 = off[rt] + lift[rt];
            float p[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) p[i] = __builtin_amdgcn_exp2f(fmaf(i < 4 ? x[i & 3] : y[i & 3], sc[rt], c0));
#pragma unroll
            for (int e = 0; e < 4; ++e) pa[rt][e] = pack_f16_rne(p[2 * e], p[2 * e + 1]);
        }
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x2, 3, 0);
            if (i >= 4 && i < 12) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
        }
        __builtin_amdgcn_sched_barrier(0);
        // ... the values, and the conversions: tile k with its share of the products
#pragma unroll
        for (int k = 0; k < TS; ++k) {
            const Raw raw = load_raw(j + 2, k);
#pragma unroll
            for (int c = 8 / TS * k; c < 8 / TS * (k + 1); ++c)
#pragma unroll
                for (int rt = 0; rt < 2; ++rt) acc[rt][c] = mfma_f16(pa[rt], vf[c], acc[rt][c]);
            if (k == TS - 1)
#pragma unroll
                for (int rt = 0; rt < 2; ++rt) l[rt] = mfma_f16(pa[rt], ones, l[rt]);
            convert(j + 2, k, raw);
            __builtin_amdgcn_sched_group_barrier(0x100, 10, 1);
            constexpr int kFirst = 4;  // products that run while the codes come in
            __builtin_amdgcn_sched_group_barrier(0x8, kFirst, 1);
#pragma unroll
            for (int i = 0; i < 16 / TS - kFirst; ++i) {
                __builtin_amdgcn_sched_group_barrier(0x2, 4 * TS, 1);
                __builtin_amdgcn_sched_group_barrier(0x8, 1, 1);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
#pragma unroll
        for (int rt = 0; rt < 2; ++rt)
#pragma unroll
            for (int r = 0; r < 2; ++r) s[rt][r] = ahead[rt][r];
        // step j + 3 is in once only the later ones' operations are in flight
        static_assert(kDepth == 4, "one step's may be");
        if (j + kDepth < n_steps)
            wait_vmcnt<kOps>();
        else
            wait_vmcnt<0>();
        __syncthreads();
    }

    // ---- the partials ----
    const bool any_bad = __syncthreads_or(bad);
    const float up = ldexpf(1.0f, Ev - kUpper - (int)kLift);
    // Of row tile rt, through LDS, so that rows are written whole: 8 rows of the
    // wavefront at a time.
    float *s_o = reinterpret_cast<float *>(&s_frag[0][0][0]) + (size_t)w * 8 * (kHeadDim + 4);
    static_assert(kWaves * 8 * (kHeadDim + 4) * 4 <= (2 + kFragsV) * kFragBytes, "the rows must fit in the operands' place");
    auto write_tile = [&](int rt, float lift_rt, f32x4_t l4, const f32x4_t (&o)[8]) {
        float sum = 0.0f;  // of row col: element col % 4 of the lanes of kg = col / 4
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float x = __shfl(l4[i], 16 * (col >> 2));
            sum = (col & 3) == i ? x : sum;
        }
        sum *= 1.0f / (1 << (int)kLift);
        if (any_bad) sum = NAN;
        const int r = row0 + 16 * rt + col;
        if (kg == 0 && r < a.rows_total) {
            const f32x2_t ml = {lift_rt == FLT_MAX ? -INFINITY : kLift - lift_rt, sum};
            __builtin_nontemporal_store(ml, reinterpret_cast<f32x2_t *>(a.ws_ml + partial_index(r)));
        }
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            // rows 4 kg + 2 half, + 1 of the tile
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int c = 0; c < 8; ++c) s_o[(2 * kg + i) * (kHeadDim + 4) + 16 * c + col] = o[c][2 * half + i] * up;
            __builtin_amdgcn_wave_barrier();
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int lr = 2 * k + (lane >> 5);  // row 4 (lr / 2) + 2 half + lr % 2 of the tile
                const int row = row0 + 16 * rt + 4 * (lr >> 1) + 2 * half + (lr & 1);
                f32x4_t x = *reinterpret_cast<const f32x4_t *>(s_o + lr * (kHeadDim + 4) + 4 * (lane & 31));
                if (any_bad) x = f32x4_t{NAN, NAN, NAN, NAN};
                if (row < a.rows_total)
                    __builtin_nontemporal_store(
                        x, reinterpret_cast<f32x4_t *>(a.ws_o + partial_index(row) * kHeadDim) + (lane & 31));
            }
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            __builtin_amdgcn_wave_barrier();
        }
    };
    if constexpr (TS == 1) {
        if (!rows_live) return;
        write_tile(0, lift[0], l[0], acc[0]);
        write_tile(1, lift[1], l[1], acc[1]);
    } else {
        // Two wavefronts have the same rows: each gives the other what it has of
        // one row tile (ts 0 of tile 1, ts 1 of tile 0) and writes the other tile.
        const bool one = ts != 0;
        f32x4_t *s_x = reinterpret_cast<f32x4_t *>(&s_frag[0][0][0]);  // [wavefront][9][lane]
        float *s_y = reinterpret_cast<float *>(&s_raw[0][0][0]);       // [wavefront][lane]
        static_assert(kWaves * 9 * 64 * 16 <= (2 + kFragsV) * TS * kFragBytes, "the exchange must fit");
#pragma unroll
        for (int c = 0; c < 8; ++c) s_x[(w * 9 + c) * 64 + lane] = one ? acc[0][c] : acc[1][c];
        s_x[(w * 9 + 8) * 64 + lane] = one ? l[0] : l[1];
        s_y[w * 64 + lane] = one ? lift[0] : lift[1];
        __syncthreads();
        const int other = w ^ (kWaves / TS);
        const float lift_other = s_y[other * 64 + lane];
        const float lift_own = one ? lift[1] : lift[0], lift_rt = fminf(lift_own, lift_other);
        const float f_own = __builtin_amdgcn_exp2f(lift_rt - lift_own), f = __builtin_amdgcn_exp2f(lift_rt - lift_other);
        float fo[4], ft[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            fo[i] = __shfl(f_own, 4 * kg + i);
            ft[i] = __shfl(f, 4 * kg + i);
        }
        f32x4_t o[9];
#pragma unroll
        for (int c = 0; c < 9; ++c) {
            const f32x4_t x = s_x[(other * 9 + c) * 64 + lane];
            const f32x4_t y = c == 8 ? (one ? l[1] : l[0]) : one ? acc[1][c & 7] : acc[0][c & 7];
#pragma unroll
            for (int i = 0; i < 4; ++i) o[c][i] = fmaf(x[i], ft[i], y[i] * fo[i]);
        }
        __syncthreads();  // the exchange is read
        if (rows_live) write_tile(ts, lift_rt, o[8], reinterpret_cast<const f32x4_t(&)[8]>(o));
    }
}

// As verify.hip's kernels: grid (worker, kv head x chunk) for the contiguous
// layout, the kv head fastest for paged ones.
template <int LAYOUT, int FIND, int TS>
__global__ __launch_bounds__(kThreads, 2) void verify_wide_kernel(VerifyArgs a) {
    const int worker = LAYOUT == 0 ? blockIdx.x : blockIdx.y;
    const int hc = LAYOUT == 0 ? blockIdx.y : blockIdx.x;
    const int h = hc % a.geo.Hkv, chunk = hc / a.geo.Hkv;
    Segment<kWorkUnit> seg;
    if (FIND == 0) {  // a unit per workgroup
        if (!seg.set_unit(a.seq_lens, a.max_seq_len, a.direct, blockIdx.z, worker)) return;
        wide_segment<LAYOUT, TS>(a, seg, h, chunk, threadIdx.x);
        return;
    }
    const WorkList<kWorkUnit, true> list(a.seq_lens, a.B, a.max_seq_len, a.workers);
    if (!seg.start(list, worker)) return;
    for (;;) {
        wide_segment<LAYOUT, TS>(a, seg, fresh_uniform(h), fresh_uniform(chunk), fresh_tid());
        if (!seg.next(list, worker)) return;
        __syncthreads();  // the segment's LDS is free again
    }
}

template <int TS>
void launch_steps(const VerifyArgs &a, dim3 grid, hipStream_t stream) {
    if (a.geo.max_blocks == 1 && a.direct)
        hipLaunchKernelGGL((verify_wide_kernel<0, 0, TS>), grid, dim3(kThreads), 0, stream, a);
    else if (a.geo.max_blocks == 1)
        hipLaunchKernelGGL((verify_wide_kernel<0, 1, TS>), grid, dim3(kThreads), 0, stream, a);
    else if (a.direct)
        hipLaunchKernelGGL((verify_wide_kernel<1, 0, TS>), grid, dim3(kThreads), 0, stream, a);
    else
        hipLaunchKernelGGL((verify_wide_kernel<1, 1, TS>), grid, dim3(kThreads), 0, stream, a);
}

}  // namespace

hipError_t launch_verify_wide(const VerifyArgs &a, int rows, hipStream_t stream) {
    if (a.rows_total < 1 || a.workers < 1 || a.workers > 65535) return hipErrorInvalidValue;
    const unsigned hc = (unsigned)(a.geo.Hkv * ((a.rows_total + rows - 1) / rows));
    const unsigned n = a.direct ? a.direct : a.workers, nz = a.direct ? a.B : 1;
    const dim3 grid = a.geo.max_blocks == 1 ? dim3(n, hc, nz) : dim3(hc, n, nz);
    if (rows == kWideRows)
        launch_steps<1>(a, grid, stream);
    else
        launch_steps<2>(a, grid, stream);
    return hipGetLastError();
}

}  // namespace lynx
