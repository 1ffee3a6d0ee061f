// Verification over the merged cache for many query rows a kv head (gfx950 MFMA,
// fp16 operands): the context part of a wide token tree.
//
// What it computes is verify.hip's: the partial (max, sum, output) of every row
// over a segment of the context.  There a wavefront folds the K scales into its
// own rows' queries, group by group, and unpacks K and V for itself, which costs
// as many vector instructions per (row, token) as the softmax does.  With 200 rows
// and more the keys are the smaller side: here the workgroup's 8 wavefronts share
// the tokens and split the rows, 32 each, so that a tile's K and V are
// reconstructed once for 256 rows, as fp16 in the matrix cores' operand order in
// LDS, and the queries are converted once.
//
// Operands:
//  * K' = (zero + code scale) 2^-e_d, e_d the exponent of the largest |K| of
//    channel d in the segment (from the metadata), so |K'| <= 1; the query is
//    q_d 2^(e_d - E), E the exponent of the row's largest product: exact in fp16
//    (BF16 has 8 significant bits) down to 2^-17 of the largest.  K' is computed in
//    fp16 as (code - 128) scale' + centre', scale', centre' = zero' + 128 scale' and
//    the result each rounded to 11 bits: off by at most 2^-12 (|K' - centre'| +
//    |centre'| + |K'|), where the BF16 key was off by 2^-9 |K'| to begin with.  128
//    such errors are independent: a score moves by some 2e-4 of the root mean
//    square of its terms times sqrt(128).
//  * V' = (zero + code scale) 2^-Ev, Ev over the segment, rounded to 11 bits, as
//    are the weights p <= 2^8 against a reference that follows the row's maximum
//    once it is 2^8 behind; l is summed in fp32.
//
// A tile of 32 tokens costs a wavefront 32 MFMAs for its 32 rows.  Iteration j:
// copies of tile j + kDepth into LDS (asynchronous), the scores of tile j + 1, the
// weights of tile j and their products with the values, the conversion of tile
// j + 2, in one stretch without branches, so that matrix and vector instructions
// take turns; one barrier.  2 x 64K tokens, 8 kv heads, 512 rows: 361 us with the
// merge (verify.hip's kernel 560), 32% of the matrix cores' cycles and 45% of the
// vector ones'; the rest are waits for LDS, whose reads (16 KB per wavefront and
// tile) come in bursts behind the barrier.  Four wavefronts of 32 rows twice on a
// CU took 470 us, four of 64 rows 627 (accumulators move through the other half
// of the register file), two orders of the stretches for the two wavefronts of a
// SIMD 444.
#include "f16_ops.h"
#include "lane_ops.h"
#include "lynx_internal.h"
#include "work_list.h"

#include <float.h>
#include <math.h>

namespace lynx {
namespace {

typedef _Float16 h2 __attribute__((ext_vector_type(2)));

constexpr int kWaves = 8;
constexpr int kThreads = 64 * kWaves;
constexpr int kRows = kWideRows;
static_assert(kRows == 32 * kWaves, "two row tiles per wavefront");
constexpr int kTile = 32;  // tokens
constexpr float kLog2e = 1.4426950408889634f;
constexpr int kRawPlane = kTile * kCodeRow;         // 4 KB of codes
constexpr int kRawMeta = 2 * kRawPlane;             // V scale[32] | V zero[32]
constexpr int kRawBytes = kRawMeta + 2 * kTile * 4;
constexpr int kFragBytes = 8 * 1024;                // a tile's 8 fragments of K, or of V
constexpr int kFragsV = 3;                          // V's buffers; K's are two
constexpr int kDepth = 4;                           // tiles whose copies are in flight or not converted yet
constexpr float kSlack = 8.0f;                      // log2 units that the reference may lag behind

template <int LAYOUT>
__device__ __forceinline__ void wide_segment(const VerifyArgs &a, const Segment<kWorkUnit> &seg, int h, int chunk,
                                             const int tid) {
    const int Hkv = a.geo.Hkv;
    const int lane = tid & 63, w = tid >> 6, col = lane & 15, kg = lane >> 4;
    const int b = seg.b, T = seg.T, g0 = seg.g0;
    const int row0 = chunk * kRows + 32 * w;  // of the wavefront
    auto partial_index = [&](int r) { return ((size_t)h * a.rows_total + r) * a.n_seg + seg.number; };
    if (seg.n_groups == 0) {  // an empty sequence: (max, sum) = (-inf, 0)
        for (int r = chunk * kRows + tid; r < min(a.rows_total, (chunk + 1) * kRows); r += kThreads)
            a.ws_ml[partial_index(r)] = make_float2(-INFINITY, 0.0f);
        return;
    }
    const int first = g0 * kKGroup, end = min(T, first + seg.n_groups * kKGroup);
    const int n_tiles = (end - first + kTile - 1) / kTile;

    __shared__ __attribute__((aligned(16))) uint8_t s_raw[kDepth][kRawBytes];
    __shared__ __attribute__((aligned(16))) uint8_t s_frag[2 + kFragsV][kFragBytes];
    __shared__ __attribute__((aligned(16))) float s_km[2][2 * kHeadDim];  // K scale | zero of a group, two groups
    __shared__ int32_t s_ids[LAYOUT == 0 ? 1 : kWaves][2 * kDepth][8];  // blocks of a tile's rows
    __shared__ int s_e[kHeadDim];                                       // channel exponents
    __shared__ float s_vmax[kWaves];
    float(*s_max)[kHeadDim] = reinterpret_cast<float(*)[kHeadDim]>(&s_frag[0][0]);  // (before there are fragments)
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
    auto token_of = [&](int j, int k) { return min(first + kTile * j + 8 * (k & 3) + crow, T - 1); };
    auto block_at = [&](int j) { return LAYOUT == 0 ? bt_row : bt_row + block_of(token_of(j, w)); };
    // Every wavefront issues as many operations per tile, so that it can wait for
    // the older ones: a copy of rows, one of metadata (K's with a group's
    // first tile, by wavefront 1; else V's, which may be written more than once),
    // and the block numbers of a later tile.
    // Wavefront w copies rows 8 (w % 4) .. + 7 of K (w < 4) or V.
    constexpr int kOps = LAYOUT == 0 ? 2 : 3;
    auto copy_ids = [&](int j) {
        if (LAYOUT != 0 && lane < 8) {
            const int t = min(first + kTile * j + 8 * (w & 3) + lane, T - 1);
            lds_copy4(bt_row + block_of(t), lds_addr(&s_ids[LAYOUT == 0 ? 0 : w][j % (2 * kDepth)][0]));
        }
    };
    auto issue = [&](int j, int id) {
        if (j >= n_tiles) return;
        const uint32_t slot = lds_addr(s_raw[j % kDepth]);
        const int t = token_of(j, w);
        if (id < 0 || id >= a.geo.num_blocks) {
            bad = true;
            id = 0;
        }
        const size_t row = ((size_t)id * Hkv + h) * a.geo.bt + (size_t)(LAYOUT == 0 ? t : t - block_of(t) * a.geo.bt);
        const int q = (lane & 7) ^ crow ^ (w < 4 ? 0 : ((w & 3) >> 1) << 2);
        lds_copy16((w < 4 ? a.k_codes : a.v_codes) + row * kCodeRow + 16 * q, slot + 1024u * w);
        if (w == 1 && (j & 3) == 0) {
            lds_copy16((lane < 32 ? a.meta.k_scale : a.meta.k_zero) + kmeta + (size_t)(g0 + (j >> 2)) * kHeadDim + 4 * (lane & 31),
                       lds_addr(s_km[(j >> 2) & 1]));
        } else {
            const int tt = min(first + kTile * j + (lane & 31), T - 1);
            lds_copy4((lane < 32 ? a.meta.v_scale : a.meta.v_zero) + vmeta + tt, slot + kRawMeta);
        }
        copy_ids(j + kDepth);
    };

    // ---- the exponents of the segment's channels and of its values ----
    {
        int ids[kDepth];
#pragma unroll
        for (int j = 0; j < kDepth; ++j) ids[j] = *block_at(min(j, n_tiles - 1));
#pragma unroll
        for (int j = 0; j < kDepth; ++j) issue(j, ids[j]);
    }
    {
        float4 m = make_float4(0.f, 0.f, 0.f, 0.f);
        const int d4 = tid & 31, gg = tid >> 5;  // 4 channels; groups gg, gg + 2 kWaves, ...
        for (int g = gg; g < seg.n_groups; g += kThreads / 32) {
            const float4 s = reinterpret_cast<const float4 *>(a.meta.k_scale + kmeta + (size_t)(g0 + g) * kHeadDim)[d4];
            const float4 z = reinterpret_cast<const float4 *>(a.meta.k_zero + kmeta + (size_t)(g0 + g) * kHeadDim)[d4];
            m.x = fmax3_abs(m.x, z.x, fmaf(255.0f, s.x, z.x));
            m.y = fmax3_abs(m.y, z.y, fmaf(255.0f, s.y, z.y));
            m.z = fmax3_abs(m.z, z.z, fmaf(255.0f, s.z, z.z));
            m.w = fmax3_abs(m.w, z.w, fmaf(255.0f, s.w, z.w));
        }
        reinterpret_cast<float4 *>(s_max[gg])[d4] = m;
        float v = 0.0f;
        for (int t = first + tid; t < end; t += kThreads) {
            const float s = a.meta.v_scale[vmeta + t], z = a.meta.v_zero[vmeta + t];
            v = fmax3_abs(v, z, fmaf(255.0f, s, z));
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
        Ev = min(max(Ev, -126), 126);  // 2^Ev and 2^-Ev are normal numbers
    }
    __syncthreads();

    // ---- the wavefront's queries: row col of each row tile, dims 8 kg + 32 kk ----
    u32x4_t qf[2][4];
    float sc[2];
#pragma unroll
    for (int rt = 0; rt < 2; ++rt) {
        const int r = min(row0 + 16 * rt + col, a.rows_total - 1);
        const uint16_t *q = a.q + (((size_t)b * a.nq + r / a.G) * a.Hq + (size_t)h * a.G + r % a.G) * kHeadDim + 8 * kg;
        float y[4][8];
#pragma unroll
        for (int kk = 0; kk < 4; ++kk) {
            const uint4 u = *reinterpret_cast<const uint4 *>(q + 32 * kk);
            const uint32_t x[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                y[kk][2 * e] = bf16_lo(x[e]);
                y[kk][2 * e + 1] = bf16_hi(x[e]);
            }
        }
        // the exponent of the row's largest product with a key, in two steps: the
        // products themselves may leave the range of fp32
        int E = -20000;
#pragma unroll
        for (int kk = 0; kk < 4; ++kk)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                int x = 0;
                frexpf(y[kk][e], &x);
                if (y[kk][e] != 0.0f) E = max(E, x + s_e[32 * kk + 8 * kg + e]);
            }
        E = max(E, __shfl_xor(E, 16));
        E = max(E, __shfl_xor(E, 32));
#pragma unroll
        for (int kk = 0; kk < 4; ++kk)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int d = 32 * kk + 8 * kg + 2 * e;
                qf[rt][kk][e] = pack_f16_rne(ldexpf(y[kk][2 * e], s_e[d] - E), ldexpf(y[kk][2 * e + 1], s_e[d + 1] - E));
            }
        // positive and finite: times the -inf of a token past the context it must
        // not be a NaN
        sc[rt] = __builtin_amdgcn_fmed3f(ldexpf(kLog2e * rsqrtf((float)kHeadDim), E), FLT_MIN, FLT_MAX);
    }

    // ---- conversion of a tile into operand order ----
    // K: fragment 4 r + kk: lane (token 16 r + col, dims 32 kk + 8 kg .. + 7); V:
    // fragment c: lane (dim 16 c + col, tokens 16 (e / 4) + 4 kg + e % 4).  Wavefront
    // w makes fragment w of each.
    const int kk_own = w & 3;
    h2 ks[4], kz[4];
    auto load_group = [&](int j) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int d = 32 * kk_own + 8 * kg + e;
            const float sc = ldexpf(s_km[(j >> 2) & 1][d], -s_e[d]);
            ks[e / 2][e % 2] = (_Float16)sc;
            kz[e / 2][e % 2] = (_Float16)fmaf(128.0f, sc, ldexpf(s_km[(j >> 2) & 1][kHeadDim + d], -s_e[d]));
        }
    };
    const float down = ldexpf(1.0f, -Ev);
    auto convert = [&](int j) {  // (of a tile past the last: what its slot holds, to where nothing reads)
        const uint8_t *raw = s_raw[j % kDepth];
        {
            const int t = 16 * (w >> 2) + col, q = 2 * kk_own + (kg >> 1);
            const uint2 c = *reinterpret_cast<const uint2 *>(raw + t * kCodeRow + ((q ^ (t & 7)) * 16) + 8 * (kg & 1));
            u32x4_t o;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                // a byte under 0x64 is 1024 + code
                const uint32_t code = __builtin_amdgcn_perm(0x64646464u, e < 2 ? c.x : c.y, e & 1 ? 0x04030402u : 0x04010400u);
                const h2 x = __builtin_bit_cast(h2, code) - (h2){(_Float16)1152.0f, (_Float16)1152.0f};
                o[e] = __builtin_bit_cast(uint32_t, __builtin_elementwise_fma(x, ks[e], kz[e]));
            }
            *reinterpret_cast<u32x4_t *>(frag_k(j) + w * 1024 + 16 * lane) = o;
        }
        const float *vm = reinterpret_cast<const float *>(raw + kRawMeta) + 4 * kg;
        const float4 s0 = *reinterpret_cast<const float4 *>(vm), s1 = *reinterpret_cast<const float4 *>(vm + 16);
        const float4 z0 = *reinterpret_cast<const float4 *>(vm + kTile), z1 = *reinterpret_cast<const float4 *>(vm + kTile + 16);
        const float vs[8] = {s0.x, s0.y, s0.z, s0.w, s1.x, s1.y, s1.z, s1.w};
        const float vz[8] = {z0.x, z0.y, z0.z, z0.w, z1.x, z1.y, z1.z, z1.w};
        const int tr = 16 * ((col >> 1) >> 2) + 4 * kg + ((col >> 1) & 3);
        {
            const intx2_t v = __builtin_amdgcn_ds_read_tr8_b64_v2i32(
                (__attribute__((address_space(3))) intx2_t *)(raw + kRawPlane + v_slot(tr, w) + 8 * (col & 1)));
            u32x4_t o;
#pragma unroll
            for (int e = 0; e < 8; e += 2) {
                const uint32_t x = (uint32_t)v[e >> 2] >> (8 * (e & 3));
                o[e / 2] = pack_f16_rne(down * fmaf((float)(x & 0xFFu), vs[e], vz[e]),
                                        down * fmaf((float)((x >> 8) & 0xFFu), vs[e + 1], vz[e + 1]));
            }
            *reinterpret_cast<u32x4_t *>(frag_v(j) + w * 1024 + 16 * lane) = o;
        }
    };

    wait_vmcnt<0>();
    __syncthreads();
    load_group(0);
    convert(0);
    if (n_tiles > 1) convert(1);
    float m_run[2] = {-INFINITY, -INFINITY}, l[2] = {0.0f, 0.0f};
    f32x4_t acc[2][8];
#pragma unroll
    for (int rt = 0; rt < 2; ++rt)
#pragma unroll
        for (int c = 0; c < 8; ++c) acc[rt][c] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    // (a wavefront without rows computes its last one over: a branch around the
    // products costs the others more, 417 us against 361 where all have rows)
    const bool rows_live = row0 < a.rows_total;  // uniform in the wavefront
    const int id0 = LAYOUT == 0 ? bt_row[0] : 0;
    asm volatile("" ::"s"(id0));  // in before the copies go on
    __syncthreads();
    f32x4_t s[2][2];
    auto scores = [&](int j, f32x4_t (&x)[2][2]) {
        const uint8_t *frag = frag_k(j) + 16 * lane;
#pragma unroll
        for (int r = 0; r < 2; ++r) {
#pragma unroll
            for (int rt = 0; rt < 2; ++rt) x[rt][r] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int kk = 0; kk < 4; ++kk) {
                const u32x4_t k = *reinterpret_cast<const u32x4_t *>(frag + (4 * r + kk) * 1024);
#pragma unroll
                for (int rt = 0; rt < 2; ++rt) x[rt][r] = mfma_f16(k, qf[rt][kk], x[rt][r]);
            }
        }
    };
    scores(0, s);
    for (int j = 0; j < n_tiles; ++j) {
        issue(j + kDepth, LAYOUT == 0 ? id0 : s_ids[LAYOUT == 0 ? 0 : w][(j + kDepth) % (2 * kDepth)][crow]);
        if (((j + 2) & 3) == 0) load_group(j + 2);
        const int t0 = first + kTile * j;
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
            top[rt] = fmax3(fmax3(x[0], x[1], x[2]), fmax3(x[3], y[0], y[1]), fmax2(y[2], y[3])) * sc[rt];
        }
        if (__any(top[0] > m_run[0] + kSlack || top[1] > m_run[1] + kSlack)) {
#pragma unroll
            for (int rt = 0; rt < 2; ++rt) {
                const float m = fmaxf(max_kg(top[rt]), m_run[rt]);
                const float alpha = m_run[rt] == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(m_run[rt] - m);
                m_run[rt] = m;
                l[rt] *= alpha;
                float af[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) af[i] = __shfl(alpha, 4 * kg + i);
#pragma unroll
                for (int c = 0; c < 8; ++c)
#pragma unroll
                    for (int i = 0; i < 4; ++i) acc[rt][c][i] *= af[i];
            }
        }
        // one stretch without branches from here
        f32x4_t ahead[2][2];
        scores(j + 1, ahead);
        u32x4_t pa[2];
#pragma unroll
        for (int rt = 0; rt < 2; ++rt) {
            const f32x4_t &x = s[rt][0], &y = s[rt][1];
            const float ref = m_run[rt] == -INFINITY ? 0.0f : -m_run[rt];
            float p[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                p[i] = __builtin_amdgcn_exp2f(fmaf(i < 4 ? x[i & 3] : y[i & 3], sc[rt], ref));
                l[rt] += p[i];
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) pa[rt][e] = pack_f16_rne(p[2 * e], p[2 * e + 1]);
        }
        const uint8_t *frag = frag_v(j) + 16 * lane;
#pragma unroll
        for (int c = 0; c < 8; ++c) {
            const u32x4_t v = *reinterpret_cast<const u32x4_t *>(frag + c * 1024);
#pragma unroll
            for (int rt = 0; rt < 2; ++rt) acc[rt][c] = mfma_f16(pa[rt], v, acc[rt][c]);
        }
        convert(j + 2);
#pragma unroll
        for (int rt = 0; rt < 2; ++rt)
#pragma unroll
            for (int r = 0; r < 2; ++r) s[rt][r] = ahead[rt][r];
        // tile j + 3 is in once only the later ones' operations are in flight
        static_assert(kDepth == 4, "one tile's may be");
        if (j + kDepth < n_tiles)
            wait_vmcnt<kOps>();
        else
            wait_vmcnt<0>();
        __syncthreads();
    }

    // ---- the partials: through LDS, so that rows are written whole ----
    const bool any_bad = __syncthreads_or(bad);
    if (!rows_live) return;
    float *s_o = reinterpret_cast<float *>(&s_frag[0][0]) + (size_t)w * 8 * (kHeadDim + 4);  // 8 rows of the wavefront
    static_assert(kWaves * 8 * (kHeadDim + 4) * 4 <= (2 + kFragsV) * kFragBytes, "the rows must fit in the operands' place");
    const float up = ldexpf(1.0f, Ev);
#pragma unroll
    for (int rt = 0; rt < 2; ++rt) {
        const float sum = any_bad ? NAN : sum_kg(l[rt]);
        const int r = row0 + 16 * rt + col;
        if (kg == 0 && r < a.rows_total) {
            const f32x2_t ml = {m_run[rt], sum};
            __builtin_nontemporal_store(ml, reinterpret_cast<f32x2_t *>(a.ws_ml + partial_index(r)));
        }
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            // rows 4 kg + 2 half, + 1 of the tile: 8 rows at a time
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int c = 0; c < 8; ++c) s_o[(2 * kg + i) * (kHeadDim + 4) + 16 * c + col] = acc[rt][c][2 * half + i] * up;
            __builtin_amdgcn_wave_barrier();
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int lr = 2 * k + (lane >> 5);  // row 4 (lr / 2) + 2 half + lr % 2 of the tile
                const int row = row0 + 16 * rt + 4 * (lr >> 1) + 2 * half + (lr & 1);
                f32x4_t o = *reinterpret_cast<const f32x4_t *>(s_o + lr * (kHeadDim + 4) + 4 * (lane & 31));
                if (any_bad) o = f32x4_t{NAN, NAN, NAN, NAN};
                if (row < a.rows_total)
                    __builtin_nontemporal_store(
                        o, reinterpret_cast<f32x4_t *>(a.ws_o + partial_index(row) * kHeadDim) + (lane & 31));
            }
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            __builtin_amdgcn_wave_barrier();
        }
    }
}

// As verify.hip's kernels: grid (worker, kv head x chunk) for the contiguous
// layout, the kv head fastest for paged ones.
template <int LAYOUT, int FIND>
__global__ __launch_bounds__(kThreads, 2) void verify_wide_kernel(VerifyArgs a) {
    const int worker = LAYOUT == 0 ? blockIdx.x : blockIdx.y;
    const int hc = LAYOUT == 0 ? blockIdx.y : blockIdx.x;
    const int h = hc % a.geo.Hkv, chunk = hc / a.geo.Hkv;
    Segment<kWorkUnit> seg;
    if (FIND == 0) {  // a unit per workgroup
        if (!seg.set_unit(a.seq_lens, a.max_seq_len, a.direct, blockIdx.z, worker)) return;
        wide_segment<LAYOUT>(a, seg, h, chunk, threadIdx.x);
        return;
    }
    const WorkList<kWorkUnit, true> list(a.seq_lens, a.B, a.max_seq_len, a.workers);
    if (!seg.start(list, worker)) return;
    for (;;) {
        wide_segment<LAYOUT>(a, seg, fresh_uniform(h), fresh_uniform(chunk), fresh_tid());
        if (!seg.next(list, worker)) return;
        __syncthreads();  // the segment's LDS is free again
    }
}

template <int LAYOUT>
void launch_find(const VerifyArgs &a, dim3 grid, hipStream_t stream) {
    if (a.direct)
        hipLaunchKernelGGL((verify_wide_kernel<LAYOUT, 0>), grid, dim3(kThreads), 0, stream, a);
    else
        hipLaunchKernelGGL((verify_wide_kernel<LAYOUT, 1>), grid, dim3(kThreads), 0, stream, a);
}

}  // namespace

hipError_t launch_verify_wide(const VerifyArgs &a, hipStream_t stream) {
    if (a.rows_total < 1 || a.workers < 1 || a.workers > 65535) return hipErrorInvalidValue;
    const unsigned hc = (unsigned)(a.geo.Hkv * ((a.rows_total + kWideRows - 1) / kWideRows));
    const unsigned n = a.direct ? a.direct : a.workers, nz = a.direct ? a.B : 1;
    const dim3 grid = a.geo.max_blocks == 1 ? dim3(n, hc, nz) : dim3(hc, n, nz);
    if (a.geo.max_blocks == 1)
        launch_find<0>(a, grid, stream);
    else
        launch_find<1>(a, grid, stream);
    return hipGetLastError();
}

}  // namespace lynx
