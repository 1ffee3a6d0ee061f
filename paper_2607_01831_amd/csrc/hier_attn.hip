// Attention over the hierarchical codec's cache on matrix cores (gfx950 MFMA).
//
// What it computes (attention of Sec. 2 over the cache of Alg. 1): for every
// query row, O = softmax(q K^T / sqrt(128)) V over the context's tokens, with
// K and V reconstructed from the 4-bit planes (anchors, or the single 4-bit
// code) or from the merged 8-bit codes as
//   x = ((+-level(code) sigma) + mu) gscale + gmin
// per channel: sigma and mu of the chunk of 32 tokens, gscale and gmin of the
// page of 256.  The BF16 tokens behind the context are the combine kernel's
// (attention.hip).
//
// The operands.  x = level b + m with b = sigma gscale, m = mu gscale + gmin: one
// affine map per channel and chunk.  The levels are a table: 256 entries by plane
// byte, for a byte of two nibbles the pair of levels as two fp16, for a byte of
// one code its level.  A byte is looked up in LDS, mapped by one packed fp16
// multiply-add, and is a matrix operand as it stands.  Both products run as
// v_mfma_f32_16x16x32_f16, the contraction of the second one chunk long.
//
// Rounding.  A level, b, m and x are rounded to fp16 (11 significant bits, 2^-11 of
// themselves at most), so x is off by at most 2^-11 (2 |level b| + |m| + |x|), an
// eighth of what so many roundings to BF16 would be; a softmax weight is rounded
// likewise (2^-11 of itself, 2^-32 of the row's largest).  Queries are BF16 and
// exact.  Scores, softmax statistics and outputs are fp32.  Powers of two keep the
// operands in fp16's range whatever the cache's: K and V are scaled by an exponent
// each that brings the largest |b| + |m| so far below 2^14, so values 2^-28 of the
// largest lose bits; a query row by its largest element.
#include "f16_ops.h"
#include "hier_levels.h"
#include "lane_ops.h"
#include "lynx_internal.h"
#include "split_merge.h"
#include "work_list.h"

#include <float.h>
#include <math.h>

namespace lynx {

namespace {

constexpr int kThreads = 256;
constexpr int kWaves = 4;
constexpr int kChunk = 32;   // tokens of a codec chunk, and of a wavefront's step
constexpr int kPage = 256;   // tokens of a codec page
constexpr float kLog2e = 1.4426950408889634f;
// The largest |b| + |m| of the scaled K and V, and the largest |q|: products up to
// 2^24, sums in fp32.
constexpr int kKvTop = 14, kQTop = 10;
// A softmax weight is exp2(score - reference + kPTop); the reference moves when a
// score passes it by kSlack, so weights stay below 2^(kPTop + kSlack) < 65504.
constexpr int kPTop = 7, kSlack = 8;

// LDS: the table, 64 copies of 256 entries (entry e of lane l at 256 e + 4 l, so a
// lookup's address is the plane byte over the lane's byte, one v_perm, and every
// lane reads a bank of its own), then a page of 16 KB: while the wavefronts attend,
// 1 KB each for a chunk's b and m; at the end what they join.  80 KB, two
// workgroups per CU.
constexpr int kTable = 256 * 256;
constexpr int kShare = 16384;

__device__ __forceinline__ uint32_t pk_fma(uint32_t a, uint32_t b, uint32_t c) {
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_fma(__builtin_bit_cast(f16x2_t, a),
                                                                  __builtin_bit_cast(f16x2_t, b),
                                                                  __builtin_bit_cast(f16x2_t, c)));
}
__device__ __forceinline__ uint32_t low16s(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x05040100u); }
__device__ __forceinline__ uint32_t high16s(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x07060302u); }
// Largest of a non-negative value over the wavefront, uniform; a NaN may be lost.
__device__ __forceinline__ float wave_max(float v) { return row_max<64>(v); }
// The exponent e with x < 2^e (x >= 0), kept where 2^(kKvTop - e) is a normal float.
constexpr int kLeast = -112;
__device__ __forceinline__ int exponent_of(float x) { return max((int)(__float_as_uint(x) >> 23) - 126, kLeast); }

// One segment of a worker's share, kv head h, rows r0 .. r0 + 16 MT - 1.
// Wavefront w owns the 128-token groups w, w + 4, ... of the segment and attends
// their chunks with an online softmax of its own: no barrier in the loop.
//
// Layouts of a wavefront's step (col = lane % 16, g = lane / 16): the scores are
// computed as K Q^T, lane (col, g) holding query row col against tokens 4 g + i and
// 16 + 4 g + i (i < 4).  That is the first operand of the second product as it
// stands, where slot e of group g is then token 4 g + e or 16 + 4 g + e - 4; the
// lane's eight V rows are those tokens', of which it takes dims 8 col .. + 7, one a
// tile of 16 columns, so an output lane holds dims 8 col .. + 7 of rows 4 g + i.
//
// LAYOUT 0: one block per sequence; 1: block_tokens a multiple of 16; 2: any other.
template <int MT, int FULL, int LAYOUT>
__device__ __forceinline__ void attend_segment(const HierArgs &a, const Segment<kWorkUnit> &seg, int h, int chunk_rows,
                                               const int tid, uint8_t *lds) {
    static_assert(kWorkUnit == kWaves, "a group per wavefront and unit");
    constexpr int kRow = FULL ? kCodeRow : kNibbleRow;
    constexpr int kKW = FULL ? 8 : 4;  // words of a lane's K row quarter
    constexpr int kVW = FULL ? 2 : 1;  // words of a lane's 8 dims of a V row
    const int Hkv = a.geo.Hkv;
    const int lane = tid & 63, w = tid >> 6, col = lane & 15, g = lane >> 4;
    const int b = seg.b, T = seg.T, live = seg.live;
    const int r0 = chunk_rows * 16 * MT;
    const int rows = min(16 * MT, a.rows_total - r0);
    const size_t prow0 = (size_t)h * a.rows_total + r0;
    auto query_row = [&](int r) {  // row r of the workgroup
        const int gr = r0 + r;
        return ((size_t)b * a.nq + gr / a.G) * a.Hq + (size_t)h * a.G + gr % a.G;
    };
    if (seg.n_groups == 0) {
        // an empty sequence: zeros, lse -inf; or, for the combine kernel, (-inf, 0)
        if (a.fused) {
            for (int i = tid; i < rows * (kHeadDim / 4); i += kThreads)
                *reinterpret_cast<uint2 *>(a.out + query_row(i / (kHeadDim / 4)) * kHeadDim + 4 * (i % (kHeadDim / 4))) =
                    make_uint2(0u, 0u);
            if (a.lse && tid < rows) a.lse[query_row(tid)] = -INFINITY;
        } else if (tid < rows) {
            a.ws_ml[(prow0 + tid) * a.n_seg + seg.number] = make_float2(-INFINITY, 0.0f);
        }
        return;
    }
    uint8_t *share = lds + kTable;
    uint8_t *stage = share + w * 1024;  // K: b, m, V: b, m of a chunk, [128] fp16 each

    // ---- where a token's rows are ----
    bool bad = false;
    const int32_t *bt_row = a.block_table + (size_t)b * a.geo.max_blocks;
    auto block_row0 = [&](int t, int blk) -> size_t {  // the row of token t in its block blk
        if (blk < 0 || blk >= a.geo.num_blocks) {
            bad = true;
            blk = 0;
        }
        const int bi = LAYOUT == 0 ? 0 : a.bt_shift >= 0 ? (t >> a.bt_shift) : t / a.geo.bt;
        return ((size_t)blk * Hkv + h) * a.geo.bt + (size_t)(t - bi * a.geo.bt);
    };
    auto block_of = [&](int t) {
        return bt_row[LAYOUT == 0 ? 0 : a.bt_shift >= 0 ? (t >> a.bt_shift) : t / a.geo.bt];
    };

    // ---- the wavefront's chunks ----
    const int my_groups = seg.n_groups > w ? (seg.n_groups - w + kWaves - 1) / kWaves : 0;
    auto chunk_t0 = [&](int j) { return (seg.g0 + w + kWaves * (j >> 2)) * kKGroup + kChunk * (j & 3); };
    // the last group of the sequence may hold fewer than four
    int n_mine = 4 * my_groups;
    while (n_mine > 0 && chunk_t0(n_mine - 1) >= T) --n_mine;

    // ---- loads of a chunk ----
    struct Raw {
        uint32_t k[2][kKW];  // token 16 a + col, bytes kRow / 4 * g ..
        uint32_t v[8][kVW];  // token slot e, dims 8 col .. + 7
        float2 ks, km, kgs, kgm, vs, vm, vgs, vgm;  // channels 2 lane, 2 lane + 1
    };
    const size_t cmeta = ((size_t)b * Hkv + h) * a.geo.n_chunks * kHeadDim + 2 * lane;
    const size_t pmeta = ((size_t)b * Hkv + h) * a.geo.n_pages * kHeadDim + 2 * lane;
    auto load_k = [&](Raw &r, int i, const uint8_t *p) {
#pragma unroll
        for (int q = 0; q < kKW / 4; ++q) {
            const uint4 u = reinterpret_cast<const uint4 *>(p)[q];
            r.k[i][4 * q] = u.x; r.k[i][4 * q + 1] = u.y; r.k[i][4 * q + 2] = u.z; r.k[i][4 * q + 3] = u.w;
        }
    };
    auto load_v = [&](Raw &r, int e, const uint8_t *p) {
        if (FULL) {
            const uint2 u = *reinterpret_cast<const uint2 *>(p);
            r.v[e][0] = u.x;
            r.v[e][kVW - 1] = u.y;
        } else {
            r.v[e][0] = *reinterpret_cast<const uint32_t *>(p);
        }
    };
    auto load_chunk = [&](Raw &r, int j) {
        const int t0 = __builtin_amdgcn_readfirstlane(chunk_t0(j));
        {
            const size_t c = cmeta + (size_t)(t0 / kChunk) * kHeadDim, p = pmeta + (size_t)(t0 / kPage) * kHeadDim;
            r.ks = *reinterpret_cast<const float2 *>(a.meta.k_sigma + c);
            r.km = *reinterpret_cast<const float2 *>(a.meta.k_mu + c);
            r.vs = *reinterpret_cast<const float2 *>(a.meta.v_sigma + c);
            r.vm = *reinterpret_cast<const float2 *>(a.meta.v_mu + c);
            r.kgs = *reinterpret_cast<const float2 *>(a.meta.k_gscale + p);
            r.kgm = *reinterpret_cast<const float2 *>(a.meta.k_gmin + p);
            r.vgs = *reinterpret_cast<const float2 *>(a.meta.v_gscale + p);
            r.vgm = *reinterpret_cast<const float2 *>(a.meta.v_gmin + p);
        }
        if (LAYOUT != 2 && t0 + kChunk <= T) {
            // two 16-token runs, each inside one block
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int t = t0 + 16 * i;
                const size_t row = block_row0(t, __builtin_amdgcn_readfirstlane(block_of(t))) * kRow;
                load_k(r, i, a.k_plane + row + (col * kRow + g * (kRow / 4)));
#pragma unroll
                for (int e = 0; e < 4; ++e) load_v(r, 4 * i + e, a.v_plane + row + ((4 * g + e) * kRow + col * (kRow / 16)));
            }
        } else {
            // a lookup per token, in lanes 0 .. 31; tokens past the context
            // repeat the last one
            const int t = min(t0 + (lane & 31), T - 1);
            const size_t row = block_row0(t, block_of(t));
            auto row_of = [&](int from) -> size_t {
                return (size_t)(uint32_t)__shfl((int)(uint32_t)row, from) | (size_t)(uint32_t)__shfl((int)(row >> 32), from) << 32;
            };
#pragma unroll
            for (int i = 0; i < 2; ++i) load_k(r, i, a.k_plane + row_of(16 * i + col) * kRow + g * (kRow / 4));
#pragma unroll
            for (int e = 0; e < 8; ++e)
                load_v(r, e, a.v_plane + row_of((e < 4 ? 0 : 16) + 4 * g + (e & 3)) * kRow + col * (kRow / 16));
        }
    };

    Raw raw;
    if (n_mine > 0) load_chunk(raw, 0);

    // ---- the queries as operands: row col of tile m, dims 32 g + 8 j .. + 7 ----
    u32x4_t qf[MT][4];
    float kq[MT];  // scores in log2 units per unit of the products, without K's exponent
#pragma unroll
    for (int m = 0; m < MT; ++m) {
        const uint4 *qp =
            reinterpret_cast<const uint4 *>(a.q + query_row(min(16 * m + col, rows - 1)) * kHeadDim + 32 * g);
        uint4 u[4];
        float top = 0.0f;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            u[j] = qp[j];
            const uint32_t x[4] = {u[j].x, u[j].y, u[j].z, u[j].w};
#pragma unroll
            for (int e = 0; e < 4; ++e) top = fmax3_abs(top, bf16_lo(x[e]), bf16_hi(x[e]));
        }
        const int e_q = exponent_of(max_kg(top));
        const float s = ldexpf(1.0f, kQTop - e_q);
        kq[m] = kLog2e * rsqrtf((float)kHeadDim) * ldexpf(1.0f, e_q - kQTop);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint32_t x[4] = {u[j].x, u[j].y, u[j].z, u[j].w};
#pragma unroll
            for (int e = 0; e < 4; ++e) qf[m][j][e] = pack_f16_rne(bf16_lo(x[e]) * s, bf16_hi(x[e]) * s);
        }
    }

    // ---- running state ----
    float m_ref[MT], l_part[MT];  // row col: the reference, the lane's share of the sum
    f32x4_t o[MT][8];             // rows 4 g + i, dim 8 col + n, in units of 2^(e_v - kKvTop)
#pragma unroll
    for (int m = 0; m < MT; ++m) {
        m_ref[m] = -INFINITY;
        l_part[m] = 0.0f;
#pragma unroll
        for (int n = 0; n < 8; ++n) o[m][n] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    }
    int e_k = kLeast, e_v = kLeast;  // |b| + |m| < 2^e so far

    const uint32_t lane4 = 4u * lane;
    // the entry of byte `by` of a word of the planes
    auto look = [&](uint32_t word, int by) -> uint32_t {
        return *reinterpret_cast<const uint32_t *>(lds + __builtin_amdgcn_perm(word, lane4, 0x0c0c0400u + ((uint32_t)by << 8)));
    };

    for (int j = 0; j < n_mine; ++j) {
        const int t0 = __builtin_amdgcn_readfirstlane(chunk_t0(j));
        // ---- the chunk's maps, scaled, to LDS and back in the operands' layouts ----
        {
            const float kb0 = raw.ks.x * raw.kgs.x, kb1 = raw.ks.y * raw.kgs.y;
            const float km0 = fmaf(raw.km.x, raw.kgs.x, raw.kgm.x), km1 = fmaf(raw.km.y, raw.kgs.y, raw.kgm.y);
            const float vb0 = raw.vs.x * raw.vgs.x, vb1 = raw.vs.y * raw.vgs.y;
            const float vm0 = fmaf(raw.vm.x, raw.vgs.x, raw.vgm.x), vm1 = fmaf(raw.vm.y, raw.vgs.y, raw.vgm.y);
            const float kt = fmaxf(fabsf(kb0) + fabsf(km0), fabsf(kb1) + fabsf(km1));
            const float vt = fmaxf(fabsf(vb0) + fabsf(vm0), fabsf(vb1) + fabsf(vm1));
            if (__any(kt >= ldexpf(1.0f, e_k))) e_k = max(e_k, __builtin_amdgcn_readfirstlane(exponent_of(wave_max(kt))));
            if (__any(vt >= ldexpf(1.0f, e_v))) {
                const int e = max(e_v, __builtin_amdgcn_readfirstlane(exponent_of(wave_max(vt))));
                const float f = ldexpf(1.0f, max(e_v - e, -120));
#pragma unroll
                for (int m = 0; m < MT; ++m)
#pragma unroll
                    for (int n = 0; n < 8; ++n)
#pragma unroll
                        for (int i = 0; i < 4; ++i) o[m][n][i] *= f;
                e_v = e;
            }
            const float sk = ldexpf(1.0f, kKvTop - e_k), sv = ldexpf(1.0f, kKvTop - e_v);
            uint32_t *st = reinterpret_cast<uint32_t *>(stage) + lane;
            st[0] = pack_f16_rne(kb0 * sk, kb1 * sk);
            st[64] = pack_f16_rne(km0 * sk, km1 * sk);
            st[128] = pack_f16_rne(vb0 * sv, vb1 * sv);
            st[192] = pack_f16_rne(vm0 * sv, vm1 * sv);
        }
        // ---- scores of the 32 tokens ----
        f32x4_t sc[MT][2];
#pragma unroll
        for (int m = 0; m < MT; ++m) sc[m][0] = sc[m][1] = f32x4_t{0.f, 0.f, 0.f, 0.f};
        const uint4 *kb = reinterpret_cast<const uint4 *>(stage + 64 * g);
#pragma unroll
        for (int jj = 0; jj < 4; ++jj) {
            const uint4 bb = kb[jj], mm = kb[16 + jj];
            const uint32_t bw[4] = {bb.x, bb.y, bb.z, bb.w}, mw[4] = {mm.x, mm.y, mm.z, mm.w};
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                u32x4_t kf;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const uint32_t lv = FULL ? low16s(look(raw.k[i][2 * jj % kKW + e / 2], 2 * (e & 1)),
                                                      look(raw.k[i][2 * jj % kKW + e / 2], 2 * (e & 1) + 1))
                                             : look(raw.k[i][jj], e);
                    kf[e] = pk_fma(lv, bw[e], mw[e]);
                }
#pragma unroll
                for (int m = 0; m < MT; ++m) sc[m][i] = mfma_f16(kf, qf[m][jj], sc[m][i]);
            }
        }
        // ---- softmax weights, the second product's first operand ----
        u32x4_t pf[MT];
        const float ek = ldexpf(1.0f, e_k - kKvTop);
        const int left = T - t0;  // tokens of the chunk
#pragma unroll
        for (int m = 0; m < MT; ++m) {
            float x[8];
            const float s = kq[m] * ek;
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = sc[m][e >> 2][e & 3] * s;
            if (left < kChunk) {
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if ((e < 4 ? 0 : 16) + 4 * g + (e & 3) >= left) x[e] = -INFINITY;
            }
            const float top = max_kg(fmax3(fmax3(x[0], x[1], x[2]), fmax3(x[3], x[4], x[5]), fmax2(x[6], x[7])));
            if (__any(top > m_ref[m] + (float)kSlack)) {
                const float next = fmax2(m_ref[m], top);
                const float f = m_ref[m] == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(m_ref[m] - next);
                m_ref[m] = next;
                l_part[m] *= f;
                float fr[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) fr[i] = __shfl(f, 4 * g + i);
#pragma unroll
                for (int n = 0; n < 8; ++n)
#pragma unroll
                    for (int i = 0; i < 4; ++i) o[m][n][i] *= fr[i];
            }
            const float off = m_ref[m] - (float)kPTop;
            float p[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) p[e] = __builtin_amdgcn_exp2f(x[e] - off);
            l_part[m] += ((p[0] + p[1]) + (p[2] + p[3])) + ((p[4] + p[5]) + (p[6] + p[7]));
#pragma unroll
            for (int e = 0; e < 4; ++e) pf[m][e] = pack_f16_rne(p[2 * e], p[2 * e + 1]);
        }
        // ---- weights times values ----
        {
            const uint4 bb = reinterpret_cast<const uint4 *>(stage + 512)[col];
            const uint4 mm = reinterpret_cast<const uint4 *>(stage + 768)[col];
            const uint32_t bw[4] = {bb.x, bb.y, bb.z, bb.w}, mw[4] = {mm.x, mm.y, mm.z, mm.w};
#pragma unroll
            for (int n2 = 0; n2 < 4; ++n2) {  // dims 8 col + 2 n2, + 1
                uint32_t x[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const uint32_t lv = FULL ? low16s(look(raw.v[e][n2 / 2 % kVW], 2 * (n2 & 1)),
                                                      look(raw.v[e][n2 / 2 % kVW], 2 * (n2 & 1) + 1))
                                             : look(raw.v[e][0], n2);
                    x[e] = pk_fma(lv, bw[n2], mw[n2]);
                }
                u32x4_t lo, hi;
#pragma unroll
                for (int d = 0; d < 4; ++d) {
                    lo[d] = low16s(x[2 * d], x[2 * d + 1]);
                    hi[d] = high16s(x[2 * d], x[2 * d + 1]);
                }
#pragma unroll
                for (int m = 0; m < MT; ++m) {
                    o[m][2 * n2] = mfma_f16(pf[m], lo, o[m][2 * n2]);
                    o[m][2 * n2 + 1] = mfma_f16(pf[m], hi, o[m][2 * n2 + 1]);
                }
            }
        }
        if (j + 1 < n_mine) load_chunk(raw, j + 1);
    }

    // ---- the wavefronts meet: (max, sum) of every row, then the outputs ----
    float2 *s_ml = reinterpret_cast<float2 *>(share);  // [wave][16 MT]
    const bool any_bad = __any(bad);                   // a block id outside the pool: NaN sums
    __syncthreads();                                   // every wavefront is done with its stage
#pragma unroll
    for (int m = 0; m < MT; ++m) {
        const float l = sum_kg(l_part[m]) * ldexpf(1.0f, -kPTop);
        if (g == 0) s_ml[w * 16 * MT + 16 * m + col] = make_float2(m_ref[m], any_bad ? NAN : l);
    }
    __syncthreads();
    const int row = tid >> 4, c16 = tid & 15;  // as the thread writes: row of a tile, dims 8 c16 ..
    float f[MT][kWaves], M[MT], L[MT];
#pragma unroll
    for (int m = 0; m < MT; ++m) {
        float2 ml[kWaves];
        M[m] = -INFINITY;
        L[m] = 0.0f;
#pragma unroll
        for (int ww = 0; ww < kWaves; ++ww) {
            ml[ww] = s_ml[ww * 16 * MT + 16 * m + row];
            M[m] = fmaxf(M[m], ml[ww].x);
        }
#pragma unroll
        for (int ww = 0; ww < kWaves; ++ww) {
            f[m][ww] = ml[ww].x == -INFINITY ? 0.0f : exp2f(ml[ww].x - M[m]);
            L[m] = fmaf(ml[ww].y, f[m][ww], L[m]);
        }
    }
    __syncthreads();
    const size_t pseg0 = prow0 * a.n_seg + seg.number0;
    const uint32_t prows = (uint32_t)(rows - 1) * a.n_seg + live;  // from the first row's first segment
    const __amdgpu_buffer_rsrc_t pair_o = buffer_rsrc(a.ws_o + pseg0 * kHeadDim, prows * kHeadDim * 4);
    const __amdgpu_buffer_rsrc_t pair_ml = buffer_rsrc(a.ws_ml + pseg0, prows * 8);
    const bool merge = a.fused && live > 1;
    const float unit = ldexpf(1.0f, e_v - kKvTop - kPTop);
    float4 *s_o = reinterpret_cast<float4 *>(share);  // [wave][row][16]: dims 8 c + 4 half ..
#pragma unroll
    for (int m = 0; m < MT; ++m) {
#pragma unroll
        for (int half = 0; half < 2; ++half) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                s_o[(w * 16 + 4 * g + i) * 16 + col] =
                    make_float4(o[m][4 * half][i] * unit, o[m][4 * half + 1][i] * unit, o[m][4 * half + 2][i] * unit,
                                o[m][4 * half + 3][i] * unit);
            __syncthreads();
            float4 O = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int ww = 0; ww < kWaves; ++ww) {
                const float4 x = s_o[(ww * 16 + row) * 16 + c16];
                O.x = fmaf(x.x, f[m][ww], O.x);
                O.y = fmaf(x.y, f[m][ww], O.y);
                O.z = fmaf(x.z, f[m][ww], O.z);
                O.w = fmaf(x.w, f[m][ww], O.w);
            }
            const int r = 16 * m + row, d4 = 2 * c16 + half;
            if (r < rows) {
                if (merge) {
                    const uint32_t sp = (uint32_t)r * a.n_seg + (seg.number - seg.number0);
                    store16_agent(pair_o, (sp * kHeadDim + 4 * d4) * 4, O);
                    if (d4 == 0) store8_agent(pair_ml, sp * 8, make_float2(M[m], L[m]));
                } else if (a.fused) {  // the whole sequence is this worker's
                    write_row4(a.out, a.lse, query_row(r), d4, O, M[m], L[m]);
                } else {
                    const size_t pi = (prow0 + r) * a.n_seg + seg.number;
                    reinterpret_cast<float4 *>(a.ws_o + pi * kHeadDim)[d4] = O;
                    if (d4 == 0) a.ws_ml[pi] = make_float2(M[m], L[m]);
                }
            }
            __syncthreads();
        }
    }
    if (!merge) return;
    // ---- fused merge (one row tile, one query a sequence): the last to arrive ----
    if (MT == 1) {
        int *flag = reinterpret_cast<int *>(share + kShare - 16);
        unsigned *ctr = a.counters + (((size_t)b * Hkv + h) * a.row_chunks) * kCounterStride;
        if (last_to_arrive(ctr, live, flag)) {
            const size_t orow0 = query_row(0);
            if (rows <= 4)
                merge_pair<4>(a, pair_o, pair_ml, orow0, rows, live, share);
            else if (rows <= 8)
                merge_pair<8>(a, pair_o, pair_ml, orow0, rows, live, share);
            else
                merge_pair<16>(a, pair_o, pair_ml, orow0, rows, live, share);
        }
    }
}

// The table's entry of every plane byte, in 64 copies.
template <int FULL>
__device__ __forceinline__ void fill_table(const HierArgs &a, uint8_t *lds) {
    const int tid = threadIdx.x;
    // the thread's byte, its entry, then rows of 64 copies, 16 bytes a lane
    uint32_t entry;
    if (FULL) {
        const uint32_t x = __builtin_bit_cast(uint16_t, signed_level_f16<1>(a.alpha, a.log1p_alpha, a.variant, tid >> 4, tid & 15));
        entry = x | x << 16;
    } else {
        entry = __builtin_bit_cast(uint16_t, signed_level_f16<0>(a.alpha, a.log1p_alpha, a.variant, tid & 15, 0)) |
                (uint32_t)__builtin_bit_cast(uint16_t, signed_level_f16<0>(a.alpha, a.log1p_alpha, a.variant, tid >> 4, 0)) << 16;
    }
    const int lane = tid & 63, w = tid >> 6;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
        const uint32_t x = __shfl(entry, 4 * r + (lane >> 4));
        *reinterpret_cast<uint4 *>(lds + (size_t)(64 * w + 4 * r + (lane >> 4)) * 256 + 16 * (lane & 15)) =
            make_uint4(x, x, x, x);
    }
    __syncthreads();
}

// Grid (worker, kv head x row chunk) for the contiguous layout, the kv head fastest
// for paged ones (anchor_decode.hip); with a workgroup per unit the sequence in z.
// WALK: the workgroup walks a list of segments.
template <int MT, int FULL, int LAYOUT, bool WALK>
__global__ __launch_bounds__(kThreads, 2) void hier_attn_kernel(HierArgs a) {
    __shared__ __attribute__((aligned(1024))) uint8_t lds[kTable + kShare];
    const int worker = LAYOUT == 0 ? blockIdx.x : blockIdx.y;
    const int hc = LAYOUT == 0 ? blockIdx.y : blockIdx.x;
    Segment<kWorkUnit> seg;
    if (!WALK) {
        if (!seg.set_unit(a.seq_lens, a.max_seq_len, a.direct, blockIdx.z, worker)) return;
        if (seg.n_groups > 0) fill_table<FULL>(a, lds);
        attend_segment<MT, FULL, LAYOUT>(a, seg, hc % a.geo.Hkv, hc / a.geo.Hkv, threadIdx.x, lds);
        return;
    }
    const WorkList<kWorkUnit, true> list(a.seq_lens, a.B, a.max_seq_len, a.workers);
    if (!seg.start(list, worker)) return;
    fill_table<FULL>(a, lds);
    for (;;) {
        attend_segment<MT, FULL, LAYOUT>(a, seg, fresh_uniform(hc % a.geo.Hkv), fresh_uniform(hc / a.geo.Hkv), fresh_tid(), lds);
        if (!seg.next(list, worker)) return;
        __syncthreads();  // the segment's LDS is free again
    }
}

template <int MT, int FULL, int LAYOUT>
void launch_walk(const HierArgs &args, dim3 grid, hipStream_t stream) {
    if (args.direct)
        hipLaunchKernelGGL((hier_attn_kernel<MT, FULL, LAYOUT, false>), grid, dim3(kThreads), 0, stream, args);
    else
        hipLaunchKernelGGL((hier_attn_kernel<MT, FULL, LAYOUT, true>), grid, dim3(kThreads), 0, stream, args);
}

template <int MT, int FULL>
void launch_layout(const HierArgs &args, dim3 grid, hipStream_t stream) {
    if (args.geo.max_blocks == 1)
        launch_walk<MT, FULL, 0>(args, grid, stream);
    else if (args.geo.bt % 16 == 0)
        launch_walk<MT, FULL, 1>(args, grid, stream);
    else
        launch_walk<MT, FULL, 2>(args, grid, stream);
}

}  // namespace

hipError_t launch_hier_attn(const HierArgs &args, hipStream_t stream) {
    if (args.workers < 1 || args.workers > 65535) return hipErrorInvalidValue;
    const int tile = args.rows_total > 16 ? 32 : 16;
    const unsigned hc = (unsigned)(args.geo.Hkv * ((args.rows_total + tile - 1) / tile));
    const unsigned n = args.direct ? args.direct : args.workers, nz = args.direct ? args.B : 1;
    const dim3 grid = args.geo.max_blocks == 1 ? dim3(n, hc, nz) : dim3(hc, n, nz);
    if (tile == 16) {
        if (args.full) launch_layout<1, 1>(args, grid, stream);
        else launch_layout<1, 0>(args, grid, stream);
    } else {
        if (args.full) launch_layout<2, 1>(args, grid, stream);
        else launch_layout<2, 0>(args, grid, stream);
    }
    return hipGetLastError();
}

}  // namespace lynx
