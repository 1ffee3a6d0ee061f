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
// likewise (2^-11 of itself, 2^-32 of the row's largest).  Scores, softmax statistics
// and outputs are fp32.  Powers of two keep the operands in fp16's range whatever the
// cache's: K and V are scaled by an exponent each that brings the largest |b| + |m| so
// far below 2^14, so values 2^-28 of the largest lose bits: b, m and x 2^-25 each, three
// times 2^-38 of the largest; a query row by its largest element to below 2^10, so its
// elements from 2^-26 of that on are exact and smaller ones off by 2^-34 of it.  A level
// is not scaled: below 2^-14, where alpha of 1000 and more puts the smallest codes, it
// is off by 2^-25, x by that of b.
//
// What bounds it.  Long decodes, memory: 4 sequences of 64K, 64 heads over 8, 85.6 us,
// 419 MB, 4.9 TB/s (a large copy 5.1); with its loads left out the same takes 58 us.
// Many rows, the vector ALU and LDS: per 32 tokens a wavefront makes operands in
// some 250 vector instructions (450 from merged codes; a v_perm, a packed multiply-add
// or a conversion takes 4.5 cycles of its SIMD) and 64 lookups (2.3 cycles of the CU's
// LDS each, 128 from merged codes), then 35 instructions and 16 matrix products per 16
// rows; 20 queries over 32K of merged codes, 80 rows a kv head, 54 us.  Short ones, the
// launch and a chain of latencies: 4K 13.1 us.
// Why so: the levels by table, since the transform's inverse is an exponential per
// element; 64 copies of it, so that an address is one instruction (32 copies are read
// as fast, but take two); lookups in batches of 16, what LDS counts; queries of 32 rows
// at most, what two wavefronts a SIMD hold (before shares were cut in groups those 20
// queries took 60.5 us, with 64 and 80 rows at one a SIMD 71 and 99).  Operands made
// once for 64 to 256 rows by 8 wavefronts through LDS cost more up to 64 rows a kv head
// (38 us, so 40; 32K) and gain from 128 on (70 us, so 59; 512 rows of 2 x 16K 157 us, so
// 120) where the workspace holds four times the partials; it is not built, since this
// call takes the workspace of the other attention calls, with which it loses (256 rows
// of 32K 90 us, so 151).  Shares of whole groups of 128 tokens: even_share.
#include "f16_ops.h"
#include "hier_ops.h"
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
constexpr int kChunk = kHierChunk;  // tokens of a wavefront's step
constexpr float kLog2e = 1.4426950408889634f;

// LDS: the table, then 16 KB: while the wavefronts attend, a stage each for a chunk's
// maps, and the queries; at the end what they join.  80 KB, two workgroups per CU.
constexpr int kShare = 16384;

// One segment of a worker's share, kv head h, rows r0 .. r0 + 16 MT - 1.
// A wavefront owns a quarter of the segment's chunks and attends them with an online
// softmax of its own: no barrier in the loop.
//
// Layouts of a wavefront's step (col = lane % 16, g = lane / 16): the scores are
// computed as K Q^T, lane (col, g) holding query row col against tokens 4 g + i and
// 16 + 4 g + i (i < 4).  That is the first operand of the second product as it
// stands, where slot e of group g is then token 4 g + e or 16 + 4 g + e - 4; the
// lane's eight V rows are those tokens', of which it takes dims 8 col .. + 7, one a
// tile of 16 columns, so an output lane holds dims 8 col .. + 7 of rows 4 g + i.
//
// LAYOUT 0: one block per sequence; 1: block_tokens a multiple of 16; 2: any other.
// FILL: the table is still to be made.
template <int MT, int FULL, int LAYOUT, bool FILL>
__device__ __forceinline__ void attend_segment(const HierArgs &a, const Segment<kWorkUnit> &seg, int h, int chunk_rows,
                                               const int tid, uint8_t *lds) {
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
    uint8_t *share = lds + kTableBytes;
    uint8_t *stage = share + w * kStageBytes;  // K: b, m, V: b, m of a chunk, [128] fp16 each

    // ---- where a token's rows are ----
    bool bad = false;
    const int32_t *bt_row = a.block_table + (size_t)b * a.geo.max_blocks;
    auto block_index = [&](int t) { return LAYOUT == 0 ? 0 : a.bt_shift >= 0 ? (t >> a.bt_shift) : t / a.geo.bt; };
    auto block_row0 = [&](int t, int blk) -> size_t {  // the row of token t in its block blk
        if (blk < 0 || blk >= a.geo.num_blocks) {
            bad = true;
            blk = 0;
        }
        return ((size_t)blk * Hkv + h) * a.geo.bt + (size_t)(t - block_index(t) * a.geo.bt);
    };

    // ---- the wavefront's chunks: a quarter of the segment's, one after the other ----
    const int base_t = seg.g0 * kKGroup;
    const int n_chunks = (min(seg.n_groups * kKGroup, T - base_t) + kChunk - 1) / kChunk;
    const int c0 = __builtin_amdgcn_readfirstlane(n_chunks * w / kWaves);
    const int n_mine = __builtin_amdgcn_readfirstlane(n_chunks * (w + 1) / kWaves) - c0;
    auto chunk_t0 = [&](int j) { return base_t + kChunk * (c0 + j); };

    // ---- loads of a chunk: keys, values, scalars ----
    // Past the last chunk they load that one again: every step issues as many, so a
    // wait for one of them is no wait for those behind it.
    uint32_t rk[2][kKW];  // token 16 i + col, bytes kRow / 4 * g ..
    uint32_t rv[8][kVW];  // token slot e, dims 8 col .. + 7
    float2 rm[8];         // channels 2 lane, 2 lane + 1: K's sigma, mu, gscale, gmin, V's
    // LAYOUT 1: the blocks of four chunks' eight 16-token runs, run r in lane r, loaded
    // four chunks ahead of the rows (entries past the table's end are clamped and unused)
    int ids = 0, ids_next = 0;
    auto load_ids = [&](int j) {
        if (LAYOUT == 1) ids_next = bt_row[min(block_index(chunk_t0(j) + 16 * (lane & 7)), a.geo.max_blocks - 1)];
    };
    // Where chunk j's rows are: run(i, offset of the first) for its two runs of 16 tokens
    // where each lies in one block, else each(row_of), row_of(t) the offset of its token t.
    auto rows_of_chunk = [&](int j, int run_ids, auto run, auto each) {
        const int t0 = __builtin_amdgcn_readfirstlane(chunk_t0(j));
        if (LAYOUT != 2 && t0 + kChunk <= T) {
#pragma unroll
            for (int i = 0; i < 2; ++i)
                run(i, block_row0(t0 + 16 * i, LAYOUT == 0 ? run_ids : __builtin_amdgcn_readlane(run_ids, 2 * (j & 3) + i)) * kRow);
        } else {
            // a lookup per token, in lanes 0 .. 31; tokens past the context repeat the
            // last one
            const int t = min(t0 + (lane & 31), T - 1);
            const size_t row = block_row0(t, bt_row[block_index(t)]) * kRow;
            each([&](int from) -> size_t {
                return (size_t)(uint32_t)__shfl((int)(uint32_t)row, from) | (size_t)(uint32_t)__shfl((int)(row >> 32), from) << 32;
            });
        }
    };
    // (unsigned 32-bit lane offsets from uniform bases: a load then takes no arithmetic)
    const uint32_t k_off = col * kRow + g * (kRow / 4), v_off = 4 * g * kRow + col * (kRow / 16), m_off = 2 * lane;
    auto load_k = [&](int j, int run_ids) {
        auto put = [&](int i, const uint8_t *p) {
#pragma unroll
            for (int q = 0; q < kKW / 4; ++q) {
                const uint4 u = reinterpret_cast<const uint4 *>(p)[q];
                rk[i][4 * q] = u.x; rk[i][4 * q + 1] = u.y; rk[i][4 * q + 2] = u.z; rk[i][4 * q + 3] = u.w;
            }
        };
        rows_of_chunk(j, run_ids, [&](int i, size_t row) { put(i, a.k_plane + row + k_off); },
                      [&](auto row_of) {
#pragma unroll
                          for (int i = 0; i < 2; ++i) put(i, a.k_plane + row_of(16 * i + col) + (uint32_t)(g * (kRow / 4)));
                      });
    };
    auto load_v = [&](int j, int run_ids) {
        auto put = [&](int e, const uint8_t *p) {
            if (FULL) {
                const uint2 u = *reinterpret_cast<const uint2 *>(p);
                rv[e][0] = u.x;
                rv[e][kVW - 1] = u.y;
            } else {
                rv[e][0] = *reinterpret_cast<const uint32_t *>(p);
            }
        };
        rows_of_chunk(j, run_ids,
                      [&](int i, size_t row) {
#pragma unroll
                          for (int e = 0; e < 4; ++e)
                              put(4 * i + e, a.v_plane + row + e * kRow + v_off);
                      },
                      [&](auto row_of) {
#pragma unroll
                          for (int e = 0; e < 8; ++e)
                              put(e, a.v_plane + row_of((e < 4 ? 0 : 16) + 4 * g + (e & 3)) + col * (kRow / 16));
                      });
    };
    const size_t cmeta = ((size_t)b * Hkv + h) * a.geo.n_chunks * kHeadDim;
    const size_t pmeta = ((size_t)b * Hkv + h) * a.geo.n_pages * kHeadDim;
    auto load_meta = [&](int j) {
        const int t0 = __builtin_amdgcn_readfirstlane(chunk_t0(j));
        const size_t c = cmeta + (size_t)(t0 / kChunk) * kHeadDim, p = pmeta + (size_t)(t0 / kHierPage) * kHeadDim;
        const float *src[8] = {a.meta.k_sigma + c, a.meta.k_mu + c, a.meta.k_gscale + p, a.meta.k_gmin + p,
                               a.meta.v_sigma + c, a.meta.v_mu + c, a.meta.v_gscale + p, a.meta.v_gmin + p};
#pragma unroll
        for (int i = 0; i < 8; ++i) rm[i] = *reinterpret_cast<const float2 *>(src[i] + m_off);
    };
    const int last = n_mine - 1;
    // the next chunk of keys; j counts up by one from 0, and the values follow it
    auto next_k = [&](int j) {
        if (LAYOUT == 1 && (j & 3) == 0 && j <= last) {
            ids = ids_next;
            load_ids(j + 4);
        }
        load_k(min(j, last), ids);
    };
    if (LAYOUT == 0) ids = __builtin_amdgcn_readfirstlane(bt_row[0]);
    if (n_mine > 0) {
        load_meta(0);
        load_ids(0);
        next_k(0);
        load_v(0, ids);
    }

    if (FILL) fill_table<FULL>(a, lds);  // (the first rows are on their way)

    // ---- the queries as operands, in LDS: row col of tile m, dims 32 g + 8 j .. + 7
    // at piece 4 m + j; piece p is made by wavefront p % 4 ----
    u32x4_t *s_q = reinterpret_cast<u32x4_t *>(share + kStageBytes * kWaves);
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
        for (int j = 0; j < 4; ++j)
            if (w == j)
                s_q[(4 * m + j) * 64 + lane] =
                    u32x4_t{pack_f16_rne(bf16_lo(u[j].x) * s, bf16_hi(u[j].x) * s),
                            pack_f16_rne(bf16_lo(u[j].y) * s, bf16_hi(u[j].y) * s),
                            pack_f16_rne(bf16_lo(u[j].z) * s, bf16_hi(u[j].z) * s),
                            pack_f16_rne(bf16_lo(u[j].w) * s, bf16_hi(u[j].w) * s)};
    }
    __syncthreads();

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
    float k_lim = ldexpf(1.0f, kLeast), v_lim = k_lim;  // 2^e

    const uint32_t lane4 = 4u * lane;
    auto look = [&](uint32_t word, int by) { return look_up(lds, word, by, lane4); };
    // Lookups go in batches, each issued before the batch ahead of it is used, so their
    // latency passes behind that one's arithmetic: a chunk's keys in kParts of them,
    // then its values.
    constexpr int kLooks = FULL ? 64 : 32, kBatch = 16, kParts = kLooks / kBatch;
    uint32_t buf[2][kBatch];
    auto look_k = [&](int part) {
#pragma unroll
        for (int i = 0; i < kBatch; ++i) {
            const int n = part * kBatch + i;
            // slice n / 16, tile n / 8 % 2, byte n % 8 of its two words; or n / 8, n / 4 % 2, n % 4
            buf[part & 1][i] = FULL ? look(rk[n >> 3 & 1][(2 * (n >> 4) + (n >> 2 & 1)) % kKW], n & 3)
                                    : look(rk[n >> 2 & 1][(n >> 3) % kKW], n & 3);
        }
        __builtin_amdgcn_sched_barrier(0);
    };
    auto look_v = [&](int part) {
        if (!FULL && part == 0) {
            // two tokens' words of 8 dims become the even dims' and the odd dims' of both:
            // a byte, looked up, is then the operand's pair of token slots
#pragma unroll
            for (int e = 0; e < 8; e += 2) {
                const uint32_t x = rv[e][0], y = rv[e + 1][0];
                rv[e][0] = (x & 0x0F0F0F0Fu) | ((y << 4) & 0xF0F0F0F0u);
                rv[e + 1][0] = ((x >> 4) & 0x0F0F0F0Fu) | (y & 0xF0F0F0F0u);
            }
        }
#pragma unroll
        for (int i = 0; i < kBatch; ++i) {
            const int n = part * kBatch + i;
            // dim n / 8, token slot n % 8; or the pair of slots 2 (n % 4), + 1 of dim n / 4
            buf[(kParts + part) & 1][i] = FULL ? look(rv[n & 7][(n >> 5) % kVW], (n >> 3) & 3)
                                               : look(rv[2 * (n & 3) + (n >> 2 & 1)][0], n >> 3);
        }
        __builtin_amdgcn_sched_barrier(0);
    };
    // A chunk's maps, scaled, to the wavefront's stage.
    auto next_maps = [&]() {
        const Maps x = maps_of(rm);
        if (__any(x.k_top >= k_lim)) {
            e_k = max(e_k, __builtin_amdgcn_readfirstlane(exponent_of(wave_max(x.k_top))));
            k_lim = ldexpf(1.0f, e_k);
        }
        if (__any(x.v_top >= v_lim)) {
            const int e = max(e_v, __builtin_amdgcn_readfirstlane(exponent_of(wave_max(x.v_top))));
            const float f = ldexpf(1.0f, max(e_v - e, -120));
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int n = 0; n < 8; ++n)
#pragma unroll
                    for (int i = 0; i < 4; ++i) o[m][n][i] *= f;
            e_v = e;
            v_lim = ldexpf(1.0f, e_v);
        }
        stage_maps(x, e_k, e_v, lane, stage);
    };
    f32x4_t sc[MT][2];
    const u32x4_t *kmap = reinterpret_cast<const u32x4_t *>(stage + 64 * g);
    // What a batch of keys meets: its slices' maps and queries.  They are read ahead of
    // the lookups of the batch behind it: LDS answers in order.
    constexpr int kSlices = 4 / kParts;
    u32x4_t kb[kSlices], km[kSlices], qf[kSlices][MT];
    auto read_k = [&](int part) {
#pragma unroll
        for (int s = 0; s < kSlices; ++s) {
            kb[s] = kmap[kSlices * part + s];
            km[s] = kmap[16 + kSlices * part + s];
#pragma unroll
            for (int m = 0; m < MT; ++m) qf[s][m] = s_q[(4 * m + kSlices * part + s) * 64 + lane];
        }
        __builtin_amdgcn_sched_barrier(0);
    };
    // Scores by the slices of dims 32 g + 8 jj .. + 7 of a batch.
    auto scores = [&](int part) {
        const uint32_t *from = buf[part & 1];
#pragma unroll
        for (int s = 0; s < kSlices; ++s) {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                u32x4_t kf;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const uint32_t lv = FULL ? low16s(from[(16 * s + 8 * i + 2 * e) % kBatch], from[(16 * s + 8 * i + 2 * e + 1) % kBatch])
                                             : from[(8 * s + 4 * i + e) % kBatch];
                    kf[e] = pk_fma(lv, kb[s][e], km[s][e]);
                }
#pragma unroll
                for (int m = 0; m < MT; ++m) sc[m][i] = mfma_f16(kf, qf[s][m], sc[m][i]);
            }
        }
    };
    u32x4_t pf[MT];  // softmax weights, the second product's first operand
    auto weights = [&](int left) {  // tokens of the chunk
        const float ek = ldexpf(1.0f, e_k - kKvTop);
#pragma unroll
        for (int m = 0; m < MT; ++m) {
            float z[8];
            const float s = fmaxf(kq[m] * ek, FLT_MIN);  // (0 would not mask)
#pragma unroll
            for (int e = 0; e < 8; ++e) z[e] = sc[m][e >> 2][e & 3];
            if (left < kChunk) {
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if ((e < 4 ? 0 : 16) + 4 * g + (e & 3) >= left) z[e] = -INFINITY;
            }
            const float top = max_kg(fmax3(fmax3(z[0], z[1], z[2]), fmax3(z[3], z[4], z[5]), fmax2(z[6], z[7]))) * s;
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
            const float off = (float)kPTop - m_ref[m];
#pragma unroll
            for (int e = 0; e < 8; ++e) z[e] = __builtin_amdgcn_exp2f(fmaf(z[e], s, off));
            l_part[m] += ((z[0] + z[1]) + (z[2] + z[3])) + ((z[4] + z[5]) + (z[6] + z[7]));
#pragma unroll
            for (int e = 0; e < 4; ++e) pf[m][e] = pack_f16_rne(z[2 * e], z[2 * e + 1]);
        }
    };
    // Weights times the values of a batch: operands of dim 8 col + n hold slots 2 d, 2 d + 1.
    u32x4_t bw, mw;  // the maps of dims 8 col .. + 7
    auto values = [&](int part) {
        const uint32_t *from = buf[(kParts + part) & 1];
        constexpr int kPer = 8 / kParts;
#pragma unroll
        for (int s = 0; s < kPer; ++s) {
            const int n = kPer * part + s;
            u32x4_t v;
            const uint32_t b1 = n & 1 ? high16s(bw[n >> 1 & 3], bw[n >> 1 & 3]) : low16s(bw[n >> 1 & 3], bw[n >> 1 & 3]);
            const uint32_t m1 = n & 1 ? high16s(mw[n >> 1 & 3], mw[n >> 1 & 3]) : low16s(mw[n >> 1 & 3], mw[n >> 1 & 3]);
#pragma unroll
            for (int d = 0; d < 4; ++d)
                v[d] = pk_fma(FULL ? low16s(from[(8 * s + 2 * d) % kBatch], from[(8 * s + 2 * d + 1) % kBatch])
                                   : from[(4 * s + d) % kBatch],
                              b1, m1);
#pragma unroll
            for (int m = 0; m < MT; ++m) o[m][n & 7] = mfma_f16(pf[m], v, o[m][n & 7]);
        }
    };
    if (n_mine > 0) {
        next_maps();
        load_meta(min(1, last));
        look_k(0);
    }
    for (int j = 0; j < n_mine; ++j) {
#pragma unroll
        for (int m = 0; m < MT; ++m) sc[m][0] = sc[m][1] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int part = 0; part < kParts; ++part) {
            read_k(part);
            if (part + 1 < kParts) {
                look_k(part + 1);
                if (part + 2 == kParts) next_k(j + 1);
            } else {
                look_v(0);
            }
            scores(part);
        }
        bw = reinterpret_cast<const u32x4_t *>(stage + 512)[col];
        mw = reinterpret_cast<const u32x4_t *>(stage + 768)[col];
        weights(T - chunk_t0(j));
#pragma unroll
        for (int part = 0; part < kParts; ++part) {
            if (part + 1 < kParts) {
                look_v(part + 1);
                if (part + 2 == kParts) load_v(min(j + 1, last), ids);
            } else {
                look_k(0);
            }
            values(part);
        }
        next_maps();
        load_meta(min(j + 2, last));
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

// Grid (worker, kv head x row chunk) for the contiguous layout, the kv head fastest
// for paged ones (anchor_decode.hip); with a workgroup per unit the sequence in z.
// WALK: the workgroup walks a list of segments.
template <int MT, int FULL, int LAYOUT, bool WALK>
__global__ __launch_bounds__(kThreads, 2) void hier_attn_kernel(HierArgs a) {
    __shared__ __attribute__((aligned(1024))) uint8_t lds[kTableBytes + kShare];
    const int worker = LAYOUT == 0 ? blockIdx.x : blockIdx.y;
    const int hc = LAYOUT == 0 ? blockIdx.y : blockIdx.x;
    Segment<kWorkUnit> seg;
    if (!WALK) {
        if (!seg.set_unit(a.seq_lens, a.max_seq_len, a.direct, blockIdx.z, worker)) return;
        attend_segment<MT, FULL, LAYOUT, true>(a, seg, hc % a.geo.Hkv, hc / a.geo.Hkv, threadIdx.x, lds);
        return;
    }
    const WorkList<kWorkUnit, true> list(a.seq_lens, a.B, a.max_seq_len, a.workers);
    if (!seg.start_even(list, worker)) return;
    fill_table<FULL>(a, lds);
    for (;;) {
        attend_segment<MT, FULL, LAYOUT, false>(a, seg, fresh_uniform(hc % a.geo.Hkv), fresh_uniform(hc / a.geo.Hkv),
                                                fresh_tid(), lds);
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

// 32 rows a workgroup where there are more than 16, whose operands are then made half
// as often: 20 rows of 32K of merged codes 29.8 us, so 37.2 in tiles of 16; 80 rows
// 55.6, so 67.7; 16 paged sequences of 1K-8K with 20 rows 56.5, so 75.6 (32 rows of 2000
// tokens, all latency, 20.6, so 17.5).
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
