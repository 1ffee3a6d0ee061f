// Internal declarations shared by the HIP translation units of liblynx.so.
// Not part of the public ABI (include/lynx.h is).
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace lynx {

constexpr int kHeadDim = 128;    // D
constexpr int kKGroup = 128;     // tokens per K quantization group
constexpr int kNibbleRow = 64;   // bytes per token row of a nibble plane
constexpr int kCodeRow = 128;    // bytes per token row of a code plane

// Geometry of a plane pool as the kernels see it.
struct Geometry {
    int Hkv;
    int bt;            // tokens per block
    int max_blocks;    // block_table row stride
    int num_blocks;    // valid block ids are [0, num_blocks)
    int max_tokens;    // metadata token stride
    int n_groups;      // ceil(max_tokens / 128): K metadata group stride
    int n_pages;       // ceil(max_tokens / 256): hierarchical page stride
    int n_chunks;      // ceil(max_tokens / 32): hierarchical chunk stride
};

struct MetaPtrs {
    float *k_scale, *k_zero, *v_scale, *v_zero;
};

// ---- encode / merge (codec.hip) ---------------------------------------------
hipError_t launch_encode(const Geometry &g, int b, int T, const int32_t *block_table,
                         const uint16_t *k, const uint16_t *v, uint8_t *k_anc, uint8_t *v_anc,
                         uint8_t *k_res, uint8_t *v_res, MetaPtrs meta, hipStream_t stream,
                         int anchor_bits = 4);
// Split widths other than 4 + 4: rows of 16 A-bit anchors per 16 A bytes
// (little-endian bit strings) and 16 (8 - A) residual bytes.
hipError_t launch_merge_split(int anchor_bits, const uint8_t *anc, const uint8_t *res, uint8_t *codes,
                              size_t n_rows, hipStream_t stream);
hipError_t launch_dequant_anchor_split(int anchor_bits, const Geometry &g, int b, int T,
                                       const int32_t *block_table, const uint8_t *k_anc,
                                       const uint8_t *v_anc, MetaPtrs meta, uint16_t *k_out,
                                       uint16_t *v_out, hipStream_t stream);
hipError_t launch_merge(const uint8_t *anc, const uint8_t *res, uint8_t *codes, size_t n_packed,
                        hipStream_t stream);

// ---- hierarchical codec of Alg. 1 (hier.hip) ----------------------------------
struct HMetaPtrs {
    float *k_gmin, *k_gscale, *k_mu, *k_sigma;  // [B][Hkv][n_pages][128], [B][Hkv][n_chunks][128]
    float *v_gmin, *v_gscale, *v_mu, *v_sigma;
};
// Codec variants (the values of lynx.h's LYNX_HQ_*).
constexpr int kHBiased = 0;
constexpr int kHCentred = 1;
constexpr int kHInt4 = 2;
// Per-(alpha, variant) tables, with M = 127 (7 for the 4-bit code): decision
// thresholds theta[k] = expm1((k + 0.5) / M * log1p(alpha)) / alpha for
// k < M, +inf beyond; levels level[i] = expm1(i / M * log1p(alpha)) / alpha
// (i <= M); the centred split's anchor-only levels alevel[V] at code
// 16 V + 7.5 of 127.  Each the fp32 value of the double expression.
// The encode's first guess at a code: yscale * log2(1 + alpha |Xf|), or
// yscale * |Xf| when `linear` (alpha < 1e-3), with yscale = M / log2(1 + alpha)
// (or M), is within one of the count the thresholds decide.
struct HTables {
    float theta[128];
    float level[128];
    float alevel[8];
    float alpha_h, one_h, yscale, yhalf;  // log2(one_h + alpha_h x) * yscale: the transform less half a code
    int linear;                           // x - yhalf in the logarithm's place
};
void make_htables(float alpha, int variant, HTables *t);
hipError_t launch_hencode(const Geometry &g, int b, int T, const int32_t *block_table,
                          const uint16_t *k, const uint16_t *v, uint8_t *k_anc, uint8_t *v_anc,
                          uint8_t *k_res, uint8_t *v_res, HMetaPtrs meta, const HTables &tab,
                          int variant, hipStream_t stream);
hipError_t launch_hdequant(bool full, const Geometry &g, int b, int T, const int32_t *block_table,
                           const uint8_t *k_plane, const uint8_t *v_plane, HMetaPtrs meta,
                           const HTables &tab, int variant, uint16_t *k_out, uint16_t *v_out,
                           hipStream_t stream);

// ---- serializer / deserializer (codec.hip) -----------------------------------
// Object: tokens t0 .. t0 + n - 1 of one sequence, all kv heads.  Anchor
// buffer: K, V anchor rows [Hkv][n][64], K scales, K zeros [Hkv][ceil(n/128)][128],
// V scales, V zeros [Hkv][n]; residual buffer: K, V residual rows.
hipError_t launch_serialize(int Hkv, int n, const uint16_t *k, const uint16_t *v,
                            uint8_t *anc_buf, uint8_t *res_buf, hipStream_t stream);
hipError_t launch_deserialize_anchor(const Geometry &g, int b, int t0, int n,
                                     const int32_t *block_table, const uint8_t *buf,
                                     uint8_t *k_anc, uint8_t *v_anc, MetaPtrs meta,
                                     hipStream_t stream);
hipError_t launch_deserialize_residual(const Geometry &g, int b, int t0, int n,
                                       const int32_t *block_table, const uint8_t *buf,
                                       const uint8_t *k_anc, const uint8_t *v_anc,
                                       uint8_t *k_codes, uint8_t *v_codes, hipStream_t stream);

// ---- attention (attention.hip) ----------------------------------------------
// Arrival counters at the head of every attention workspace (the value of
// lynx.h's LYNX_ATTN_COUNTER_BYTES): zero before a workspace's first use,
// left zero by every call.
// One counter per 256 bytes: arrivals on one cache line serialise (512
// workgroups counting in on one line took 5 us, 64 per line 0.4 us).
constexpr size_t kCounterBytes = 262144;
constexpr int kCounterStride = 64;  // uint32 slots between counters
constexpr int kCounters = (int)(kCounterBytes / (kCounterStride * sizeof(unsigned)));
enum class KvMode : int { kAnchor = 0, kCodes = 1, kAnchorSplit = 2, kCodesWide = 3, kCodesHalfWide = 4, kHier = 5 };

// 128-token groups per unit of the attention kernels' work list (work_list.h):
// one per wavefront of a workgroup.
constexpr int kWorkUnit = 4;

struct AttnPlan {
    int rows_total;   // nq * G query rows per (sequence, kv head)
    int direct;       // units of a sequence at most where each has a workgroup of its own, else 0
    int workers;      // workgroups per (kv head, row chunk)
    int n_seg;        // partials per query row: workers + B - 1, or B direct
    int max_live;     // partials of one sequence at most
    int row_chunks;   // ceil(rows_total / 16): arrival counters per (sequence, kv head)
    bool counters_fit;  // B * Hkv * row_chunks <= kCounters
    size_t o_bytes;   // workspace bytes for the partial outputs
    size_t ml_bytes;  // workspace bytes for the partial (max, sum) pairs
    // [arrival counters, kCounterBytes][outputs][(max, sum)]: the counters sit
    // at the same place for every call shape, so calls of different shapes
    // can share a workspace without one's partials landing on the counters
    size_t workspace_bytes() const { return kCounterBytes + o_bytes + ml_bytes; }
};

// Arguments of the matrix-core anchor decode kernel (anchor_decode.hip).
struct DecodeArgs {
    Geometry geo;
    int B, Hq, G, max_seq_len;
    int direct, workers, chunk_heads;
    int bt_shift;   // log2(block_tokens) when it is a power of two, else -1
    const int32_t *seq_lens;
    const int32_t *block_table;
    const uint8_t *k_anc;
    const uint8_t *v_anc;
    MetaPtrs meta;
    const uint16_t *q;
    float *ws_o;    // partials [Hkv][rows_total][n_seg][128]
    float2 *ws_ml;  // [Hkv][rows_total][n_seg]
    int rows_total, n_seg;
    // Fused merge: the last workgroup of a (sequence, kv head, head chunk) to
    // finish merges its partials and writes out / lse.
    // Arrival counters uint32 [B][Hkv][row_chunks], zero on entry, left zero.
    int fused;
    int row_chunks;
    unsigned *counters;
    uint16_t *out;  // BF16 [B][Hq][128]
    float *lse;     // fp32 [B][Hq] or nullptr
};

hipError_t launch_anchor_decode_mfma(const DecodeArgs &args, int chunks, hipStream_t stream);

// Arguments of the matrix-core verification kernel (verify.hip): the context
// only; the combine kernel attends the BF16 draft tail.
struct VerifyArgs {
    Geometry geo;
    int B, Hq, G, nq, max_seq_len;
    int rows_total;    // nq * G query rows per (sequence, kv head)
    int direct;        // as in AttnPlan
    int workers;       // workgroups per (kv head, row chunk)
    int n_seg;         // partials per row
    int bt_shift;      // log2(block_tokens) when it is a power of two, else -1
    const int32_t *seq_lens;
    const int32_t *block_table;
    const uint8_t *k_codes;
    const uint8_t *v_codes;
    MetaPtrs meta;
    const uint16_t *q;  // BF16 [B][nq][Hq][128]
    float *ws_o;
    float2 *ws_ml;
};

hipError_t launch_verify_mfma(const VerifyArgs &args, hipStream_t stream);
// The same for many rows a kv head (verify_wide.hip), `rows` per workgroup:
// kWideRows or half of them.
constexpr int kWideRows = 256;
hipError_t launch_verify_wide(const VerifyArgs &args, int rows, hipStream_t stream);

// Arguments of the anchor decode over split-width anchors (anchor_split.hip):
// one query per sequence over A-bit anchor planes (rows of 16 A bytes).
struct SplitDecodeArgs {
    Geometry geo;
    int B, Hq, G, max_seq_len;
    int anchor_bits;      // A: 2, 4 or 6
    int direct;           // as in AttnPlan
    int workers;          // workgroups per (kv head, row chunk)
    int bt_shift;         // log2(block_tokens) when it is a power of two, else -1
    int rows_total;       // G query rows per (sequence, kv head)
    int n_seg;            // partials per row
    const int32_t *seq_lens;
    const int32_t *block_table;
    const uint8_t *k_anc;
    const uint8_t *v_anc;
    MetaPtrs meta;
    const uint16_t *q;    // BF16 [B][Hq][128]
    float *ws_o;
    float2 *ws_ml;
    // merge in the same launch (as DecodeArgs): arrival counters
    // uint32 [B][Hkv][row_chunks], zero on entry, left zero
    int fused;
    int row_chunks;
    unsigned *counters;
    uint16_t *out;        // BF16 [B][Hq][128]
    float *lse;           // fp32 [B][Hq] or nullptr
};

hipError_t launch_anchor_split_decode(const SplitDecodeArgs &args, hipStream_t stream);

// Arguments of the attention over the hierarchical codec's planes (hier_attn.hip):
// the context only; the combine kernel attends the BF16 tail.
struct HierArgs {
    Geometry geo;
    int B, Hq, G, nq, max_seq_len;
    int rows_total;    // nq * G query rows per (sequence, kv head)
    int direct, workers, n_seg;  // as in AttnPlan
    int bt_shift;      // log2(block_tokens) when it is a power of two, else -1
    int full;          // merged codes instead of 4-bit planes
    int variant;
    float alpha, log1p_alpha;
    const int32_t *seq_lens;
    const int32_t *block_table;
    const uint8_t *k_plane;
    const uint8_t *v_plane;
    HMetaPtrs meta;
    const uint16_t *q;  // BF16 [B][nq][Hq][128]
    float *ws_o;
    float2 *ws_ml;
    // merge in the same launch (as DecodeArgs)
    int fused;
    int row_chunks;
    unsigned *counters;
    uint16_t *out;      // BF16 [B][nq][Hq][128]
    float *lse;         // fp32 [B][nq][Hq] or nullptr
};

hipError_t launch_hier_attn(const HierArgs &args, hipStream_t stream);

// The plan of a call; its workspace is at most `most` bytes where fewer workers
// can make it so.
AttnPlan plan_attention(KvMode mode, const Geometry &g, int B, int Hq, int nq, int max_seq_len,
                        size_t most = SIZE_MAX);
// Workspace bytes that suffice for every decode and verification of at most B
// sequences, nq queries each, and max_seq_len tokens, trees among them; and with
// which a tree has every kernel to choose from.
size_t attention_workspace_bound(const Geometry &g, int B, int Hq, int nq, int max_seq_len);
size_t tree_workspace_bound(const Geometry &g, int B, int Hq, int n, int max_seq_len);
// The kernel of a tree's context part: more rows a kv head than verify.hip's
// two row tiles serve at less cost.
KvMode tree_mode(const Geometry &g, int B, int Hq, int n, int max_seq_len);
// Bytes that lynx_attn_workspace_bytes reports at least for a decode, and that
// lynx_attn_anchor_decode_noalloc compares with its scratch.
size_t decode_limit_bytes(const Geometry &g, int B, int Hq, int max_seq_len);

// k_new / v_new: the BF16 tail, or nullptr.  Verification (kCodes): k drafts
// per sequence, causal among the drafts.  Decode (kAnchor, nq == 1):
// tail_count generated tokens per sequence, all visible to the query.
hipError_t launch_attention(KvMode mode, const Geometry &g, const AttnPlan &plan, int B, int Hq,
                            int nq, int max_seq_len, const int32_t *seq_lens,
                            const int32_t *block_table, const uint8_t *k_plane,
                            const uint8_t *v_plane, MetaPtrs meta, const uint16_t *q,
                            const uint16_t *k_new, const uint16_t *v_new, int tail_count,
                            uint16_t *out, float *lse, void *workspace, hipStream_t stream,
                            int anchor_bits = 4);

// Attention over the hierarchical codec's planes (plan_attention of KvMode::kHier):
// the context, then where there is a tail (n_tail BF16 tokens, of which query i of
// nq sees the first n_tail - nq + 1 + i) or the context's kernel does not merge its
// own partials, the combine kernel.
hipError_t launch_attn_hier(const Geometry &g, const AttnPlan &plan, int B, int Hq, int nq, int max_seq_len,
                            const int32_t *seq_lens, const int32_t *block_table, bool full, const uint8_t *k_plane,
                            const uint8_t *v_plane, float alpha, int variant, HMetaPtrs meta, const uint16_t *q,
                            int n_tail, const uint16_t *k_tail, const uint16_t *v_tail, uint16_t *out, float *lse,
                            void *workspace, hipStream_t stream);

// ---- verification of a token tree (attention.hip, tree.hip) --------------------
// Arguments of the merge of a tree's context partials with its own nodes.
struct TreeArgs {
    Geometry geo;
    int B, Hq, G, n, max_seq_len;  // n nodes per sequence (<= 64)
    int rows_total, direct, workers, n_seg, max_live;  // as in AttnPlan
    const int32_t *seq_lens;
    const int32_t *parents;        // [B][n]
    const uint16_t *q;             // BF16 [B][n][Hq][128]
    const uint16_t *k_new, *v_new; // BF16 [B][n][Hkv][128]
    const float *ws_o;
    const float2 *ws_ml;
    uint16_t *out;                 // BF16 [B][n][Hq][128]
};

// rows: those of a workgroup, 4 or 16.
hipError_t launch_tree_combine(const TreeArgs &args, int rows, hipStream_t stream);
// The tree's rows over the context (plan_attention of KvMode::kCodes, or
// kCodesWide, with n queries), then the merge.
hipError_t launch_verify_tree(KvMode mode, const Geometry &g, const AttnPlan &plan, int B, int Hq, int n, int max_seq_len,
                              const int32_t *seq_lens, const int32_t *block_table, const uint8_t *k_codes,
                              const uint8_t *v_codes, MetaPtrs meta, const uint16_t *q, const uint16_t *k_new,
                              const uint16_t *v_new, const int32_t *parents, uint16_t *out, void *workspace,
                              hipStream_t stream);

// ---- the cache written token by token, and read back (append.hip) --------------
// BF16 K rows kept per sequence behind its end (lynx.h's LYNX_OPEN_ROWS): the
// open 128-token group's and the one's before it.
constexpr int kOpenRows = 256;

struct AppendArgs {
    Geometry geo;
    int max_new, n_src;       // tokens appended at most; rows of k_new per sequence
    int capacity;             // tokens a sequence may hold
    int bt_shift;             // log2(block_tokens) when it is a power of two, else -1
    const int32_t *seq_lens;  // [B], before the append
    const int32_t *counts;    // [B]
    const int32_t *path;      // [B][max_new] rows of k_new, or nullptr: row i
    const int32_t *block_table;
    const uint16_t *k_new, *v_new;  // BF16 [B][n_src][Hkv][128]
    uint16_t *k_open;               // BF16 [B][kOpenRows][Hkv][128]
    uint8_t *codes[2], *anc[2], *res[2];  // planes of K and V, or nullptr
    MetaPtrs meta;
};

struct DequantArgs {
    Geometry geo;
    int max_n;                // rows of the output per sequence
    int unit0;                // the launch's first unit of rows (set by the launcher)
    int capacity;
    int bt_shift;
    const int32_t *starts;    // [B]; append_begin: the lengths
    const int32_t *counts;    // [B]
    const int32_t *block_table;
    const uint8_t *k_codes, *v_codes;
    MetaPtrs meta;
    uint16_t *k_out, *v_out;  // BF16 [B][max_n][Hkv][128]
};

hipError_t launch_append(const AppendArgs &args, int B, hipStream_t stream);
hipError_t launch_dequant(const DequantArgs &args, int B, hipStream_t stream);
hipError_t launch_append_begin(const DequantArgs &args, int B, hipStream_t stream);

// ---- norms and rotation of query and key heads (rope.hip) -----------------------
struct RopeArgs {
    int n_tokens, Hq, Hkv;
    int rotary;               // dims of a head that turn, a multiple of 16
    int pairs;                // dims 2 i and 2 i + 1 turn together, else i and i + rotary / 2
    int n_rows;               // of the outputs
    int64_t q_stride, k_stride, v_stride;  // elements between tokens
    const uint16_t *q, *k, *v;             // BF16 heads of 128; v may be nullptr
    const int32_t *positions; // [n_tokens]; negative: no token
    const int32_t *rows;      // [n_tokens] output rows, or nullptr: row n
    const uint16_t *q_weight, *k_weight;   // BF16 [128], or nullptr: no norm
    float eps, scale;
    const float *inv_freq;    // [rotary / 2]
    uint16_t *q_out, *k_out, *v_out;
};
hipError_t launch_rope(const RopeArgs &args, hipStream_t stream);

// ---- the plan of a step: blocks, slots, positions (blocks.hip) -------------------
struct BlocksArgs {
    int B, bt, max_blocks, num_blocks;
    int capacity;             // tokens a sequence may hold
    int n_src;                // new tokens per sequence at most
    int max_rows;             // of the token arrays
    const int32_t *seq_lens;  // [B]
    const int32_t *counts;    // [B] new tokens; of a release the tokens kept
    int32_t *block_table;     // [B][max_blocks]
    int32_t *free_blocks;     // [num_blocks]
    int32_t *state;           // blocks on the stack; arrivals, zero between calls
    int32_t *granted, *starts;  // [B], [B + 1]
    int32_t *seq_of, *positions, *slots, *rows;  // [max_rows], each may be nullptr
};
hipError_t launch_blocks_extend(const BlocksArgs &args, hipStream_t stream);
hipError_t launch_blocks_release(const BlocksArgs &args, hipStream_t stream);

// ---- acceptance of a token tree (spec_tree.hip) ---------------------------------
constexpr int kTreeStateBytes = 64;
struct TreeAcceptArgs {
    int n, vocab;
    const float *scores;     // [B][n + 1][vocab]: logits, or probabilities where uniforms are given
    const int32_t *tokens;   // [B][n]
    const int32_t *parents;  // [B][n]
    const float *uniforms;   // [B][n + 1], or nullptr: greedy
    int32_t *accepted;       // [B]
    int32_t *path;           // [B][n]
    int32_t *next_token;     // [B]
    // filled by the launch
    int chunks;       // of the vocabulary
    int looks;        // at a row that is not in, before a workgroup stops waiting
    void *state;      // [B][n + 2] states of kTreeStateBytes
    uint64_t *words;  // [B][n + 1][chunks]
};
size_t spec_tree_workspace(int B, int n, int vocab);
struct TreeAcceptWay {
    bool rows;  // every row at once, or along the path
    int looks;
};
TreeAcceptWay spec_tree_way(int B, int n, int vocab, bool drawn);
hipError_t launch_spec_accept_tree(TreeAcceptArgs args, int B, TreeAcceptWay way, void *workspace, hipStream_t stream);

// ---- acceptance of drafts (spec.hip) ------------------------------------------
// Sampled acceptance workspace: B * (k + 1) * spec_accept_chunks(vocab) pairs of
// uint64 chunk sums.
hipError_t launch_spec_accept_sample(int B, int k, int vocab, const float *p, const float *q,
                                     const int32_t *drafts, const float *u, int32_t *accepted,
                                     int32_t *next_token, void *workspace, hipStream_t stream);
// greedy acceptance
// Workspace: B * (k + 1) * spec_accept_chunks(vocab) (score, index) pairs.
int spec_accept_chunks(int vocab);
hipError_t launch_spec_accept_greedy(int B, int k, int vocab, const float *logits,
                                     const int32_t *drafts, int32_t *accepted,
                                     int32_t *next_token, void *workspace, hipStream_t stream);

}  // namespace lynx
