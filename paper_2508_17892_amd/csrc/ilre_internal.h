// Internal declarations shared by the translation units of libilre (not part of the C ABI).
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "ilre.h"

namespace ilre {

constexpr int kHeadDim = ILRE_HEAD_DIM;
constexpr int kNumCU = 256;  // MI355X: 256 compute units in 8 XCDs
constexpr int kNumXCD = 8;

// Asynchronous 16-byte-per-lane copy from a buffer resource straight into LDS: lane l of the
// wavefront lands at lds_addr + 16*l; bytes past the resource's num_records read as zero.  Tracked
// by vmcnt.  Issued as inline assembly so that the compiler's conservative alias handling does not
// put a full vmcnt wait in front of every later LDS read.  (s_nop: a copy to LDS has to be one wait state behind a scalar write
// of M0, which the assembler does not insert by itself.)
typedef __attribute__((ext_vector_type(4))) int i32x4;
__device__ __forceinline__ void lds_dma16(i32x4 rsrc, unsigned lds_addr, int voffset)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(lds_addr), "v"(voffset), "s"(rsrc)
                 : "memory", "m0");
}
// The same of lines that nobody reads again, which take no place in L2.
__device__ __forceinline__ void lds_dma16_past(i32x4 rsrc, unsigned lds_addr, int voffset)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen nt lds" ::"s"(lds_addr), "v"(voffset), "s"(rsrc)
                 : "memory", "m0");
}
// The same from an address a lane.
__device__ __forceinline__ void lds_dma16(uint64_t src, unsigned lds_addr)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(lds_addr), "v"(src) : "memory", "m0");
}

// ---------------------------------------------------------------- scoring (Eq. 4 / Eq. 5)

// How one scoring pass is cut into workgroups.  A workgroup owns (kv head g, query block qb,
// token split s): `waves` wavefronts of 32*nb query rows each, streaming its token tiles.
struct ScorePlan {
    int dtype;            // ilre_dtype
    int waves;            // wavefronts per workgroup (4 or 8)
    int nb;               // 32-row query blocks per wavefront
    int rows_per_group;   // G * Lq query rows served by one kv head
    int rows_per_wg;      // waves * nb * 32
    bool mixed;           // two query blocks a kv head, the second with one 32-row block a wavefront
    int nqb;              // query blocks per kv group
    int tile_tokens;      // tokens per LDS tile
    int64_t ntiles;       // ceil(L / tile_tokens)
    int nsplit;           // token splits per (g, qb)
    int64_t tiles_per_split;
    int nunits;           // Hkv * nqb  (partial score vectors of pass 2)
    int grid;             // workgroups launched (a few may be idle padding for the XCD mapping)
    bool merge_in_cols;   // whole path: pass 2 merges the partial row statistics (no launch in between)
    bool balanced;        // pass 2's token ranges are sized by the XCDs' speed in pass 1
    uint64_t table_tag;   // header of a range table made for this plan
    size_t lds_bytes_stats, lds_bytes_cols;
};

// Words a launch sets to zero on the side, for a kernel behind it.
struct ClearWords {
    uint32_t *at;  // 16-byte aligned (n = 0: nothing to clear)
    uint32_t n;    // a multiple of 4
};

struct ScoreArgs {
    const void *q;
    const void *k;
    int64_t L;
    int Lq, Hq, Hkv, G;
    int64_t q_stride_head, q_stride_token, k_stride_head, k_stride_token;  // in elements
    float c;  // scale * log2(e): logits leave the MFMA in raw units and are exponentiated base 2
    int rows_per_group, rows_per_wg, nqb, nsplit;
    int64_t ntiles, tiles_per_split;
    // pass 1 (row statistics): per-split partial maxima (base-2 units) and sums
    float *part_m, *part_z;  // [nsplit][Hq*Lq]
    int force_online;        // 1: follow the running maximum throughout (the always-safe form)
    uint32_t *wg_time;       // [grid] how long each workgroup of pass 1 ran, 10 ns ticks (null: not recorded)
    int32_t *split_table;    // [2 + nsplit + 1] pass 2's token ranges: written behind pass 1, read by pass 2 (null: even ranges)
    uint64_t table_tag;
    // pass 2 (column scores)
    const float *row_max, *row_sumexp;  // [Hq*Lq]
    bool merge;                         // whole path: no row statistics, pass 2 merges the partials itself
    ClearWords clear;                   // what pass 2 sets to zero on the side
    float *partial;                     // [nunits][L]
    float *dump;                        // 16 floats nobody reads: target of stores that have nothing to store
};

// `roomy`: query blocks may be of unequal size, which can take one partial score vector more a kv head, and workgroups may be
// more (in several rounds, and with few tiles of fp32 states), which takes more partial row statistics.
ScorePlan make_score_plan(int dtype, int64_t L, int Lq, int Hq, int Hkv, bool roomy);

// With a.merge the partials are all that is left behind.
hipError_t launch_row_stats(const ScorePlan &p, const ScoreArgs &a, float *row_max, float *row_sumexp, hipStream_t s);
// reduce = false leaves the per-unit partial score vectors in a.partial for launch_reduce_units (or for the
// selection's first pass, which can do the reduction on its way).
hipError_t launch_col_scores(const ScorePlan &p, const ScoreArgs &a, int score_mode, float *out_scores,
                             hipStream_t s, bool reduce = true);
hipError_t launch_reduce_units(const float *partial, int nunits, int64_t L, int rmax, float *out_scores, hipStream_t s);

// ---------------------------------------------------------------- selection (Algorithm 1)

constexpr int kSelFine = 256;       // elements a wavefront pools at a time ("fine chunk")
constexpr int kAvgBins = 256;       // printed form: histogram bins per combination
constexpr int kSeedBins = 2048;     // window-max form: histogram bins
constexpr int kSelSmall = 2048;     // seeds beyond the wanted ones that are not worth sorting out
constexpr int kCandCap = 10240;     // candidate capacity in tokens (>= ILRE_MAX_BUDGET + kSelSmall)

// Two forms of Algorithm 1 share the selection kernels.  A "combination" j ranks the elements of a
// source array (value descending, element ascending) and offers the tokens of its best elements:
//   kSelWindowMax  stride-1 max pooling: source = the scores, element = token, value = maximum over a
//                  window of radius r_j clipped to the context; candidates are never exhausted.
//   kSelMaxAvg     the algorithm as printed: source = the cells of a strided max pooling (size = stride
//                  = m), value = stride-1 average over n cells (zeros outside), element p stands for
//                  tokens p*m .. p*m+m-1, and only the best K_m = B/m + 1 cells are candidates.
enum SelMode { kSelWindowMax = 0, kSelMaxAvg = 1 };

struct SelectJob {
    int mode;                    // SelMode
    int64_t L;                   // tokens the pooling sees (the context without its sink part)
    int sink;                    // leading tokens that are always allocated (indices are offset by it)
    int budget;
    int n_max, n_avg;            // kSelWindowMax: n_max window sizes, n_avg = 1
    const int32_t *max_kernels;  // host: window sizes w_j, or max-pooling sizes m_i
    const int32_t *avg_kernels;  // host: average-pooling sizes n_j (kSelMaxAvg only)
    int combos() const { return n_max * n_avg; }
};

// Histogram bins of the window-max form: monotone in the key (ordered_bits of a score), fine where the cut is expected,
// coarse on either side.  Bin 0 is what lies below the first range and is not counted.
constexpr int kBinRanges = 5;
struct KeyBins {
    uint32_t start[kBinRanges];  // keys where the ranges start (a range may be empty)
    uint32_t shift[kBinRanges];  // keys a bin spans, as a shift
    uint32_t pad[2];
};

// Device state of one seed search (window-max form); all zero when its first pass starts.
struct SeedState {
    KeyBins bins;         // left by seed_init where the scores' scale is not known to the host
    uint64_t lists_n;     // keys above the cut bin, collected in `cand` (low half), keys in it, collected in `tie` (high half)
    uint32_t cut;         // bin that holds the K-th largest key
    uint32_t refined;     // not 0: the seeds are the first `refined` of `cand`, else both lists
    uint32_t active_n;    // pre-pass: fine chunks left
    uint32_t done[2];     // workgroups finished: counting, collecting
    uint32_t pad[45];
    uint32_t hist[kSeedBins];
};
static_assert(sizeof(SeedState) % 16 == 0 && sizeof(KeyBins) % 16 == 0 && offsetof(SeedState, hist) % 16 == 0, "cleared in 16-byte words");

struct SelectLayout {
    size_t state;     // kSelWindowMax: SeedState [2]  (the seeds, the pruning pre-pass)
    size_t hist;      // kSelMaxAvg: uint32 [n][kAvgBins]
    size_t ctrl;      // kSelMaxAvg: SelCtrl [n]
    size_t done;      // kSelMaxAvg: uint32 [n]: workgroups finished per max kernel and group of average kernels
    size_t cmax;      // kSelWindowMax: float [ceil(L / kSelFine)]: fine-chunk maxima (pruning pre-pass)
    size_t active;    // kSelWindowMax: uint32 [ceil(L / kSelFine)]: fine chunks left after pruning
    size_t cells;     // float: the max-pooled cell arrays, one per max kernel (kSelMaxAvg)
    size_t picked;    // uint32 [ILRE_MAX_BUDGET] the allocated tokens in the order they were taken, then their count
    size_t seed;      // kSelWindowMax, by rank: uint32 token[kCandCap], uint32 distances to the outranking neighbours[kCandCap]
    size_t cand;      // uint64 [n][kCandCap], one list per combination (kSelWindowMax: one, the seeds)
    size_t tie;       // uint64: per combination two ping-pong lists of boundary elements, each as long as its source
    size_t total;
};

// Printed form: one combination's state.
struct SelCtrl {
    uint32_t want;        // K_j: ranked elements that are candidates
    uint32_t tie_n;       // elements collected
    uint32_t len;         // elements in the source array
    float edge;           // window sums below it are not counted: the bins start here
    uint32_t span[2];     // keys (of float bits) from there on that the first range of bins covers, the first two cover
    uint32_t shifts;      // keys a bin of the three ranges spans, as shifts, a byte each
    uint32_t cut;         // 1 + the lowest bin of which elements are collected (0: all elements)
    uint64_t tie_off;     // lists of elements: uint64 words from the base of the tie region
};

// Workspace carving for a job (only mode, L, counts and the max kernels are read).
SelectLayout make_select_layout(const SelectJob &job);

// Scores that still lie as per-unit partial vectors (the whole path): the selection reduces them into
// `scores` (all L positions, sink part included) itself, in its first pass where it can.
struct FusedScores {
    const float *partial;  // [nunits][L]
    int nunits;
    int rmax;              // 0 sum, 1 max over the units
    float *scores;         // L floats
    int64_t L;
    float mean;            // the scores' scale (window-max form): their mean (sum over the rows) or a lower bound of it (max)
};

// The words of a workspace's selection region (at `base`) that have to be zero before a window-max selection with
// FusedScores starts.
ClearWords select_clear_words(const SelectJob &job, const SelectLayout &lay, void *base);

// `scores` points at the body (the first token after the sink part).
hipError_t launch_select(const float *scores, const SelectJob &job, int32_t *out_idx, int32_t *out_count,
                         void *workspace, const SelectLayout &lay, hipStream_t s, const FusedScores *fused = nullptr);

hipError_t launch_gather_ids(const int32_t *ids, int64_t L, const int32_t *idx, int n, int32_t *out, hipStream_t s);

// ---------------------------------------------------------------- DCA re-RoPE of the key cache

struct RopeArgs {
    const unsigned char *in;
    unsigned char *out;
    int64_t L;
    int Hkv;
    int64_t stride_head, stride_token;  // in elements, the same for in and out
    int chunk, first_extra, nchunks;
    double inv_freq[ILRE_HEAD_DIM / 2];
};

hipError_t launch_rerope(const RopeArgs &a, int dtype, int pairing, hipStream_t s);

// ---------------------------------------------------------------- rotary positions, fill of a paged cache

struct TurnArgs {
    const unsigned char *q, *k, *v;  // [T, heads, d]; each may be null
    unsigned char *q_out;
    int64_t q_token, q_head, out_token, out_head, k_token, k_head, v_token, v_head;  // bytes
    const int32_t *positions;        // null: first_position + token, or the place in the cache
    int T, Hq, Hkv, rotary, first_position;
    float magnitude;
    // the cache
    unsigned char *k_pages, *v_pages;
    int64_t page_bytes, head_bytes, token_bytes;
    const int32_t *table, *kv_len, *cu_q;
    int64_t table_stride, kv_limit;
    int n_seq, num_pages, page_shift;
    double turns[ILRE_HEAD_DIM / 2];  // of pair j, a position
};

hipError_t launch_turn(const TurnArgs &a, int dtype, int pairing, hipStream_t s);

// ---------------------------------------------------------------- norms, rotary positions on axes, fill of a quantised cache; reading a cache back

constexpr int kPlain = 0;  // beside ILRE_KV_FP8, ILRE_KV_FP4: a cache of the states' element type

struct FillArgs {
    const unsigned char *q, *k, *v;  // [T, heads, d]; each may be null
    unsigned char *q_out;
    int64_t q_token, q_head, out_token, out_head, k_token, k_head, v_token, v_head;  // bytes
    const unsigned char *q_weight, *k_weight;  // null: weight + offset is one
    int q_norm, k_norm;
    float offset;
    double eps;
    const int32_t *positions;        // [n_axes, T]; null: first_position + token, or the place in the cache
    int T, Hq, Hkv, rotary, first_position;  // rotary 0: nothing is turned
    double magnitude;
    // the cache
    unsigned char *k_pages, *v_pages, *k_scales, *v_scales;
    int64_t page, head, token;       // strides in channels
    const int32_t *table, *kv_len, *cu_q;
    int64_t table_stride, kv_limit;
    int n_seq, num_pages, page_shift;
    double turns[ILRE_HEAD_DIM / 2], turns_rest[ILRE_HEAD_DIM / 2];  // of pair j, a position; what fp64 left out of them
    uint8_t axes[ILRE_HEAD_DIM / 2];
};

// How many wavefronts share a token's heads.
inline int fill_wavefronts(int T) { return T <= 512 ? 8 : T < 4096 ? 4 : 1; }
hipError_t launch_fill(const FillArgs &a, int dtype, int format, int pairing, hipStream_t s);

struct ReadArgs {
    unsigned char *k_out, *v_out;    // [T, Hkv, d]; each may be null
    int64_t k_token, k_head, v_token, v_head;  // bytes
    const int32_t *tokens;           // null: a sequence's last tokens
    int T, Hkv;
    const unsigned char *k_pages, *v_pages, *k_scales, *v_scales;
    int64_t page, head, token;       // strides in channels
    const int32_t *table, *kv_len, *cu_q;
    int64_t table_stride, kv_limit;
    int n_seq, num_pages, page_shift;
};

// How many rows (token, head) a lane has.
inline int read_rows(int64_t rows) { return rows <= 1 << 18 ? 1 : 4; }
hipError_t launch_read(const ReadArgs &a, int dtype, int format, hipStream_t s);

// ---------------------------------------------------------------- attention over a paged cache or packed keys and values

struct AttnArgs {
    const unsigned char *q, *k, *v;
    unsigned char *out;
    float *lse;
    int64_t q_token, q_head, out_token, out_head, k_page, k_head, k_token, v_page, v_head, v_token;  // bytes
    const int32_t *table, *kv_len;  // null: contiguous keys and values, cut up by cu_k
    const int32_t *cu_q, *cu_k;
    int64_t table_stride, kv_limit;
    int table_width, page_shift, num_pages;
    int T, Tk, n_seq, Hq, Hkv, G;
    int causal, sink, window;
    float c;  // scale * log2(e)
    // the plan
    int nsplit, split_tiles, nblocks, rows, tile;
    float *part_o, *part_e;  // [nsplit][T * Hq][d], [nsplit][T * Hq]
    // a quantised cache: k and v are its codes, and a code's scale lies at its offset in channels / ILRE_KV_BLOCK
    const unsigned char *k_scales, *v_scales;
    // a tree of drafted tokens: which of its sequence's new tokens each one sees, as bits of words
    const uint32_t *tree;
    int64_t tree_stride;
    int tree_words;
};

// How a call is cut up: blocks of `rows` query rows a kv head (16: attend_codes16, 32: attend_tokens or attend_codes, otherwise attend_rows), tiles of `tile` tokens, up to nsplit ranges of
// split_tiles tiles a block.
struct AttnPlan {
    int dtype, rows, tile, nblocks, nsplit, split_tiles;
    bool one_block;  // of rows a sequence, as promised
    int heads;       // kv heads a workgroup
    bool many_tiles; // eight and more for each of two workgroups a compute unit
    size_t bytes;  // of workspace
};

// Most workgroups of a launch (a dimension counts threads in 32 bits, and no workgroup here has more than 512).
constexpr int64_t kMaxUnits = (int64_t)1 << 22;

AttnPlan make_attn_plan(int dtype, int format, bool tree, int T, int n_seq, int Hq, int Hkv, int max_q, int max_kv, int64_t total_kv, int sink, int window, size_t workspace,
                        bool beside = false);  // beside: a token's kv heads follow each other in memory
// The same for a cache of the states' own type and no tree.
inline AttnPlan make_attn_plan(int dtype, int T, int n_seq, int Hq, int Hkv, int max_q, int max_kv, int64_t total_kv, int sink, int window, size_t workspace)
{
    return make_attn_plan(dtype, kPlain, false, T, n_seq, Hq, Hkv, max_q, max_kv, total_kv, sink, window, workspace);
}
hipError_t launch_attention(const AttnPlan &p, AttnArgs a, int format, void *workspace, hipStream_t s);
// The kernels by kind of call; `a` has its plan already.
hipError_t launch_attention_fp8(const AttnPlan &p, const AttnArgs &a, hipStream_t s);
hipError_t launch_attention_fp4(const AttnPlan &p, const AttnArgs &a, hipStream_t s);
hipError_t launch_attention_tree(const AttnPlan &p, const AttnArgs &a, hipStream_t s);
hipError_t launch_attention_tree_fp8(const AttnPlan &p, const AttnArgs &a, hipStream_t s);
hipError_t launch_attention_tree_fp4(const AttnPlan &p, const AttnArgs &a, hipStream_t s);

// ---------------------------------------------------------------- of api.hip, for the other entry points

int fail(int status, const char *fmt, ...) __attribute__((format(printf, 2, 3)));
int hip_fail(hipError_t e, const char *what);
int check_opts(const ilre_opts *o);

// ---------------------------------------------------------------- measurement aid: MFMA ceiling probes

int probe_variants();
const char *probe_describe(int variant);
hipError_t launch_probe(int variant, int iters, const void *operands, float *out, unsigned long long *clocks, double *flops,
                        hipStream_t s);

}  // namespace ilre
