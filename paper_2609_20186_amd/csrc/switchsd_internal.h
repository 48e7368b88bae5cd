// switchsd_internal.h -- parameters shared by the host API and the kernels.
// Not part of the public interface (see include/switchsd.h).
#pragma once

#include <stdint.h>

#include "switchsd.h"

namespace switchsd {

// Work-group shape of every kernel of the step: 256 lanes = 4 wave64s.
constexpr int kThreads = 256;
// 16-byte logits vectors per lane in one chunk of the argmax stream.
constexpr int kUnroll = 4;
// 16-byte vectors in one chunk (16 KB); two chunks are in flight per work-group.
constexpr int kChunkVecs = kThreads * kUnroll;
// Context end positions covered by one scan work-group.
constexpr int kScanTile = 1024;
// Weight sums per 16 KB chunk of the draw at T > 0: one per wave (each wave
// reads 256 contiguous vectors of the chunk).
constexpr int kCsumPerChunk = kThreads / 64;
// Per-sequence workspace slots live on their own 256-byte lines: atomics to
// one line serialize, and every work-group of a sequence arrives at its line.
constexpr int kLineU32 = 64;
constexpr int kLineU64 = 32;
// Copy candidates per sequence, at most.
constexpr int kMaxCand = SWITCHSD_MAX_CAND;
// Argmax segments per logits row, at most (the fused step's per-segment
// result slots hold R * kMaxSegs keys per sequence).
constexpr int kMaxSegs = 16;
// Workspace slots one poll of wave 0 covers, at most (8 per lane).
constexpr int kMaxPollSlots = 512;
// Scan tiles per sequence, at most, for which the last tile polls per-tile
// match slots instead of an arrival (the other tiles' 8 slots each).
constexpr int kMaxPollTiles = kMaxPollSlots / 8;

enum : int32_t { EPI_NONE = 0, EPI_MATCH = 1, EPI_SELECT = 2 };
enum : int32_t {
    ROWS_ALL = 0,
    ROWS_NEURAL_OR_COPY = 1,
    ROWS_DRAFT = 2,
    ROWS_LISTED = 3,
    ROWS_Q = 4  // the draft's rows r < dn - 1 of sequences verified with q
};
// Sequences a work-list verify launch handles (its item prefix sums live in
// four registers per lane).
constexpr int kListMaxB = 256;

// The draw at T > 0 with whole rows in registers (a 1024-thread work-group per
// row and compute unit): 16-byte vectors per lane, at most.
constexpr int kRowVecs = 20;
// Rows of up to this many vectors per lane are taken by work-groups of half the
// size with twice the vectors, two per compute unit.
constexpr int kRowVecsTwo = 4;

struct Workspace {
    uint32_t *tk_front;        // [B] x 256 B: arrivals of the scan/probe work-groups
    uint32_t *tk_all;          // [B] x 256 B: arrivals of every work-group of a sequence
    int32_t *mslot;            // [B] x 256 B: most recent end + 1 per n-gram length
    unsigned long long *keys;  // [B] x key_stride: packed (value key, ~index) row maxima
    int32_t key_stride;        // u64 per sequence (R rounded up to a 256-byte line)
    uint32_t *rtk;             // [B] x rtk_stride: arrivals of the sum work-groups per row
                               // (draw at T > 0)
    int32_t rtk_stride;        // u32 per sequence (R rounded up to a 256-byte line)
    int32_t *cand;             // [B] x cand_stride: per scan tile and n-gram length, the
                               // tile's W most recent ends + 1 (0: none); W > 1 and
                               // more than one tile only
    int32_t cand_stride;       // int32 per sequence (whole 256-byte lines)
    unsigned long long *qkeys; // [B] x key_stride: row maxima of the draft's distribution q
                               // (between keys and rtk)
    unsigned long long *skeys; // [B] x skey_stride: the fused step's per-segment row maxima,
                               // segment s of row r at s * R + r (0: not yet written,
                               // 1: the segment has no candidate); between rtk and cand
    int32_t skey_stride;       // u64 per sequence (R * kMaxSegs on whole lines; 0 if R > 64)
    int32_t *tslot;            // [B] x tslot_stride: per scan tile t and n-gram length j at
                               // t * 8 + j, the tile's most recent end + 2 (1: none, 0: not
                               // yet written); between skeys and cand
    int32_t tslot_stride;      // int32 per sequence (tiles * 8 on whole lines; 0 unless
                               // 1 < tiles <= kMaxPollTiles)
};

struct StepParams {
    // inputs
    const int32_t *tokens;
    const int32_t *lengths;
    const uint16_t *hidden;
    const float *w;
    const int32_t *ntok;
    const int32_t *npar;
    const int32_t *nn;
    const uint16_t *logits;
    const int32_t *copy_tokens_in;  // select stage only
    const int32_t *match_n_in;      // select stage only
    const int32_t *copy_len_in;     // select stage only
    const float *z_in;              // select stage only
    int32_t B, Lmax, d, R, V;
    float bias;
    // configuration
    int32_t n_ngram;
    int32_t lens[SWITCHSD_MAX_NGRAM];
    int32_t nmax;
    int32_t kappa;
    int32_t k;
    float theta;
    int32_t W;  // copy candidates (>= 1)
    // outputs
    int32_t *match_n, *match_end, *copy_len, *copy_tokens;
    float *z;
    int32_t *use_copy, *dtok, *dpar, *dn;
    int32_t *amax;
    int32_t *accept_len, *accept_node, *bonus, *out_tokens;
    Workspace ws;
    // grid layout: [probe][scan tiles][argmax row segments, segment-major]
    int32_t scan_tiles;  // per sequence (0: no scan role)
    int32_t probe_on;    // 1: one probe work-group per sequence, first in the grid
    int32_t scan_probe;  // 1: scan tile 0 of each sequence also computes the probe
    int32_t segs;        // argmax work-groups per row (0: no argmax role)
    int32_t seg_elems;   // logits elements per row segment (multiple of 8)
    int32_t n_scan_wg;   // B * scan_tiles
    int32_t n_front_wg;  // n_scan_wg + B * probe_on
    int32_t rows_mode;
    int32_t speculate;   // 1: issue a row's first chunk before reading whether it is needed
    int32_t epi_front;
    int32_t epi_accept;
    int32_t poll_accept; // 1 (R <= 64, T = 0): each argmax work-group stores its result in
                         // its own slot, and the work-group holding the sequence's draft
                         // (the front's chooser in the fused step, a poller work-group
                         // in the verify launch) polls the slots and runs the accept
                         // epilogue (no arrivals at tk_all)
    int32_t n_poll_wg;   // verify launch with poll_accept: one waiting work-group per
                         // sequence, first in the grid, runs its accept epilogue
    int32_t poll_front;  // 1 (the step, 1 < scan_tiles <= kMaxPollTiles): each scan tile
                         // stores its match slots in its own line (with several candidates
                         // after its completed candidate lists) and the last tile polls
                         // them (no arrivals at tk_front)
    int32_t list_mode;   // 1: verify only, a fixed grid streaming the chunks of the drafted
                         // rows r < dn[b] (segs = chunks per row)
    // decode loop: the accept epilogue appends to the context (read-write)
    int32_t commit;
    int32_t *ctok;       // [B, Lmax] the context, written at positions >= its length
    int32_t *clen;       // [B] its length
    int32_t *draft_pos;  // [B] draft-model cache position (in/out)
    int32_t *lag;        // [B] tokens the next neural drafting pass must consume first
    // draws at T > 0 (the weight-sum launch)
    const uint64_t *uniforms;  // [B, R]
    float samp_c;              // log2(e) / T
    unsigned long long *csum;  // [B, R, cpr, waves] integer weight sums per chunk and wave
    int32_t cpr;               // 16 KB chunks per row
    int32_t seg_chunks;        // chunks per work-group of the sum launch
    int32_t draw_poll;         // 1: the polled draw (no q, R <= 64): sums stored + 1, the
                               // work-group of each row's first segment draws the row's token
                               // and row 0's runs the accept epilogue (no arrivals)
    int32_t csum_clear;        // the row maxima launch before a polled draw: each argmax
                               // work-group zeroes its share of its row's sum slots
    int32_t qmax;              // 1: the row maxima launch also takes the draft's q rows, its
                               // last B * R * segs work-groups (q keys); else a launch of
                               // their own follows
    // speculative sampling with the draft's own distribution q (chains, T > 0)
    const uint16_t *qlogits;          // [B, R, V] the draft's logits, or null (one-hot drafts)
    const uint64_t *accept_uniforms;  // [B, R] uniforms of the accept tests
    const int32_t *spec_copy;         // [B] use_copy of the step (copy drafts stay one-hot)
                                      // or null (every sequence uses q)
    unsigned long long *qcsum;        // [B, R, cpr, waves] integer weight sums of the q rows
    unsigned long long *rcsum;        // [B, cpr * 16, 4] per block of 64 vectors of the
                                      // rejected row: residual sum (lo, hi), P sum, unused
    uint32_t *rdec;                   // [B, R] test of row r: 1 accepted, 2 rejected
    unsigned long long *rz;           // [B, R, 2] Zp, Zq of each tested row
    int32_t rsegs;                    // residual work-groups per sequence (8 KB each)
    // bounded waits: spin limit of the front's wait for the probe flag and of
    // its poll of the segment slots; with withhold_flag (a test knob) the
    // probe never sets its flag
    int32_t spin_cap;
    int32_t withhold_flag;
    int32_t withhold_seg;  // test knob: sequence 0's row 0 segment 0 (of the argmax, and of the
                           // weight sums in a polled draw) and its scan tile 0 never store
                           // their slots
    unsigned long long *tl;  // timeline build only: per work-group phase stamps
    uint32_t exp_front;  // arrivals per sequence at tk_front
    uint32_t exp_all;    // arrivals per sequence at tk_all
};

// Every check of switchsd_step's arguments except its two workspaces
// (switchsd_step and switchsd_step_noalloc run it before anything else).
int check_step_args(const switchsd_step_args *a);

int launch_step_kernel(const StepParams &p, int64_t grid, hipStream_t stream);
int launch_select_kernel(const StepParams &p, hipStream_t stream);
int launch_commit_kernel(const StepParams &p, hipStream_t stream);
int launch_label_kernels(const StepParams &p, int32_t n, uint8_t *labels, int32_t tsize,
                         void *table, hipStream_t stream);
int launch_sample_sums_kernel(const StepParams &p, int64_t grid, hipStream_t stream);
int launch_row_draw_kernel(const StepParams &p, int64_t grid, hipStream_t stream);
int launch_spec_residual_kernel(const StepParams &p, int64_t grid, hipStream_t stream);
int launch_status_kernel(int32_t *mslot, int32_t B, int32_t *out, hipStream_t stream);
int launch_tree_mask_kernel(const int32_t *dpar, const int32_t *dn, int32_t B, int32_t R,
                            uint32_t *mask, hipStream_t stream);

// ---- calls around the step (switchsd_logits.hip, switchsd_pages.hip)

// Rows a work-group of the logits kernels takes, at most (one wave handles a
// row's result per lane).
constexpr int kRowGroup = 64;
// 16-byte vectors per lane and row of the logits kernels, at most.
constexpr int kLogitsUnroll = 2;
// 16-byte vectors of the blocks that make a chunk: every 2^k-th of a row.
constexpr int kVerifyBlk = 16;
constexpr int kProcessBlk = 32;
// Rows of a work-group of k_verify from which its waves take whole rows.
constexpr int kWholeRows = 16;
// LDS bytes of the path counts of a work-group's rows.
constexpr int kPathBytes = 8192;

// Drafted rows a work-group of the page plan takes, at most (one sequence at
// least), and positions of a range that one of the packed slots takes.
constexpr int kPlanNodes = 1024;
constexpr int kSpanPart = 1024;
static_assert(kPlanNodes >= SWITCHSD_MAX_R, "a plan work-group holds a sequence's rows");

struct LogitsParams {
    switchsd_logits_args a;
    void *out;          // process: the processed logits; verify: null
    int32_t in_place;   // out is logits: only what changes is written
    int32_t penal;      // any of the three penalties
    // grid: [sequence][row group][vocabulary chunk]
    int32_t unroll;     // 16-byte vectors per lane and row
    int32_t chunks;     // vocabulary chunks: a power of two, 2^chunk_log
    int32_t chunk_log;
    int32_t split;      // verify: waves that share a row (1 or 4)
    int32_t rows;       // rows per group (at most kRowGroup)
    int32_t groups;
    // verify
    int32_t *accept_len, *accept_node, *bonus, *out_tokens, *amax;
    unsigned long long *keys;  // [B] x key_stride row maxima (R > 64)
    int32_t key_stride;
    unsigned long long *skeys; // [B] x skey_stride copies of them (R <= 64)
    int32_t skey_stride;
    uint32_t *tickets;         // [B] x kLineU32
};

struct PageParams {
    const int32_t *lengths, *dpar, *dn;
    int32_t B, R, Lmax, page_size, max_pages, ring_pages;
    int32_t *table, *held, *ring, *ring_state;
    int64_t *slots;
    int32_t *positions, *missing;
    int32_t page_log;  // page_size = 2^page_log, or -1
    int32_t seqs;      // sequences per work-group
    uint32_t *ticket;
};

struct SpanParams {
    const int32_t *begin, *end, *tokens, *table, *held;
    int32_t B, Lmax, max_pages, page_size;
    int32_t page_log;  // page_size = 2^page_log, or -1
    int32_t *cu;
    int64_t *slots;
    int32_t *positions, *packed, *seq;
    int32_t capacity;
    int32_t seqs, parts;  // sequences per work-group, parts of a range
};

struct CompactParams {
    void *cache;
    int64_t plane_stride, n_slots;
    int32_t row_vecs;    // pieces per row (16 or 4 bytes each)
    int64_t pieces;      // planes * row_vecs
    const int64_t *slots;
    const int32_t *dpar, *dn, *accept_node;
    int32_t B, R;
    int32_t blocks;      // work-groups per sequence
};

// ---- attention over the paged cache (switchsd_attention.hip)

struct StoreParams {
    const void *k, *v;
    int64_t k_stride, v_stride;  // bytes
    const int64_t *slots;
    const int32_t *count;
    int32_t n, Hkv, D;
    void *k_cache, *v_cache;
    int64_t n_slots;
    const float *k_scale, *v_scale;
};

struct AttnParams {
    switchsd_attention_args a;
    const void *q;
    int64_t q_stride;  // elements
    const void *k_cache, *v_cache;
    int64_t n_slots;
    const float *k_scale, *v_scale;
    void *out;
    float *lse;
    float *part;       // partial results
    int32_t G;         // query heads per head of the cache
    int32_t page_log;  // page_size = 2^page_log, or -1
    int32_t whole;     // no item is cut
    int32_t groups;    // work-groups that share the keys of few items
};

// Work-groups that share an attention's keys where there are few items (tiles of rows
// and heads of the cache): as many as the device holds at once, two on a compute unit
// (half as many where registers allow one).
constexpr int kAttnGroups = 512;
// The fewest units of keys for a work-group.  With 4 one token over 17195 keys takes 23.4
// us (20.7), 17 drafted ones over 8972 28.8 (27.1).
constexpr int kAttnLeast = 2;
// Contexts of up to so many tokens are never cut: the join costs more than it saves.  13
// prompts of 285 tokens (40 + 8 heads of 256) take 85 us so, 147 where 512 is the most; 7 x
// 128 heads over 924 keys 13.6 and 21.7.
constexpr int kAttnShort = 1024;
// Work-groups that join what was cut.  With 2048 13 x 35 rows over 1859 keys take 38.9
// us (36.2), with 4096 48.7.
constexpr int kAttnMerge = 1024;

// Query rows (new tokens times query heads of one head of the cache) of a work-group,
// by the most that a sequence has.  64 rows in the form for few took longer in the most
// cases (20 x 64 over 6221 keys: 116 us, in the form for many 106; 183 x 60 over 99: 29
// and 17).  17 to 32 rows in the form for many take less of long contexts (14 x 30 over
// 8373: 34 us, not 38), more of short ones (7 x 31 over 317: 16.2, not 12.8) and of
// 256-wide heads (54 x 29 over 9117: 408, not 307).
constexpr int attention_tile(int64_t most) { return most <= 32 ? 32 : 128; }
// With so many items each work-group takes a whole one, and nothing has to be joined: more
// with few rows, whose work-groups are bound by the memory and end apart (1048 items of
// 28 rows, 131 sequences of up to 8598 keys: 430 us, whole 574; 3696 of 30 rows over 1219:
// 249, whole 264) than with many (1672 tiles of prompts: 156 us, cut 185; 4096 of trees:
// 608, cut 735).
constexpr uint32_t attention_whole(int64_t tile) { return tile == 32 ? 4096 : 1024; }
// Floats of the partial results: each of kAttnGroups work-groups leaves at most
// two, of as many rows as a work-group takes, D sums, a maximum and a sum each.
constexpr size_t attention_part_floats(int64_t most, int32_t D) {
    return (size_t)2 * kAttnGroups * attention_tile(most) * (D + 2);
}

int launch_store_kernel(const StoreParams &p, int32_t type, int32_t cache_type,
                        hipStream_t stream);
int launch_attention_kernel(const AttnParams &p, int32_t type, int32_t cache_type,
                            hipStream_t stream);

// ---- log probabilities (switchsd_logprobs.hip)

// Along accepted paths a large batch's sequences have few entries of their R:
// work-groups for kLogprobSlots of them, each of which takes every so many-th.  32
// paths of 1 to 9 entries, rows of 128256 16-bit logits: 29.6 us with 16, with 4 and 8
// 41 and 35 (a path's second round waits for its first), with 32 29.6.
constexpr int kLogprobSlots = 16;
inline int32_t logprob_slots(const switchsd_logprob_args &a) {
    return a.accept_node && a.R > kLogprobSlots && (int64_t)a.B * a.R > 512 ? kLogprobSlots : a.R;
}
// Pieces of a row, for about kLogprobGroups work-groups together, which is as many as
// are held at once (145 rows of 27830 16-bit logits: 15.5 us; for 2048 22.5), or for
// twice as many where the most of a path's have no work (those 32 paths: 29.6; for 1024
// 35.0, for 4096 35.3).  A piece is at least two vectors of each lane.
constexpr int kLogprobGroups = 1024, kLogprobPathGroups = 2048;
constexpr int kLogprobPieces = 64;
constexpr size_t kLogprobRecord = 16 + 8 * SWITCHSD_MAX_TOP;
struct LogprobCut {
    int32_t pieces, vecs;
};
inline LogprobCut logprob_cut(const switchsd_logprob_args &a, bool may) {
    const int64_t rows = (int64_t)a.B * logprob_slots(a);
    const int64_t per = a.logits_type == SWITCHSD_F32 ? 4 : 8;
    const int64_t vecs = (a.V + per - 1) / per, least = 2 * kThreads;
    const int64_t most = logprob_slots(a) < a.R ? kLogprobPathGroups : kLogprobGroups;
    int64_t n = may && rows > 0 ? most / rows : 1;
    n = n < vecs / least ? n : vecs / least;
    n = n < kLogprobPieces ? n : kLogprobPieces;
    n = n > 1 ? n : 1;
    const int64_t each = ((vecs + n - 1) / n + kThreads - 1) / kThreads * kThreads;
    return {(int32_t)((vecs + each - 1) / each), (int32_t)each};
}

struct LogprobParams {
    switchsd_logprob_args a;
    float inv_t;  // 1 / temperature
    float *logprob, *lse, *entropy;
    int32_t *rank;
    int32_t n_top;
    int32_t *top_ids;
    float *top_logprobs;
    int32_t slots;      // entries of a sequence that are taken side by side
    int32_t pieces;     // of a row, piece_vecs vectors each
    int32_t piece_vecs;
    uint32_t *tickets;  // [B, R], with the records of a cut row's pieces
    void *records;      // [B, R, pieces]
    // gradient
    const float *in_lse, *in_entropy, *g_logprob, *g_entropy;
    void *grad;
};

int launch_logprob_kernel(const LogprobParams &p, hipStream_t stream);
int launch_logprob_grad_kernel(const LogprobParams &p, hipStream_t stream);

int launch_logits_kernel(const LogitsParams &p, int32_t out_type, hipStream_t stream);
int launch_page_plan_kernel(const PageParams &p, hipStream_t stream);
int launch_span_kernel(const SpanParams &p, hipStream_t stream);
int launch_compact_kernel(const CompactParams &p, bool wide, hipStream_t stream);

}  // namespace switchsd
