// cache_internal.h -- arguments and launchers of the operators of shared and
// scored caches, shared by the host entry points (logo_api.cpp) and their
// kernels.  Not installed.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "cache_plan.h"

namespace logo {

// One decoding step of sequences that share prefixes (decode_prefix.hip).
// Kinds of work item, in this order: the prefix's part of the global branch,
// the sequence's own part of it, the prefix's part of the local branch, the
// own part.  Partial results: (O [D], then m, l apart) per slot, sequence and
// head, where chunk c of kind i has slot slot0[i] + c.
constexpr int kPrefixThreads = 256;
constexpr int kWidePrefixMerge = 16;        // chunks above which a head's merge takes four waves
struct PrefixArgs {
    const uint16_t *q, *k, *v, *kp, *vp;           // local branch: [B][Hq][d], own rows, prefixes
    const uint16_t *q_g, *k_g, *v_g, *kp_g, *vp_g; // global branch
    const int32_t *cu, *cu_pre, *cu_grp;
    const float *gate, *gain_local, *gain_global;
    float eps, scale_log2;
    int32_t num_seqs, num_prefixes, hq, hkv, group, head_dim, window;
    int32_t share;                           // the branches' tensors are the same
    int32_t pfx_tiles, own_tiles;            // row tiles of a group / of one sequence
    int32_t kc[4], chunks[4], slot0[4];
    int32_t first[5];                        // first work item of each kind
    int32_t *act, *n_act;                    // selected sequences (compacted), count; or NULL
    int32_t sel_mode;                        // 0: threshold thr_host, 2: device threshold thr_dev[0]
    float thr_host;
    const float *thr_dev;
    float *part, *ml;
    uint16_t *out;
};
hipError_t launch_decode_prefix(const PrefixArgs &a, hipStream_t s);

// Attention weight received by every key (cache_score.hip).
constexpr int kScoreThreads = 256;
struct ScoreArgs {
    const uint16_t *q, *k;
    const int32_t *cu, *sel_idx, *cu_sel;    // cu_sel NULL: every token is a row
    const float *lse;                        // [Hq][cap], or NULL:
    float *lse_part;                         // (m, l) [lse_chunks][Hq][cap], to be computed
    const float *score_in;                   // [Hkv][n] or NULL (zeros)
    float *score;
    int64_t n;                               // tokens
    int32_t cap, num_seqs, hq, hkv, group, head_dim;
    float scale_log2;
    int32_t key_waves, items;                // waves side by side over the keys; workgroups
    int32_t lse_kc, lse_chunks, lse_items;
    int32_t per_seq, lse_per_seq;            // key blocks / row tiles of every sequence, 0: search
};
hipError_t launch_cache_score(const ScoreArgs &a, hipStream_t s);

constexpr int kStepThreads = 128;           // of the scores' pass; the weights' kScoreThreads
struct StepScoreArgs {
    const uint16_t *q, *k;
    const int32_t *cu;
    const float *gate;
    const float *score_in;                   // [Hkv][n] or NULL (zeros)
    float *score, *logits, *ml;              // logits [Hq][n]; ml [B][Hq][chunks][2]
    int64_t n;
    int32_t num_seqs, hq, hkv, group, head_dim;
    int32_t head_copies, head_blocks;        // 16 rows hold 16 / head_copies heads, head_copies times
    float scale_log2;
    int32_t kc, chunks, items, out_chunks, out_items;
    int32_t sel_mode;                        // as PrefixArgs
    float thr_host;
    const float *thr_dev;
};
hipError_t launch_decode_score(const StepScoreArgs &a, hipStream_t s);

// Eviction (cache_evict.hip): in / out hold up to four caches (NULL: none).
struct EvictArgs {
    const float *score;                      // [Hkv][n]
    const int32_t *cu;
    int64_t n;
    int32_t num_seqs, hkv, head_dim, budget, recent, cap;
    int32_t rows;                            // of the outputs, at most (cap may be larger)
    const uint16_t *in[4];
    uint16_t *out[4];
    float *score_out;                        // [Hkv][cap]
    int32_t *keep_idx, *cu_keep;             // [Hkv][cap], [B + 1]
    // caches of more than kEvPartRows rows, in `parts` parts: two digits'
    // histograms [2][B Hkv][parts][1024], two picks [2][B Hkv][2], rows above
    // them [B Hkv][parts]
    int32_t parts;
    int32_t small;                           // no cache of more than kEvSmallRows
    uint32_t *hist, *picks, *above;
};
constexpr int kEvThreads = 1024;            // of a part of kEvPartRows
constexpr int kEvSmallRows = 2048;
constexpr int kEvSmallThreads = kEvSmallRows / (kEvPartRows / kEvThreads);
hipError_t launch_cache_evict(const EvictArgs &a, hipStream_t s);

}  // namespace logo
