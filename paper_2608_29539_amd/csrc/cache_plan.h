// cache_plan.h -- how the cache operators cut their work, and the workspaces
// that this needs.  Host code apart from the entry points so that a test can
// compile it without a GPU.
//
// The number of chunks is what a plan chooses, and partial results of every
// chunk are what a workspace holds, so a smaller call can want more of it than
// a larger one (shorter chunks while there are few workgroups).  The plans take
// the room at hand: they make fewer chunks where theirs do not fit, down to one
// per range, which needs no more than any call of longer caches or more rows
// was given.
#pragma once

#include <algorithm>
#include <cstddef>
#include <cstdint>

#include "../../include/logo.h"

namespace logo {

constexpr int kPrefixRows = 128;            // (sequence, head) rows per workgroup
constexpr int kMaxPrefixChunks = 128;       // per kind of key range
constexpr int kLseRows = 128;               // flattened (rank, head) rows per workgroup
constexpr int kStepKeys = 1024;             // keys per workgroup of the weights' pass
constexpr int kEvPartRows = 8192;           // rows of an eviction's workgroup
constexpr int kPlanXcds = 8;
constexpr int kPlanKeys = 64;               // chunks are multiples of it
constexpr size_t kPlanAlign = 256;

inline size_t plan_align(size_t x) { return (x + kPlanAlign - 1) & ~(kPlanAlign - 1); }

// The most chunks of `unit` bytes each that fit into `room` bytes, at least 1.
inline long long plan_fit(long long chunks, size_t unit, size_t room) {
    const size_t fit = (room & ~(kPlanAlign - 1)) / std::max<size_t>(unit, 1);
    return std::max(1LL, fit < (size_t)chunks ? (long long)fit : chunks);
}

// The key length of a chunk where n keys are cut into `chunks` (or fewer).
inline long long plan_chunk(long long n, long long chunks, long long most) {
    const long long kc = (n + chunks - 1) / chunks;
    return std::min((kc + kPlanKeys - 1) / kPlanKeys * kPlanKeys, most);
}

struct PrefixPlan {
    int pfx_tiles, own_tiles;
    int kc[4], chunks[4], slot0[4], slots;
    long long first[5];
    size_t ml, total;
};

// Keys per chunk.  The prefix's part of the global branch: about 320
// workgroups over the KV heads and row tiles (one per CU and some, the other
// ranges' beside them), at least 256 keys each: 32 sequences behind 16K tokens
// 45.9 us (with 256, 384 and 512 workgroups 46.6, 47.2, 51.3), 64 behind 32K 88.7
// (87.1, 85.1, 86.6), three groups behind 17.6K in all 23.0 (23.9, 23.1, 23.2; 384
// of at least 128 keys 25.6 where 256 were 21.9).
// The sequences' own rows: 512 keys, 256 where that makes fewer than 512
// workgroups (23 sequences, 2 KV heads: 32 and 24 us; 32 and 8: 38 and 39).
// The window's part of a prefix: 256.  At most kMaxPrefixChunks each; fewer
// where the partial results do not fit into `room` bytes, the kinds with the
// most first.
inline PrefixPlan prefix_plan(const logo_problem *p, const logo_prefix *x, bool share,
                              size_t room) {
    PrefixPlan d;
    const long long G = p->num_q_heads / p->num_kv_heads, w = p->window;
    const long long maxP = x->max_prefix, maxS = p->max_seqlen;
    d.pfx_tiles = (int)(((long long)x->max_group * G + kPrefixRows - 1) / kPrefixRows);
    d.own_tiles = (int)((G + kPrefixRows - 1) / kPrefixRows);
    const long long span[4] = {maxP, share ? (maxS > w ? maxS - w : 0) : maxS,
                               maxP < w ? maxP : w, maxS < w ? maxS : w};
    const long long work = (long long)x->total_tokens * p->num_kv_heads * d.pfx_tiles;
    const long long own_items = p->num_seqs * (long long)p->num_kv_heads * d.own_tiles *
                                ((maxS + 511) / 512);
    const long long own = own_items >= 512 ? 512 : 256;
    const long long want[4] = {std::max(256LL, (work + 319) / 320), own, 256, own};
    const long long most = 1LL << 26;       // (a position and a chunk behind it stay 32-bit)
    long long slots = 0;
    for (int i = 0; i < 4; i++) {
        const long long kc = std::max(want[i], (span[i] + kMaxPrefixChunks - 1) / kMaxPrefixChunks);
        d.kc[i] = (int)plan_chunk(kc, 1, most);
        d.chunks[i] = (int)((span[i] + d.kc[i] - 1) / d.kc[i]);
        slots += d.chunks[i];
    }
    const size_t rows = (size_t)p->num_seqs * p->num_q_heads;
    auto size = [&]() {
        d.ml = plan_align(sizeof(float) * rows * slots * p->head_dim);
        return d.ml + plan_align(sizeof(float) * 2 * rows * slots);
    };
    while ((d.total = size()) > room) {
        int i = -1;
        for (int j = 0; j < 4; j++)
            if (d.kc[j] < most && d.chunks[j] > (i < 0 ? 1 : d.chunks[i]))
                i = j;
        if (i < 0)
            break;
        slots -= d.chunks[i];
        d.kc[i] = (int)plan_chunk(span[i], d.chunks[i] - 1, most);
        d.chunks[i] = (int)((span[i] + d.kc[i] - 1) / d.kc[i]);
        slots += d.chunks[i];
    }
    long long first = 0;
    slots = 0;
    for (int i = 0; i < 4; i++) {
        d.slot0[i] = (int)slots;
        slots += d.chunks[i];
        const bool is_own = i & 1;
        const long long pairs = (long long)(is_own ? p->num_seqs : x->num_prefixes) * d.chunks[i] *
                                p->num_kv_heads;
        d.first[i] = first;
        first += (pairs + kPlanXcds - 1) / kPlanXcds * kPlanXcds *
                 (is_own ? d.own_tiles : d.pfx_tiles);
    }
    d.first[4] = first;
    d.slots = (int)slots;
    return d;
}

struct ScorePlan {
    int key_waves, lse_kc, lse_chunks, per_seq, lse_per_seq;
    long long items, lse_items;
    size_t total;
};

// Blocks of `block` over sequences of at most `longest` with `total` in all:
// the same number for every sequence where that is at most twice the sum of
// their own (a workgroup then finds its sequence by a division), else what
// bounds the sum.
inline long long score_blocks(long long total, long long longest, long long B, long long block,
                              int &per_seq) {
    const long long bound = total / block + B, each = (longest + block - 1) / block;
    per_seq = each * B <= 2 * bound ? (int)each : 0;
    return per_seq > 0 ? each * B : bound;
}

// Keys per workgroup (64, 128 or 256): the most that still makes 256
// workgroups, one per CU.  More keys share the staged rows; fewer make up for
// a small problem: 64 rows on 13324 keys, 8 KV heads, 21.8 us with 256 keys,
// 29.5 with 128, 47.8 with 64; 256 rows on 1024 keys, 2 KV heads, d = 64, 29.3,
// 20.4 and 14.7.  Key chunks of the log-sum-exp: about 1024 workgroups, of at
// least 512 keys; fewer where their sums do not fit into `room` bytes.
inline ScorePlan score_plan(const logo_problem *p, int32_t cap, size_t room) {
    ScorePlan d;
    const long long N = p->total_tokens, B = p->num_seqs, H = p->num_kv_heads;
    const long long G = p->num_q_heads / p->num_kv_heads;
    d.key_waves = N * H >= 256 * 256 ? 4 : N * H >= 256 * 128 ? 2 : 1;
    const long long maxL = std::max(1, p->max_seqlen);
    d.items = score_blocks(N, maxL, B, 64 * d.key_waves, d.per_seq) * H;
    // (one sequence may have all the rows, and a row may be listed twice)
    const long long tiles = score_blocks(cap * G, cap * G, B, kLseRows, d.lse_per_seq);
    const long long full = ((long long)cap * G / kLseRows + B) * H;   // without the empty places
    const size_t unit = 2 * sizeof(float) * (size_t)cap * p->num_q_heads;
    const long long chunks = plan_fit(
        std::min({(1024 + full - 1) / full, (maxL + 511) / 512, 64LL}), unit, room);
    d.lse_kc = (int)plan_chunk(maxL, chunks, (1LL << 31) - 64);
    d.lse_chunks = (int)((maxL + d.lse_kc - 1) / d.lse_kc);
    d.lse_items = tiles * H * d.lse_chunks;
    d.total = plan_align(unit * d.lse_chunks);
    return d;
}

// Keys per chunk of the scores' pass: 1024, down to 256 while there are fewer
// than 512 workgroups (two per CU).  16 caches of 32K tokens, 8 KV heads: 256
// keys 254 us, 512 and 1024 220, 2048 229, 4096 258.  More where the chunks'
// sums do not fit into `room` bytes behind the scores.
struct StepScorePlan {
    int kc, chunks, out_chunks, head_copies, head_blocks;
    long long items, out_items;
    size_t ml, total;
};
inline StepScorePlan step_score_plan(const logo_problem *p, size_t room) {
    StepScorePlan d;
    const long long maxL = std::max(1, p->max_seqlen), B = p->num_seqs, H = p->num_kv_heads;
    const long long G = p->num_q_heads / p->num_kv_heads;
    d.head_copies = G <= 4 ? 4 : G <= 8 ? 2 : 1;
    d.head_blocks = (int)((G + 15) / 16);
    d.kc = 1024;
    while (d.kc > 256 && B * H * d.head_blocks * ((maxL + d.kc - 1) / d.kc) < 512)
        d.kc /= 2;
    // (one float behind the scores that nothing reads)
    d.ml = plan_align(sizeof(float) * ((size_t)p->num_q_heads * p->total_tokens + 1));
    const size_t unit = 2 * sizeof(float) * (size_t)B * p->num_q_heads;
    const long long chunks = (maxL + d.kc - 1) / d.kc;
    const long long fit = plan_fit(chunks, unit, room > d.ml ? room - d.ml : 0);
    if (fit < chunks)
        d.kc = (int)plan_chunk(maxL, fit, 1LL << 30);
    d.chunks = (int)((maxL + d.kc - 1) / d.kc);
    d.out_chunks = (int)((maxL + kStepKeys - 1) / kStepKeys);
    d.items = B * H * d.head_blocks * d.chunks;
    d.out_items = B * H * d.out_chunks;
    d.total = d.ml + plan_align(unit * d.chunks);
    return d;
}

struct EvictPlan {
    long long parts, items;
    size_t picks, above, total;
};
inline EvictPlan evict_plan(const logo_problem *p) {
    EvictPlan d;
    const size_t problems = (size_t)p->num_seqs * p->num_kv_heads;
    d.parts = std::max(1LL, ((long long)p->max_seqlen + kEvPartRows - 1) / kEvPartRows);
    d.items = (long long)problems * d.parts;
    d.picks = d.above = d.total = 0;
    if (d.parts > 1) {
        d.picks = plan_align(sizeof(uint32_t) * 2 * 1024 * problems * d.parts);
        d.above = d.picks + plan_align(sizeof(uint32_t) * 4 * problems);
        d.total = d.above + plan_align(sizeof(uint32_t) * problems * d.parts);
    }
    return d;
}

}  // namespace logo
