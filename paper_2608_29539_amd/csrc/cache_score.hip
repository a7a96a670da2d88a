// cache_score.hip -- the attention weight that every cached key has received
// (logo_cache_score for a prompt's queries, logo_decode_score for one decoding
// step):
//   a[h][j] = a_in[h][j] + sum_i sum_{g < G} 2^(c q_{i, hG+g} . k_{j, h} - lse_{i, hG+g})
// over the query rows i that see key j, lse the base-2 log-sum-exp of the
// row's scaled scores, c = softmax_scale log2(e).  The G heads of a KV head add
// to the same key; every sum is taken in a fixed order, so results do not
// change from run to run.
//
//   score_lse_kernel        (m, l) of the rows by chunks of keys, where the
//                           caller has no lse
//   score_kernel            key-stationary: a wave keeps 64 keys of one KV head
//                           in registers (the MFMA's B operand) and walks over
//                           the rows that see them, so a key's sum stays in
//                           its lane
//   step_logits_kernel      one query per sequence: the scaled scores of a
//                           chunk of keys and their (m, l) per head
//   step_weights_kernel     2^(score - lse) summed over the heads
#include "cache_internal.h"
#include "cache_tiles.h"
#include "decode_common.h"
#include "logo_internal.h"

#include <type_traits>

namespace logo {
namespace {

constexpr int kScoreWaves = kScoreThreads / 64;
constexpr int kLseBuffers = 4;

// Item t of the blocks that sequences have n(b) of each, sequence-major: its
// sequence and block; false past the last.  per_seq > 0: every sequence has
// that many places (of which n(b) are blocks); else every wave searches for
// itself.
template <class F>
__device__ __forceinline__ bool find_block(int t, int B, int per_seq, F &&n, int &b, int &j) {
    const int lane = threadIdx.x & 63;
    if (per_seq > 0) {
        b = t / per_seq;
        j = t % per_seq;
        return b < B && j < n(b);
    }
    int before = 0;
    for (int b0 = 0; b0 < B; b0 += 64) {
        const int c = b0 + lane < B ? n(b0 + lane) : 0;
        int incl = c;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int x = __shfl_up(incl, d, 64);
            if (lane >= d)
                incl += x;
        }
        const int total = __shfl(incl, 63, 64);
        if (t < before + total) {
            const int src = __ffsll((unsigned long long)__ballot(t < before + incl)) - 1;
            b = uni(b0 + src);
            j = uni(t - before - __shfl(incl - c, src, 64));
            return true;
        }
        before += total;
    }
    return false;
}

// The query rows of sequence b: ranks [s0, s1) of sel_idx, or its tokens.
__device__ __forceinline__ void row_span(const ScoreArgs &a, int b, int &s0, int &s1) {
    if (a.cu_sel) {
        s0 = min(a.cu_sel[b], a.cap);
        s1 = min(a.cu_sel[b + 1], a.cap);
    } else {
        s0 = a.cu[b];
        s1 = a.cu[b + 1];
    }
}
__device__ __forceinline__ int token_of(const ScoreArgs &a, int rank) {
    return a.cu_sel ? a.sel_idx[rank] : rank;
}

// ---------------------------------------------------------------------------
// lse of the query rows.  Workgroup: 128 flattened (rank, head) rows of one
// sequence and KV head x a chunk of keys.
// ---------------------------------------------------------------------------
template <int D>
__global__ __launch_bounds__(kScoreThreads, 2) void score_lse_kernel(const ScoreArgs a) {
    __shared__ __attribute__((aligned(16))) uint16_t s_k[kLseBuffers][kBlockN][D];
    const int tid = threadIdx.x, lane = tid & 63, wave = uni(tid >> 6);
    const int g = lane >> 5, m = lane & 31;
    const int G = a.group;
    int item = blockIdx.x;
    const int kvh = item % a.hkv;
    item /= a.hkv;
    const int c = item % a.lse_chunks;
    int b, t;
    if (!find_block(item / a.lse_chunks, a.num_seqs, a.lse_per_seq, [&](int i) {
            int s0, s1;
            row_span(a, i, s0, s1);
            return (int)(((int64_t)(s1 - s0) * G + kLseRows - 1) / kLseRows);
        }, b, t))
        return;
    const int64_t base = a.cu[b];
    int s0, s1;
    row_span(a, b, s0, s1);
    const int64_t rows = (int64_t)(s1 - s0) * G, r0 = (int64_t)t * kLseRows;
    const int nrows = (int)(rows - r0 < kLseRows ? rows - r0 : kLseRows);
    // this lane's row
    const int64_t flat = r0 + min(wave * 32 + m, nrows - 1);
    const int rank = s0 + (int)(flat / G), head = kvh * G + (int)(flat % G);
    const int64_t tok = token_of(a, rank);
    const int pos = (int)(tok - base);
    const int pos_end = (int)(token_of(a, s0 + (int)((r0 + nrows - 1) / G)) - base);
    const int k0 = c * a.lse_kc, k1 = k0 + min(pos_end + 1 - k0, a.lse_kc);
    if (k0 >= k1)
        return;
    const int pos_min = uni(pos);                // rows ascend
    bf16x8 qf[D / 16];
    const uint16_t *qp = a.q + (tok * a.hq + head) * D + g * 8;
#pragma unroll
    for (int s = 0; s < D / 16; s++)
        qf[s] = *(const bf16x8 *)(qp + s * 16);

    // K tiles of 64 keys in four buffers, loaded three tiles ahead: kLoads loads
    // of a wave each; rows at or past k1 read as zeros (they are masked).
    constexpr int kAhead = kLseBuffers - 1;
    constexpr int kPc = D / 8, kLoads = kBlockN * kPc / 64 / kScoreWaves;
    const int row_bytes = a.hkv * D * 2;
    const uint16_t *kt = a.k + (base * a.hkv + kvh) * (int64_t)D;
    int koff[kLoads];
#pragma unroll
    for (int i = 0; i < kLoads; i++) {
        const int row = ((i * kScoreWaves + wave) * 64 + lane) / kPc;
        koff[i] = row * row_bytes + ((lane % kPc) ^ piece_swz<D>(row)) * 16;
    }
    auto stage = [&](int key, int buf) {
        if (key >= k1)
            return;
        const uint32_t dst = lds_addr_of(&s_k[buf][0][0]);
        const u32x4 r = raw_rsrc((const char *)kt + (int64_t)key * row_bytes,
                                 min(kBlockN, k1 - key) * row_bytes);
#pragma unroll
        for (int i = 0; i < kLoads; i++)
            lds_load16_at(r, dst + (i * kScoreWaves + wave) * 1024, koff[i]);
    };
#pragma unroll
    for (int i = 0; i < kAhead; i++)
        stage(k0 + i * kBlockN, i);
    // (the queries are waited for here: a wait inside the loop would be for
    // the tiles behind the current one too)
#pragma unroll
    for (int s = 0; s < D / 16; s++)
        asm volatile("" : "+v"(qf[s]));
    const bool live = wave * 32 < nrows;
    float mr = kNegInf, l = 0.f;
    int buf = 0;
    for (int key = k0; key < k1; key += kBlockN, buf = (buf + 1) % kLseBuffers) {
        if (key + (kAhead - 1) * kBlockN < k1)
            dma_wait_barrier_but<(kAhead - 1) * kLoads>();
        else
            dma_wait_barrier();
        stage(key + kAhead * kBlockN, (buf + kAhead) % kLseBuffers);
        if (!live)
            continue;
        // every fragment is on its way before the first product
        bf16x8 kf[2][D / 16];
#pragma unroll
        for (int sb = 0; sb < 2; sb++)
#pragma unroll
            for (int ss = 0; ss < D / 16; ss++)
                kf[sb][ss] = *(const bf16x8 *)&s_k[buf][sb * 32 + m]
                                                    [((ss * 2 + g) ^ piece_swz<D>(m)) * 8];
        __builtin_amdgcn_sched_barrier(0);
        f32x16 s[2] = {};
#pragma unroll
        for (int ss = 0; ss < D / 16; ss++)
#pragma unroll
            for (int sb = 0; sb < 2; sb++)
                s[sb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[sb][ss], qf[ss], s[sb], 0, 0, 0);
        if (key + 63 > pos_min || key + 64 > k1) {
#pragma unroll
            for (int sb = 0; sb < 2; sb++)
#pragma unroll
                for (int i = 0; i < 16; i++) {
                    const int j = key + sb * 32 + (i >> 2) * 8 + g * 4 + (i & 3);
                    if (j > pos || j >= k1)
                        s[sb][i] = kNegInf;
                }
        }
        float top[4];
#pragma unroll
        for (int i = 0; i < 4; i++) {
            const float x = max2(max2(s[0][i], s[0][i + 4]), max2(s[0][i + 8], s[0][i + 12]));
            const float y = max2(max2(s[1][i], s[1][i + 4]), max2(s[1][i + 8], s[1][i + 12]));
            top[i] = max2(x, y);
        }
        const float mx = pair_max(max2(max2(top[0], top[1]), max2(top[2], top[3]))) * a.scale_log2;
        const float mn = fmaxf(mr, mx), mc = mn == kNegInf ? 0.f : mn;
        float sum[2] = {};
#pragma unroll
        for (int sb = 0; sb < 2; sb++)
#pragma unroll
            for (int i = 0; i < 16; i++)
                sum[i & 1] += __builtin_amdgcn_exp2f(fmaf(s[sb][i], a.scale_log2, -mc));
        l = fmaf(l, __builtin_amdgcn_exp2f(mr - mc), sum[0] + sum[1]);
        mr = mn;
    }
    l = pair_sum(l);
    if (live && wave * 32 + m < nrows && g == 0)
        *(f32x2 *)(a.lse_part + (((int64_t)c * a.hq + head) * a.cap + rank) * 2) = f32x2{mr, l};
}

// ---------------------------------------------------------------------------
// The weights' sums.  Workgroup: KW x 64 keys of one sequence and KV head (KW
// waves side by side, 4 / KW rows of waves).  The rows that see them pass
// through LDS, kScoreRows at a time in two buffers filled by direct loads: a
// step has the next one's rows on their way while it multiplies its own, and
// the addresses, positions and lse of the one after that, so that a step waits
// for no chain of loads.  A row's 16-byte pieces are permuted (piece_swz).
// Each Q fragment feeds two products (the wave's two blocks of 32 keys), and
// the exponentials of one block of rows are issued between the products of the
// next.  A key's sum is compensated: what an addition drops is taken off the
// next block's sum.  4096 rows on 32768 keys, 32 / 8 heads: 576-606 us on four
// cards, 910-955 TFLOP/s, with or without that (1088 with rows staged through
// registers in 64-row steps); matrix cores busy in 44% of the cycles, the vector
// unit in 59%, of which the exponentials are half.
// ---------------------------------------------------------------------------
constexpr int kScoreRows = 128;

// First rank in [lo, hi) whose token is at or past `tok` (tokens ascend):
// every lane probes one of 64 equally spaced ranks.
__device__ __forceinline__ int first_rank(const ScoreArgs &a, int lo, int hi, int tok) {
    if (!a.cu_sel)
        return min(max(tok, lo), hi);
    const int lane = threadIdx.x & 63;
    while (lo < hi) {
        const int step = (hi - lo + 63) >> 6;
        const int64_t at = lo + (int64_t)lane * step;
        const int n = (int)__popcll(__ballot(at < hi && a.sel_idx[at] < tok));
        if (n == 0)
            break;
        const int64_t end = lo + (int64_t)n * step;
        lo += (n - 1) * step + 1;
        hi = (int)min((int64_t)hi, end);
    }
    return uni(lo);
}

template <int D, int KW>
__global__ __launch_bounds__(kScoreThreads, 2) void score_kernel(const ScoreArgs a) {
    constexpr int R = kScoreRows;
    constexpr int RW = kScoreWaves / KW;         // waves that share their keys
    constexpr int kBlocks = R / 32 / RW;         // row blocks per wave and step
    constexpr int kPc = D / 8;                   // 16-byte pieces of a row
    __shared__ __attribute__((aligned(16))) uint16_t s_q[2][R * D];
    __shared__ __attribute__((aligned(16))) float s_lse[3][R];
    __shared__ __attribute__((aligned(16))) int s_pos[3][R];
    __shared__ const uint16_t *s_row[3][R];
    const int tid = threadIdx.x, lane = tid & 63, wave = uni(tid >> 6);
    const int g = lane >> 5, m = lane & 31;
    const int kw = wave % KW, rw = wave / KW;
    const int G = a.group;
    const int kvh = blockIdx.x % a.hkv;
    int b, jb;
    if (!find_block(blockIdx.x / a.hkv, a.num_seqs, a.per_seq,
                    [&](int i) { return (a.cu[i + 1] - a.cu[i] + KW * 64 - 1) / (KW * 64); }, b, jb))
        return;
    const int base = a.cu[b];
    const int T = a.cu[b + 1] - base;
    const int key0 = jb * KW * 64, my0 = key0 + kw * 64;
    // this wave's keys
    bf16x8 kf[2][D / 16];
#pragma unroll
    for (int kb = 0; kb < 2; kb++) {
        const int key = my0 + kb * 32 + m;
        const uint16_t *kp = a.k + ((int64_t)(base + key) * a.hkv + kvh) * D + g * 8;
#pragma unroll
        for (int s = 0; s < D / 16; s++)
            kf[kb][s] = key < T ? *(const bf16x8 *)(kp + s * 16) : bf16x8{};
    }
    // the rows that see key0 (a row is a rank and one of the G heads)
    int s0, s1;
    row_span(a, b, s0, s1);
    s0 = first_rank(a, s0, s1, base + key0);
    const int rows = (s1 - s0) * G;              // (cap * Hq < 2^31 - 1024)
    const int steps = (rows + R - 1) / R;

    // Row tid / kSub of a step: kSub threads each, which join the key chunks
    // of a row whose lse is not given.  Rows past the last have the last one's
    // address and see nothing.
    constexpr int kSub = kScoreThreads / R;
    struct Meta {
        int tok, head;
        bool seen;
        float lse;
    };
    // rank and head (of the G) of the row that meta_load takes next, one step
    // of R rows at a time without a division
    int next_flat = tid / kSub, next_rank = s0 + next_flat / G, next_head = next_flat % G;
    const int step_ranks = R / G, step_heads = R % G;
    auto meta_load = [&]() {
        Meta x;
        const int rank = min(next_rank, s1 - 1), head = kvh * G + next_head;
        x.tok = token_of(a, rank);
        x.head = head;
        x.seen = next_flat < rows;
        next_flat += R;
        next_rank += step_ranks;
        next_head += step_heads;
        if (next_head >= G) {
            next_head -= G;
            next_rank++;
        }
        if (!a.lse_part) {
            x.lse = a.lse[head * a.cap + rank];
        } else {
            const int n = min((x.tok - base) / a.lse_kc + 1, a.lse_chunks);
            const f32x2 *pp = (const f32x2 *)a.lse_part + (int64_t)head * a.cap + rank;
            const int64_t stride = (int64_t)a.hq * a.cap;
            float M = kNegInf, l = 0.f;
#pragma unroll 1
            for (int c = tid % kSub; c < n; c += 4 * kSub) {
                f32x2 v[4];
#pragma unroll
                for (int i = 0; i < 4; i++)
                    v[i] = c + i * kSub < n ? pp[(c + i * kSub) * stride] : f32x2{kNegInf, 0.f};
                const float mn = fmaxf(fmaxf(fmaxf(v[0][0], v[1][0]), fmaxf(v[2][0], v[3][0])), M);
                const float mc = mn == kNegInf ? 0.f : mn;
                l *= __builtin_amdgcn_exp2f(M - mc);
#pragma unroll
                for (int i = 0; i < 4; i++)
                    l = fmaf(v[i][1], __builtin_amdgcn_exp2f(v[i][0] - mc), l);
                M = mn;
            }
#pragma unroll
            for (int sh = 1; sh < kSub; sh <<= 1) {
                const float mo = __shfl_xor(M, sh, 64), lo = __shfl_xor(l, sh, 64);
                const float mn = fmaxf(M, mo), mc = mn == kNegInf ? 0.f : mn;
                l = l * __builtin_amdgcn_exp2f(M - mc) + lo * __builtin_amdgcn_exp2f(mo - mc);
                M = mn;
            }
            x.lse = M + __builtin_amdgcn_logf(l);
        }
        return x;
    };
    auto meta_put = [&](int step, Meta x) {
        // not before here: a wait for these loads at the step's start would
        // wait for the rows that are loaded behind them too
        asm volatile("" : "+v"(x.tok), "+v"(x.lse));
        if (tid % kSub == 0) {
            s_row[step % 3][tid / kSub] = a.q + ((int64_t)x.tok * a.hq + x.head) * D;
            s_lse[step % 3][tid / kSub] = x.lse;
            s_pos[step % 3][tid / kSub] = x.seen ? x.tok - base : -1;
        }
    };
    // rows of a step into buffer step % 2: 64 / kPc rows per load
    auto stage = [&](int step) {
        constexpr int kRowsPer = 64 / kPc, kLoads = R / kRowsPer / kScoreWaves;
        const uint32_t dst = lds_addr_of(&s_q[step & 1][0]);
#pragma unroll
        for (int i = 0; i < kLoads; i++) {
            const int ld = i * kScoreWaves + wave, row = ld * kRowsPer + lane / kPc;
            lds_gather16(s_row[step % 3][row] + ((lane % kPc) ^ piece_swz<D>(row)) * 8, dst + ld * 1024);
        }
    };
    // (with what its roundings have dropped: a key's sum may have 100 000
    // blocks of terms)
    float sum[2] = {0.f, 0.f}, lost[2] = {0.f, 0.f};
    if (steps > 0) {
        meta_put(0, meta_load());
        __syncthreads();
        stage(0);
        if (steps > 1)
            meta_put(1, meta_load());
        dma_wait_barrier();
    }
    // (the keys are waited for here: a wait inside the loop would be for the
    // next step's rows too)
#pragma unroll
    for (int kb = 0; kb < 2; kb++)
#pragma unroll
        for (int s = 0; s < D / 16; s++)
            asm volatile("" : "+v"(kf[kb][s]));
#pragma unroll 1
    for (int step = 0; step < steps; step++) {
        const uint16_t *q = &s_q[step & 1][0];
        const float *lse = s_lse[step % 3];
        const int *pos = s_pos[step % 3];
        Meta next = {};
        if (step + 2 < steps)
            next = meta_load();
        if (step + 1 < steps)
            stage(step + 1);
        // scores of block x (of this wave's share of the step's rows)
        auto scores = [&](int x, f32x16 (&s)[2]) {
            const int row = (x * RW + rw) * 32 + m;
            s[0] = f32x16{};
            s[1] = f32x16{};
#pragma unroll
            for (int ss = 0; ss < D / 16; ss++) {
                const bf16x8 qf =
                    *(const bf16x8 *)&q[row * D + (((ss * 2 + g) ^ piece_swz<D>(m)) * 8)];
#pragma unroll
                for (int kb = 0; kb < 2; kb++)
                    s[kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(qf, kf[kb][ss], s[kb], 0, 0, 0);
            }
        };
        // their weights on this lane's two keys, added to each other before
        // they are added to the sum
        auto weights = [&](int x, const f32x16 (&s)[2], auto masked) {
            float part[2] = {0.f, 0.f};
#pragma unroll
            for (int qd = 0; qd < 4; qd++) {
                const int r = (x * RW + rw) * 32 + qd * 8 + g * 4;
                const f32x4 ls = *(const f32x4 *)&lse[r];
#pragma unroll
                for (int kb = 0; kb < 2; kb++)
#pragma unroll
                    for (int i = 0; i < 4; i++) {
                        float w = __builtin_amdgcn_exp2f(
                            fmaf(s[kb][qd * 4 + i], a.scale_log2, -ls[i]));
                        if constexpr (decltype(masked)::value)
                            w = my0 + kb * 32 + m > pos[r + i] ? 0.f : w;
                        part[kb] += w;
                    }
            }
#pragma unroll
            for (int kb = 0; kb < 2; kb++) {
                const float x = part[kb] - lost[kb], t = sum[kb] + x;
                lost[kb] = (t - sum[kb]) - x;
                sum[kb] = t;
            }
        };
        // rows ascend: the first one's position bounds what all see
        if (uni(pos[0]) < my0 + 63 || (step + 1) * R > rows) {
#pragma unroll 1
            for (int x = 0; x < kBlocks; x++) {
                f32x16 s[2];
                scores(x, s);
                weights(x, s, std::true_type{});
            }
        } else {
            f32x16 s[2][2];
            scores(0, s[0]);
#pragma unroll
            for (int x = 0; x < kBlocks; x++) {
                if (x + 1 < kBlocks)
                    scores(x + 1, s[(x + 1) & 1]);
                weights(x, s[x & 1], std::false_type{});
            }
        }
        if (step + 2 < steps)
            meta_put(step + 2, next);
        dma_wait_barrier();
    }
    // lane pairs, then the waves that share the keys
    float *s_sum = (float *)&s_q[0][0];
#pragma unroll
    for (int kb = 0; kb < 2; kb++) {
        sum[kb] = pair_sum(sum[kb]);
        if (g == 0)
            s_sum[(rw * KW + kw) * 64 + kb * 32 + m] = sum[kb];
    }
    __syncthreads();
    for (int x = tid; x < KW * 64; x += kScoreThreads) {
        const int key = key0 + x;
        if (key >= T)
            continue;
        float v = s_sum[x];
#pragma unroll
        for (int i = 1; i < RW; i++)
            v += s_sum[i * KW * 64 + x];
        const int64_t at = (int64_t)kvh * a.n + base + key;
        a.score[at] = (a.score_in ? a.score_in[at] : 0.f) + v;
    }
}

// ---------------------------------------------------------------------------
// One decoding step.  The scores of a chunk of keys: 16 x 16 x 32 products of
// the heads (rows) and 16 keys (columns).  With 4 P heads (P = 1, 2 or 4, heads
// past the last repeat it) the rows hold them 4 / P times, so that lane l's
// four rows are heads 4 ((l / 16) % P) + 0..3 whichever copy it looks at; of
// the four products of 64 keys it keeps those P whose keys are its own, and
// every lane has P keys' scores of four heads to exponentiate and store in
// whole lines.
//
// Bound by reading K.  Each wave streams keys of its own, 16 at a time, through
// a ring of slots in LDS (32 KB) filled by direct loads, whose lanes read
// whole rows (their pieces permuted, piece_swz); no barrier,
// a wave waits for its own oldest slots.  Workgroups of two waves, so that two
// of them share a CU's LDS and one's start and end hide behind the other.  16
// caches of 32K tokens, 8 KV heads: 1.14 GB in 220 us, 5.2 TB/s (278 us with
// fragments loaded from global memory).
// ---------------------------------------------------------------------------
constexpr int kStepWaves = kStepThreads / 64;
template <int D>
constexpr int step_ring() { return D == 128 ? 8 : 16; }

// Waits until at most N of the wave's vector-memory operations are outstanding.
template <int N>
__device__ __forceinline__ void wait_outstanding() {
    constexpr int n = N < 63 ? N : 63;
    __builtin_amdgcn_s_waitcnt(kWaitVmcnt0 | (n & 15) | ((n >> 4) << 14));
}

template <int D, int P>
__global__ __launch_bounds__(kStepThreads) void step_logits_kernel(const StepScoreArgs a) {
    constexpr int kRing = step_ring<D>(), kPc = D / 8;
    constexpr int kLoads = 16 * D * 2 / 1024;              // loads per slot
    constexpr int kCopies = 4 / P;
    __shared__ __attribute__((aligned(16))) uint16_t s_k[kStepWaves][kRing][16 * D];
    __shared__ f32x2 s_ml[kStepWaves][16];
    const int tid = threadIdx.x, lane = tid & 63, wave = uni(tid >> 6);
    const int kg = lane >> 4, n = lane & 15;
    const int G = a.group;
    int item = blockIdx.x;
    const int c = item % a.chunks;
    item /= a.chunks;
    const int hb = item % a.head_blocks;
    item /= a.head_blocks;
    const int kvh = item % a.hkv, b = item / a.hkv;
    if (!(a.gate[b] > decode_threshold(a)))
        return;
    const int base = a.cu[b];
    const int L = a.cu[b + 1] - base;
    const int k0 = c * a.kc, k1 = k0 + min(L - k0, a.kc);   // (a chunk may be 2^30 keys)
    if (k0 >= k1)
        return;
    // this wave's keys: its share of the chunk's blocks of 64
    const int blocks = (k1 - k0 + 63) / 64, per = (blocks + kStepWaves - 1) / kStepWaves;
    const int w0 = k0 + wave * per * 64, w1 = min(k1, w0 + per * 64);
    const char *kt = (const char *)(a.k + ((int64_t)base * a.hkv + kvh) * D);
    const int row_bytes = a.hkv * D * 2;
    // slot i of the wave: keys w0 + 16 i .. + 15; rows past the last key read as
    // zeros
    const int slots = w1 > w0 ? ((w1 - w0 + 63) / 64) * 4 : 0;
    int koff[kLoads];
#pragma unroll
    for (int x = 0; x < kLoads; x++) {
        const int row = (x * 64 + lane) / kPc;
        koff[x] = row * row_bytes + ((lane % kPc) ^ piece_swz<D>(row)) * 16;
    }
    auto stage = [&](int i) {
        const uint32_t dst = lds_addr_of(&s_k[wave][i % kRing][0]);
        const int key = w0 + i * 16;
        const u32x4 r = raw_rsrc(kt + (int64_t)key * row_bytes, max(min(16, w1 - key), 0) * row_bytes);
#pragma unroll
        for (int x = 0; x < kLoads; x++)
            lds_load16_at(r, dst + x * 1024, koff[x]);
    };
    const int nh = min(4 * P, G - hb * 4 * P), h0 = kvh * G + hb * 4 * P;
    bf16x8 qf[D / 32];
    {
        const int h = h0 + min(n % (4 * P), nh - 1);
#pragma unroll
        for (int s = 0; s < D / 32; s++)
            qf[s] = *(const bf16x8 *)(a.q + ((int64_t)b * a.hq + h) * D + s * 32 + kg * 8);
    }
    // (waited for before the ring is filled: a wait inside the loop would be
    // for the ring too)
#pragma unroll
    for (int s = 0; s < D / 32; s++)
        asm volatile("" : "+v"(qf[s]));
    for (int i = 0; i < min(kRing, slots); i++)
        stage(i);
    float mr[4], l[4];
#pragma unroll
    for (int i = 0; i < 4; i++) {
        mr[i] = kNegInf;
        l[i] = 0.f;
    }
    for (int s0 = 0; s0 < slots; s0 += 4) {
        f32x4 own[P];
        // The four slots are in when no more than what was issued behind them
        // is outstanding: the loads of the ring's other slots, and the stores
        // of the last kRing / 4 steps where there were as many.
        constexpr int kBehind = (kRing - 4) * kLoads;
        if (s0 + kRing > slots)
            wait_outstanding<0>();
        else if (s0 < kRing)
            wait_outstanding<kBehind>();
        else
            wait_outstanding<kBehind + kRing * P>();
        asm volatile("" ::: "memory");
#pragma unroll
        for (int j = 0; j < 4; j++) {
            const uint16_t *t = &s_k[wave][(s0 + j) % kRing][0];
            f32x4 s = {};
#pragma unroll
            for (int x = 0; x < D / 32; x++) {
                const bf16x8 kf =
                    *(const bf16x8 *)&t[n * D + (((x * 4 + kg) ^ piece_swz<D>(n)) * 8)];
                s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(qf[x], kf, s, 0, 0, 0);
            }
            // keys 16 j .. + 15 belong to copy j % kCopies
            if (kCopies == 1 || kg / P == j % kCopies)
                own[j / kCopies] = s;
        }
        asm volatile("" ::: "memory");
        if (s0 + kRing < slots) {
            // (the fragments have been read: the products took them)
#pragma unroll
            for (int j = 0; j < 4; j++)
                stage(s0 + kRing + j);
        }
#pragma unroll
        for (int x = 0; x < P; x++) {
            const int key = w0 + s0 * 16 + (x * kCopies + kg / P) * 16 + n;
            // (lanes past the last key store to the room behind the scores, past
            // the last head its score again: the number of stores is what the
            // waits count on)
            float *lp = a.logits + (key < w1 ? base + key : a.n * a.hq);
            const int64_t hs = key < w1 ? a.n : 0;
#pragma unroll
            for (int i = 0; i < 4; i++) {
                const float v = own[x][i] * a.scale_log2;
                lp[(h0 + min(4 * (kg % P) + i, nh - 1)) * hs] = v;
                const float y = key < w1 ? v : kNegInf;
                const float mn = fmaxf(mr[i], y), mc = mn == kNegInf ? 0.f : mn;
                l[i] = fmaf(l[i], __builtin_amdgcn_exp2f(mr[i] - mc), __builtin_amdgcn_exp2f(y - mc));
                mr[i] = mn;
            }
        }
    }
    // the lanes of a head (all but the bits of (kg % P)), then the waves
#pragma unroll
    for (int i = 0; i < 4; i++) {
#pragma unroll
        for (int sh = 1; sh < 64; sh <<= 1) {
            if (sh >= 16 && sh < 16 * P)
                continue;
            const float mo = __shfl_xor(mr[i], sh, 64), lo = __shfl_xor(l[i], sh, 64);
            const float mn = fmaxf(mr[i], mo), mc = mn == kNegInf ? 0.f : mn;
            l[i] = l[i] * __builtin_amdgcn_exp2f(mr[i] - mc) + lo * __builtin_amdgcn_exp2f(mo - mc);
            mr[i] = mn;
        }
        if (n == 0 && kg < P)
            s_ml[wave][kg * 4 + i] = f32x2{mr[i], l[i]};
    }
    __syncthreads();
    if (tid < nh) {
        float M = kNegInf, sum = 0.f;
#pragma unroll
        for (int w = 0; w < kStepWaves; w++) {
            const f32x2 v = s_ml[w][tid];
            const float mn = fmaxf(M, v[0]), mc = mn == kNegInf ? 0.f : mn;
            sum = sum * __builtin_amdgcn_exp2f(M - mc) + v[1] * __builtin_amdgcn_exp2f(v[0] - mc);
            M = mn;
        }
        *(f32x2 *)(a.ml + (((int64_t)b * a.hq + h0 + tid) * a.chunks + c) * 2) = f32x2{M, sum};
    }
}

// Workgroup: a chunk of kStepKeys keys of one sequence and KV head; each
// wave joins the (m, l) of its share of the heads first.  s_lse: as many
// floats as a KV head has query heads.
__global__ __launch_bounds__(kScoreThreads) void step_weights_kernel(const StepScoreArgs a) {
    extern __shared__ float s_lse[];
    const int tid = threadIdx.x, lane = tid & 63, wave = uni(tid >> 6);
    const int G = a.group;
    int item = blockIdx.x;
    const int kvh = item % a.hkv;
    item /= a.hkv;
    const int c = item % a.out_chunks, b = item / a.out_chunks;
    const int64_t base = a.cu[b];
    const int L = a.cu[b + 1] - (int)base;
    const int k0 = c * kStepKeys, k1 = min(L, k0 + kStepKeys);
    if (k0 >= k1)
        return;
    const int64_t at = (int64_t)kvh * a.n + base;
    if (!(a.gate[b] > decode_threshold(a))) {
        if (a.score_in != a.score)
            for (int j = k0 + tid; j < k1; j += kScoreThreads)
                a.score[at + j] = a.score_in ? a.score_in[at + j] : 0.f;
        return;
    }
    const int nch = min((L + a.kc - 1) / a.kc, a.chunks);
    for (int h = wave; h < G; h += kScoreWaves) {
        const f32x2 *ml = (const f32x2 *)(a.ml + ((int64_t)b * a.hq + kvh * G + h) * a.chunks * 2);
        float M = kNegInf;
        for (int x = lane; x < nch; x += 64)
            M = fmaxf(M, ml[x][0]);
#pragma unroll
        for (int sh = 1; sh < 64; sh <<= 1)
            M = fmaxf(M, __shfl_xor(M, sh, 64));
        const float Mc = M == kNegInf ? 0.f : M;
        float l = 0.f;
        for (int x = lane; x < nch; x += 64)
            l = fmaf(ml[x][1], __builtin_amdgcn_exp2f(ml[x][0] - Mc), l);
#pragma unroll
        for (int sh = 1; sh < 64; sh <<= 1)
            l += __shfl_xor(l, sh, 64);
        if (lane == 0)
            s_lse[h] = M + __builtin_amdgcn_logf(l);
    }
    __syncthreads();
    // every key's scores are on their way before the first sum is stored
    constexpr int kPer = kStepKeys / kScoreThreads;
    float w[kPer], in[kPer];
#pragma unroll
    for (int i = 0; i < kPer; i++) {
        const int j = min(k0 + tid + i * kScoreThreads, k1 - 1);
        in[i] = a.score_in ? a.score_in[at + j] : 0.f;
        w[i] = 0.f;
    }
#pragma unroll 4
    for (int h = 0; h < G; h++) {
        const float *lp = a.logits + (int64_t)(kvh * G + h) * a.n + base;
        const float lse = s_lse[h];
#pragma unroll
        for (int i = 0; i < kPer; i++)
            w[i] += __builtin_amdgcn_exp2f(lp[min(k0 + tid + i * kScoreThreads, k1 - 1)] - lse);
    }
#pragma unroll
    for (int i = 0; i < kPer; i++)
        if (k0 + tid + i * kScoreThreads < k1)
            a.score[at + k0 + tid + i * kScoreThreads] = in[i] + w[i];
}

template <int D>
hipError_t launch_score_d(const ScoreArgs &a, hipStream_t s) {
    if (a.lse_part) {
        hipLaunchKernelGGL((score_lse_kernel<D>), dim3(a.lse_items), dim3(kScoreThreads), 0, s, a);
        hipError_t e = hipGetLastError();
        if (e != hipSuccess)
            return e;
    }
    if (a.key_waves == 4)
        hipLaunchKernelGGL((score_kernel<D, 4>), dim3(a.items), dim3(kScoreThreads), 0, s, a);
    else if (a.key_waves == 2)
        hipLaunchKernelGGL((score_kernel<D, 2>), dim3(a.items), dim3(kScoreThreads), 0, s, a);
    else
        hipLaunchKernelGGL((score_kernel<D, 1>), dim3(a.items), dim3(kScoreThreads), 0, s, a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_cache_score(const ScoreArgs &a, hipStream_t s) {
    return a.head_dim == 128 ? launch_score_d<128>(a, s) : launch_score_d<64>(a, s);
}

hipError_t launch_decode_score(const StepScoreArgs &a, hipStream_t s) {
    auto launch = [&](auto d, auto p) {
        hipLaunchKernelGGL((step_logits_kernel<decltype(d)::value, decltype(p)::value>),
                           dim3(a.items), dim3(kStepThreads), 0, s, a);
    };
    auto launch_d = [&](auto d) {
        if (a.head_copies == 4)
            launch(d, std::integral_constant<int, 1>{});
        else if (a.head_copies == 2)
            launch(d, std::integral_constant<int, 2>{});
        else
            launch(d, std::integral_constant<int, 4>{});
    };
    if (a.head_dim == 128)
        launch_d(std::integral_constant<int, 128>{});
    else
        launch_d(std::integral_constant<int, 64>{});
    hipError_t e = hipGetLastError();
    if (e != hipSuccess)
        return e;
    hipLaunchKernelGGL(step_weights_kernel, dim3(a.out_items), dim3(kScoreThreads),
                       a.group * sizeof(float), s, a);
    return hipGetLastError();
}

}  // namespace logo
