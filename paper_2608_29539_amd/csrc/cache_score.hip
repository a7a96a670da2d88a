// cache_score.hip -- the attention weight that every cached key has received
// (logo_cache_score for a prompt's queries, logo_decode_score for one decoding
// step):
//   a[h][j] = a_in[h][j] + sum_i sum_{g < G} 2^(c q_{i, hG+g} . k_{j, h} - lse_{i, hG+g})
// over the query rows i that see key j, lse the base-2 log-sum-exp of the
// row's scaled scores, c = softmax_scale log2(e).  The G heads of a KV head add
// to the same key; every sum is taken in a fixed order, so results do not
// change from run to run.
//
//   score_lse_kernel, score_lse_join_kernel   lse where the caller has none
//   score_kernel            key-stationary: a wave keeps 64 keys of one KV head
//                           in registers (the MFMA's B operand) and walks over
//                           the rows that see them, so a key's sum stays in
//                           its lane
//   step_logits_kernel      one query per sequence: the scaled scores of a
//                           chunk of keys and their (m, l) per head
//   step_weights_kernel     2^(score - lse) summed over the heads
#include "attn_common.h"
#include "decode_common.h"
#include "logo_internal.h"

namespace logo {
namespace {

constexpr int kScoreThreads = 256;
constexpr int kScoreWaves = kScoreThreads / 64;
constexpr int kRowPad = 8;                  // bf16 of padding per staged row (bank offset)

// Item t of the blocks that sequences have n(b) of each, sequence-major: its
// sequence and block; false past the last.  Every wave searches for itself.
template <class F>
__device__ __forceinline__ bool find_block(int t, int B, F &&n, int &b, int &j) {
    const int lane = threadIdx.x & 63;
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
    if (a.sel_idx) {
        s0 = min(a.cu_sel[b], a.cap);
        s1 = min(a.cu_sel[b + 1], a.cap);
    } else {
        s0 = a.cu[b];
        s1 = a.cu[b + 1];
    }
}
__device__ __forceinline__ int token_of(const ScoreArgs &a, int rank) {
    return a.sel_idx ? a.sel_idx[rank] : rank;
}

// 32 x 32 block of scores: rows of A (16-byte fragments in LDS, `stride`
// bf16 apart) with the B fragments in registers.
template <int D>
__device__ __forceinline__ f32x16 block_scores(const uint16_t *frag, const bf16x8 (&bf)[D / 16]) {
    f32x16 s = {};
#pragma unroll
    for (int ss = 0; ss < D / 16; ss++)
        s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(*(const bf16x8 *)(frag + ss * 16), bf[ss], s,
                                                    0, 0, 0);
    return s;
}

// ---------------------------------------------------------------------------
// lse of the query rows.  Workgroup: 128 flattened (rank, head) rows of one
// sequence and KV head x a chunk of keys, 64 keys staged at a time.
// ---------------------------------------------------------------------------
template <int D>
__global__ __launch_bounds__(kScoreThreads) void score_lse_kernel(const ScoreArgs a) {
    __shared__ __attribute__((aligned(16))) uint16_t s_k[2][64][D + kRowPad];
    const int tid = threadIdx.x, lane = tid & 63, wave = uni(tid >> 6);
    const int g = lane >> 5, m = lane & 31;
    const int G = a.group;
    int item = blockIdx.x;
    const int kvh = item % a.hkv;
    item /= a.hkv;
    const int c = item % a.lse_chunks;
    int b, t;
    if (!find_block(item / a.lse_chunks, a.num_seqs, [&](int i) {
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
    const int k0 = c * a.lse_kc, k1 = min(pos_end + 1, k0 + a.lse_kc);
    if (k0 >= k1)
        return;
    const int pos_min = uni(pos);                // rows ascend
    bf16x8 qf[D / 16];
    const uint16_t *qp = a.q + (tok * a.hq + head) * D + g * 8;
#pragma unroll
    for (int s = 0; s < D / 16; s++)
        qf[s] = *(const bf16x8 *)(qp + s * 16);

    // 64 keys x D: each thread D / 32 pieces of 8
    constexpr int kPieces = 64 * D / 8 / kScoreThreads;
    const uint16_t *kb = a.k + (base * a.hkv + kvh) * (int64_t)D;
    u32x4 reg[kPieces];
    auto load = [&](int key) {
#pragma unroll
        for (int i = 0; i < kPieces; i++) {
            const int x = tid + i * kScoreThreads, row = x / (D / 8), col = x % (D / 8);
            reg[i] = key + row < k1
                         ? *(const u32x4 *)(kb + (int64_t)(key + row) * a.hkv * D + col * 8)
                         : u32x4{};
        }
    };
    auto put = [&](int buf) {
#pragma unroll
        for (int i = 0; i < kPieces; i++) {
            const int x = tid + i * kScoreThreads, row = x / (D / 8), col = x % (D / 8);
            *(u32x4 *)&s_k[buf][row][col * 8] = reg[i];
        }
    };
    const bool live = wave * 32 < nrows;
    float mr = kNegInf, l = 0.f;
    load(k0);
    put(0);
    int buf = 0;
    for (int key = k0; key < k1; key += 64, buf ^= 1) {
        __syncthreads();
        const bool more = key + 64 < k1;
        if (more)
            load(key + 64);
        if (live) {
            f32x16 s[2];
#pragma unroll
            for (int sb = 0; sb < 2; sb++)
                s[sb] = block_scores<D>(&s_k[buf][sb * 32 + m][g * 8], qf);
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
            float mx = kNegInf;
#pragma unroll
            for (int sb = 0; sb < 2; sb++)
#pragma unroll
                for (int i = 0; i < 16; i++)
                    mx = fmaxf(mx, s[sb][i]);
            mx = pair_max(mx) * a.scale_log2;
            const float mn = fmaxf(mr, mx), mc = mn == kNegInf ? 0.f : mn;
            float sum = 0.f;
#pragma unroll
            for (int sb = 0; sb < 2; sb++)
#pragma unroll
                for (int i = 0; i < 16; i++)
                    sum += __builtin_amdgcn_exp2f(fmaf(s[sb][i], a.scale_log2, -mc));
            l = fmaf(l, __builtin_amdgcn_exp2f(mr - mc), sum);
            mr = mn;
        }
        if (more)
            put(buf ^ 1);
    }
    l = pair_sum(l);
    if (live && wave * 32 + m < nrows && g == 0)
        *(f32x2 *)(a.lse_part + (((int64_t)c * a.hq + head) * a.cap + rank) * 2) = f32x2{mr, l};
}

// lse[head][rank] from the chunks' (m, l); chunks past the row's position
// were not written.
__global__ __launch_bounds__(256) void score_lse_join_kernel(const ScoreArgs a) {
    const int64_t x = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int rank = (int)(x % a.cap), head = (int)(x / a.cap);
    if (head >= a.hq || (a.sel_idx && rank >= a.cu_sel[a.num_seqs]))
        return;
    const int64_t tok = token_of(a, rank);
    int lo = 0, hi = a.num_seqs - 1;             // the token's sequence
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (a.cu[mid] <= tok)
            lo = mid;
        else
            hi = mid - 1;
    }
    const int n = min((int)(tok - a.cu[lo]) / a.lse_kc + 1, a.lse_chunks);
    float M = kNegInf, l = 0.f;
    for (int c = 0; c < n; c++) {
        const f32x2 v = *(const f32x2 *)(a.lse_part + (((int64_t)c * a.hq + head) * a.cap + rank) * 2);
        const float mn = fmaxf(M, v[0]), mc = mn == kNegInf ? 0.f : mn;
        l = l * __builtin_amdgcn_exp2f(M - mc) + v[1] * __builtin_amdgcn_exp2f(v[0] - mc);
        M = mn;
    }
    a.lse_out[(int64_t)head * a.cap + rank] = M + __builtin_amdgcn_logf(l);
}

// ---------------------------------------------------------------------------
// The weights' sums.  Workgroup: KW x 64 keys of one sequence and KV head (KW
// waves side by side, 4 / KW rows of waves); the rows that see them are staged
// kScoreRows at a time, and each row of waves takes its share.
// ---------------------------------------------------------------------------
constexpr int kScoreRows = 128;

template <int D, int KW>
__global__ __launch_bounds__(kScoreThreads, 2) void score_kernel(const ScoreArgs a) {
    constexpr int RW = kScoreWaves / KW;         // waves that share their keys
    constexpr int kBlocks = kScoreRows / 32 / RW;   // row blocks per wave and step
    __shared__ __attribute__((aligned(16))) uint16_t s_q[kScoreRows][D + kRowPad];
    __shared__ __attribute__((aligned(16))) float s_lse[kScoreRows];
    __shared__ __attribute__((aligned(16))) int s_pos[kScoreRows];
    __shared__ float s_sum[RW][KW * 64];
    const int tid = threadIdx.x, lane = tid & 63, wave = uni(tid >> 6);
    const int g = lane >> 5, m = lane & 31;
    const int kw = wave % KW, rw = wave / KW;
    const int G = a.group;
    const int kvh = blockIdx.x % a.hkv;
    int b, jb;
    if (!find_block(blockIdx.x / a.hkv, a.num_seqs,
                    [&](int i) { return (a.cu[i + 1] - a.cu[i] + KW * 64 - 1) / (KW * 64); }, b, jb))
        return;
    const int64_t base = a.cu[b];
    const int T = a.cu[b + 1] - (int)base;
    const int key0 = jb * KW * 64, my0 = key0 + kw * 64;
    // the rows that see key0: from the first of position >= key0
    int s0, s1;
    row_span(a, b, s0, s1);
    {
        int hi = s1;
        while (s0 < hi) {
            const int mid = s0 + ((hi - s0) >> 1);
            if (token_of(a, mid) - base < key0)
                s0 = mid + 1;
            else
                hi = mid;
        }
    }
    const int64_t rows = (int64_t)(s1 - s0) * G;

    // this wave's keys
    bf16x8 kf[2][D / 16];
#pragma unroll
    for (int kb = 0; kb < 2; kb++) {
        const int key = my0 + kb * 32 + m;
        const uint16_t *kp = a.k + ((base + key) * a.hkv + kvh) * (int64_t)D + g * 8;
#pragma unroll
        for (int s = 0; s < D / 16; s++)
            kf[kb][s] = key < T ? *(const bf16x8 *)(kp + s * 16) : bf16x8{};
    }
    float sum[2] = {0.f, 0.f};

    for (int64_t r0 = 0; r0 < rows; r0 += kScoreRows) {
        const int nrows = (int)(rows - r0 < kScoreRows ? rows - r0 : kScoreRows);
        __syncthreads();                         // the last step's rows are read
        constexpr int kPieces = kScoreRows * D / 8 / kScoreThreads;
#pragma unroll
        for (int i = 0; i < kPieces; i++) {
            const int x = tid + i * kScoreThreads, row = x / (D / 8), col = x % (D / 8);
            u32x4 v = {};
            if (row < nrows) {
                const int64_t flat = r0 + row;
                const int64_t tok = token_of(a, s0 + (int)(flat / G));
                v = *(const u32x4 *)(a.q + (tok * a.hq + kvh * G + flat % G) * D + col * 8);
            }
            *(u32x4 *)&s_q[row][col * 8] = v;
        }
        if (tid < kScoreRows) {
            float lse = 0.f;
            int pos = -1;                        // rows past the last see nothing
            if (tid < nrows) {
                const int64_t flat = r0 + tid;
                const int rank = s0 + (int)(flat / G);
                lse = a.lse[(int64_t)(kvh * G + flat % G) * a.cap + rank];
                pos = (int)(token_of(a, rank) - base);
            }
            s_lse[tid] = lse;
            s_pos[tid] = pos;
        }
        __syncthreads();
#pragma unroll 1
        for (int x = 0; x < kBlocks; x++) {
            const int rb = x * RW + rw;          // 32-row block of the staged rows
            // rows ascend: the first one's position bounds what all see, and
            // the last block may have rows past the end
            const bool masked = uni(s_pos[rb * 32]) < my0 + 63 || (rb + 1) * 32 > nrows;
#pragma unroll
            for (int kb = 0; kb < 2; kb++) {
                const f32x16 s = block_scores<D>(&s_q[rb * 32 + m][g * 8], kf[kb]);
                const int key = my0 + kb * 32 + m;
                float part = 0.f;
#pragma unroll
                for (int q = 0; q < 4; q++) {
                    const f32x4 ls = *(const f32x4 *)&s_lse[rb * 32 + q * 8 + g * 4];
#pragma unroll
                    for (int i = 0; i < 4; i++) {
                        float w = __builtin_amdgcn_exp2f(fmaf(s[q * 4 + i], a.scale_log2, -ls[i]));
                        if (masked && key > s_pos[rb * 32 + q * 8 + g * 4 + i])
                            w = 0.f;
                        part += w;
                    }
                }
                sum[kb] += part;
            }
        }
    }
    // lane pairs, then the waves that share the keys
#pragma unroll
    for (int kb = 0; kb < 2; kb++) {
        sum[kb] = pair_sum(sum[kb]);
        if (g == 0)
            s_sum[rw][kw * 64 + kb * 32 + m] = sum[kb];
    }
    __syncthreads();
    for (int x = tid; x < KW * 64; x += kScoreThreads) {
        const int key = key0 + x;
        if (key >= T)
            continue;
        float v = s_sum[0][x];
#pragma unroll
        for (int i = 1; i < RW; i++)
            v += s_sum[i][x];
        const int64_t at = (int64_t)kvh * a.n + base + key;
        a.score[at] = (a.score_in ? a.score_in[at] : 0.f) + v;
    }
}

// ---------------------------------------------------------------------------
// One decoding step.  The scores of a chunk of keys: 16 x 16 x 32 products of
// up to 16 heads (rows, of which G exist) and 16 keys; lane l holds key l % 16
// and heads 4 (l / 16) + 0..3.
// ---------------------------------------------------------------------------
template <int D>
__global__ __launch_bounds__(kScoreThreads) void step_logits_kernel(const StepScoreArgs a) {
    __shared__ f32x2 s_ml[kScoreWaves][16];
    const int tid = threadIdx.x, lane = tid & 63, wave = uni(tid >> 6);
    const int kg = lane >> 4, n = lane & 15;
    const int G = a.group;
    int item = blockIdx.x;
    const int kvh = item % a.hkv;
    item /= a.hkv;
    const int hb = item % a.head_blocks;
    item /= a.head_blocks;
    const int c = item % a.chunks, b = item / a.chunks;
    if (!(a.gate[b] > decode_threshold(a)))
        return;
    const int64_t base = a.cu[b];
    const int L = a.cu[b + 1] - (int)base;
    const int k0 = c * a.kc, k1 = min(L, k0 + a.kc);
    if (k0 >= k1)
        return;
    const int nh = min(16, G - hb * 16), h0 = kvh * G + hb * 16;
    bf16x8 qf[D / 32];
#pragma unroll
    for (int s = 0; s < D / 32; s++)
        qf[s] = n < nh ? *(const bf16x8 *)(a.q + ((int64_t)b * a.hq + h0 + n) * D + s * 32 + kg * 8)
                       : bf16x8{};
    float mr[4], l[4];
#pragma unroll
    for (int i = 0; i < 4; i++) {
        mr[i] = kNegInf;
        l[i] = 0.f;
    }
    const uint16_t *kb = a.k + (base * a.hkv + kvh) * (int64_t)D + kg * 8;
    for (int key = k0 + wave * 16; key < k1; key += kScoreWaves * 16) {
        const int j = key + n;
        const uint16_t *kp = kb + (int64_t)j * a.hkv * D;
        f32x4 s = {};
#pragma unroll
        for (int x = 0; x < D / 32; x++) {
            const bf16x8 kf = j < k1 ? *(const bf16x8 *)(kp + x * 32) : bf16x8{};
            s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(qf[x], kf, s, 0, 0, 0);
        }
#pragma unroll
        for (int i = 0; i < 4; i++) {
            const int h = kg * 4 + i;
            const float v = s[i] * a.scale_log2;
            if (h < nh && j < k1)
                a.logits[(int64_t)(h0 + h) * a.n + base + j] = v;
            const float x = j < k1 ? v : kNegInf;
            const float mn = fmaxf(mr[i], x), mc = mn == kNegInf ? 0.f : mn;
            l[i] = fmaf(l[i], __builtin_amdgcn_exp2f(mr[i] - mc), __builtin_amdgcn_exp2f(x - mc));
            mr[i] = mn;
        }
    }
    // the 16 lanes of a head, then the waves
#pragma unroll
    for (int i = 0; i < 4; i++) {
#pragma unroll
        for (int sh = 1; sh < 16; sh <<= 1) {
            const float mo = __shfl_xor(mr[i], sh, 64), lo = __shfl_xor(l[i], sh, 64);
            const float mn = fmaxf(mr[i], mo), mc = mn == kNegInf ? 0.f : mn;
            l[i] = l[i] * __builtin_amdgcn_exp2f(mr[i] - mc) + lo * __builtin_amdgcn_exp2f(mo - mc);
            mr[i] = mn;
        }
        if (n == 0)
            s_ml[wave][kg * 4 + i] = f32x2{mr[i], l[i]};
    }
    __syncthreads();
    if (tid < nh) {
        float M = kNegInf, sum = 0.f;
#pragma unroll
        for (int w = 0; w < kScoreWaves; w++) {
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
    for (int j = k0 + tid; j < k1; j += kScoreThreads) {
        float w = 0.f;
        for (int h = 0; h < G; h++)
            w += __builtin_amdgcn_exp2f(a.logits[(int64_t)(kvh * G + h) * a.n + base + j] - s_lse[h]);
        a.score[at + j] = (a.score_in ? a.score_in[at + j] : 0.f) + w;
    }
}

template <int D>
hipError_t launch_score_d(const ScoreArgs &a, hipStream_t s) {
    if (a.lse_out) {
        hipLaunchKernelGGL((score_lse_kernel<D>), dim3(a.lse_items), dim3(kScoreThreads), 0, s, a);
        hipError_t e = hipGetLastError();
        if (e != hipSuccess)
            return e;
        const int64_t n = (int64_t)a.cap * a.hq;
        hipLaunchKernelGGL(score_lse_join_kernel, dim3((n + 255) / 256), dim3(256), 0, s, a);
        if ((e = hipGetLastError()) != hipSuccess)
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
    const dim3 grid(a.items), block(kScoreThreads);
    if (a.head_dim == 128)
        hipLaunchKernelGGL((step_logits_kernel<128>), grid, block, 0, s, a);
    else
        hipLaunchKernelGGL((step_logits_kernel<64>), grid, block, 0, s, a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess)
        return e;
    hipLaunchKernelGGL(step_weights_kernel, dim3(a.out_items), block, a.group * sizeof(float), s, a);
    return hipGetLastError();
}

}  // namespace logo
