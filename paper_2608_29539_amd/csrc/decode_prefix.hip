// decode_prefix.hip -- one decoding step of the layer for groups of sequences
// that share a prefix (Sec. 3.3 and App. B, Autoregressive Decoding, with the
// shared rows read once per group instead of once per sequence).  Sequence b
// of prefix r has the cache [prefix r ; its own rows], P_r + S_b keys; its new
// token's query attends to the last min(P_r + S_b, w) of them and, when its
// gate passes the threshold, to all of them.
//
// Mathematics.  The softmax over the union of disjoint key ranges is joined
// from the ranges' (O, m, l) = (sum_j 2^(s_j - m) v_j, m, sum_j 2^(s_j - m)):
//   O = sum_i 2^(m_i - M) O_i / sum_i 2^(m_i - M) l_i,   M = max_i m_i.
// So a prefix's keys are attended to by the queries of its whole group at
// once -- (sequence, head) pairs of one KV head are the rows of a matrix
// product -- and each sequence's own keys by its own heads.  Where the global
// branch reads the local one's tensors, its keys outside the window are
// attended to only, and the local branch's result joined for the others.
//
//   prefix_attn_kernel     one workgroup per (range, KV head, chunk of keys,
//                          128 rows): the ranges are the prefix's part of the
//                          local and of the global branch (rows: the group's
//                          sequences whose window reaches it, the selected
//                          ones) and the sequence's own part of either (rows:
//                          the heads of one sequence).  Four waves of 32 rows;
//                          with 64 rows or fewer two waves take the keys of a
//                          tile by halves.  K / V tiles of 64 keys go to LDS
//                          directly, one tile ahead.
//   prefix_combine_kernel  joins the chunks of each (sequence, head), applies
//                          ContextNorm and the fusion, rounds once to bf16.
//
// P is rounded to bf16 for the PV product, as in the layer's kernels (its row
// sum takes the rounded values); everything else is fp32.
#include "attn_tiles.h"
#include "decode_common.h"
#include "logo_internal.h"

#include <type_traits>

namespace logo {
namespace {

constexpr int kPfWaves = kPrefixThreads / 64;
constexpr float kLazyP = 8.f;               // exp2-domain headroom of the running max

// Kinds of key range (the order of the work items).
enum { kPfxGlobal = 0, kOwnGlobal = 1, kPfxLocal = 2, kOwnLocal = 3 };

// Keys [lo, hi) of range `kind` that a sequence with P prefix rows and S rows
// of its own sees, in rows of the prefix or of the sequence.
__device__ __forceinline__ void key_range(const PrefixArgs &a, int kind, int P, int S, int &lo,
                                          int &hi) {
    if (kind == kPfxGlobal || kind == kPfxLocal) {
        const int edge = S >= a.window ? P : max(0, P - (a.window - S));   // the window's first row
        lo = kind == kPfxLocal ? edge : 0;
        hi = kind == kPfxLocal || !a.share ? P : edge;
    } else {
        const int edge = S > a.window ? S - a.window : 0;
        lo = kind == kOwnLocal ? edge : 0;
        hi = kind == kOwnLocal || !a.share ? S : edge;
    }
}
// First key of chunk 0 of a range: the first that any row can see.
__device__ __forceinline__ int chunk_base(const PrefixArgs &a, int kind, int len) {
    return kind == kPfxLocal || kind == kOwnLocal ? max(0, len - a.window) : 0;
}

template <int D>
struct alignas(16) PrefixSmem {
    uint16_t k[2][kBlockN][D + kKPad];
    uint16_t v[2][kBlockN][D];
};

template <int D>
__global__ __launch_bounds__(kPrefixThreads, 2) void prefix_attn_kernel(const PrefixArgs a) {
    __shared__ PrefixSmem<D> sm;
    __shared__ int s_seq[kPrefixRows], s_cnt[kPfWaves];
    const int tid = threadIdx.x, lane = tid & 63, wave = uni(tid >> 6);
    const int g = lane >> 5, m = lane & 31;

    // work item -> range, sequence or prefix, KV head, chunk, row tile; the
    // workgroup past them builds the list of selected sequences instead
    int item = blockIdx.x, kind = 0;
    if (item == a.first[4]) {
        build_active_list<kPrefixThreads>(a);
        return;
    }
    while (item >= a.first[kind + 1])
        kind++;
    item -= a.first[kind];
    const int nch = a.chunks[kind], kc = a.kc[kind];
    const bool global = kind == kPfxGlobal || kind == kOwnGlobal;
    const bool own = kind == kOwnGlobal || kind == kOwnLocal;
    // the row tiles of one chunk run on the same XCD (workgroups go to the
    // XCDs in turn), so that the later ones find its keys in that XCD's L2
    const int tiles = own ? a.own_tiles : a.pfx_tiles;
    const int u = item / (kQueues * tiles), rem = item % (kQueues * tiles);
    const int t = rem / kQueues, pair = u * kQueues + rem % kQueues;
    const int kvh = pair % a.hkv, c = (pair / a.hkv) % nch, r = pair / a.hkv / nch;
    if (r >= (own ? a.num_seqs : a.num_prefixes))
        return;
    const float thr = decode_threshold(a);
    if (own && global && !(a.gate[r] > thr))
        return;                                  // an unselected token: window only

    // the chunk's keys [k0, k1) and the tile's rows: s_seq[i] for the
    // sequences of ranks rank0, rank0 + 1, ... among those that see the chunk
    const int32_t *cu = own ? a.cu : a.cu_pre;
    const int64_t base = cu[r];
    const int len = cu[r + 1] - (int)base;
    int k0 = chunk_base(a, kind, len) + c * kc;
    int k1 = min(len, k0 + kc);
    if (k0 >= k1)
        return;
    const int rank0 = t * kPrefixRows / a.group;
    int count = 0;
    if (own) {
        int lo, hi;
        key_range(a, kind, 0, len, lo, hi);
        k0 = max(k0, lo);
        k1 = min(k1, hi);
        if (k0 >= k1)
            return;
        if (tid == 0)
            s_seq[0] = r;
        count = 1;
        __syncthreads();
    } else {
        const int g0 = a.cu_grp[r], g1 = a.cu_grp[r + 1];
        const int most = (t * kPrefixRows + kPrefixRows - 1) / a.group - rank0 + 1;
        for (int c0 = g0; c0 < g1; c0 += kPrefixThreads) {
            const int b = c0 + tid;
            bool in = b < g1 && (!global || a.gate[b] > thr);
            if (in) {
                int lo, hi;
                key_range(a, kind, len, a.cu[b + 1] - a.cu[b], lo, hi);
                in = max(lo, k0) < min(hi, k1);
            }
            const uint64_t bal = __ballot(in);
            if (lane == 0)
                s_cnt[wave] = (int)__popcll(bal);
            __syncthreads();
            int at = count + (int)__builtin_amdgcn_mbcnt_hi(
                                 (uint32_t)(bal >> 32),
                                 __builtin_amdgcn_mbcnt_lo((uint32_t)bal, 0)) - rank0;
#pragma unroll
            for (int i = 0; i < kPfWaves; i++) {
                const int n = s_cnt[i];
                at += i < wave ? n : 0;
                count += n;
            }
            if (in && at >= 0 && at < most)
                s_seq[at] = b;
            __syncthreads();
        }
    }
    const int64_t left = (int64_t)count * a.group - (int64_t)t * kPrefixRows;
    if (left <= 0)
        return;
    const int nrows = left < kPrefixRows ? (int)left : kPrefixRows;

    // waves: row block rb, and with few rows the key half kg of each tile
    const int wr = nrows > 64 ? 4 : nrows > 32 ? 2 : 1;
    const int wk = wr == 4 ? 1 : 2;
    const int rb = wave % wr, kg = wave / wr;
    const bool live = kg < wk && rb * 32 < nrows;

    const int row_bytes = a.hkv * D * 2;
    const uint16_t *kt = own ? (global ? a.k_g : a.k) : (global ? a.kp_g : a.kp);
    const uint16_t *vt = own ? (global ? a.v_g : a.v) : (global ? a.vp_g : a.vp);
    kt += (base * a.hkv + kvh) * (int64_t)D;
    vt += (base * a.hkv + kvh) * (int64_t)D;
    Dma<D, kPfWaves> dma;
    dma_plan<D, kPfWaves>(dma, wave, lane, row_bytes);
    auto stage = [&](int buf, int key) {
        dma_k<D, kPfWaves>(&sm.k[buf][0][0], dma, kt, k1, key, row_bytes, wave);
        dma_v<D, kPfWaves>(&sm.v[buf][0][0], dma, vt, k1, key, row_bytes, wave);
    };
    stage(0, k0);

    // this lane's query row; rows past the last repeat it and are not stored
    const int ri = min(rb * 32 + m, nrows - 1);
    const bool row_valid = rb * 32 + m < nrows;
    const int flat = t * kPrefixRows + ri;
    const int b = s_seq[flat / a.group - rank0];
    const int head = kvh * a.group + flat % a.group;
    const uint16_t *qp = (global ? a.q_g : a.q) + ((int64_t)b * a.hq + head) * D + g * 8;
    bf16x8 qf[D / 16];
#pragma unroll
    for (int s = 0; s < D / 16; s++)
        qf[s] = *(const bf16x8 *)(qp + s * 16);
    int lo, hi;
    {
        const int S = a.cu[b + 1] - a.cu[b];
        key_range(a, kind, len, own ? len : S, lo, hi);
        lo = max(lo, k0);
        hi = min(hi, k1);
    }
    // keys that every row of the wave sees: tiles inside need no mask
    int all_lo = lo, all_hi = hi;
#pragma unroll
    for (int sh = 1; sh < 32; sh <<= 1) {
        all_lo = max(all_lo, __shfl_xor(all_lo, sh, 64));
        all_hi = min(all_hi, __shfl_xor(all_hi, sh, 64));
    }
    all_lo = uni(all_lo);
    all_hi = uni(all_hi);

    const int vt_row = 4 * g + ((lane & 15) >> 2);
    const int vt_col = 16 * ((lane >> 4) & 1) + 4 * (lane & 3);
    int vt_scol[D / 32];
#pragma unroll
    for (int cb = 0; cb < D / 32; cb++)
        vt_scol[cb] = (cb ^ vswz<D>(vt_row)) * 32 + vt_col;
    const float sc = a.scale_log2;
    const bf16x2 ones = {(__bf16)1.0f, (__bf16)1.0f};
    f32x16 acc[D / 32];
#pragma unroll
    for (int cb = 0; cb < D / 32; cb++)
        acc[cb] = f32x16{};
    float m_ref = kNegInf, l_run = 0.f;

    // One wave's share of the tile in buffer `buf`, keys key0 + 32 sb0 ...:
    // N blocks of 32 keys.
    auto step = [&](auto n_blocks, int buf, int sb0, int key0) {
        constexpr int N = decltype(n_blocks)::value;
        f32x16 s[N];
#pragma unroll
        for (int sb = 0; sb < N; sb++)
            s[sb] = f32x16{};
#pragma unroll
        for (int ss = 0; ss < D / 16; ss++)
#pragma unroll
            for (int sb = 0; sb < N; sb++) {
                const bf16x8 kf = *(const bf16x8 *)&sm.k[buf][(sb0 + sb) * 32 + m][ss * 16 + g * 8];
                s[sb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, qf[ss], s[sb], 0, 0, 0);
            }
        if (key0 + sb0 * 32 < all_lo || key0 + (sb0 + N) * 32 > all_hi) {
#pragma unroll
            for (int sb = 0; sb < N; sb++)
#pragma unroll
                for (int i = 0; i < 16; i++) {
                    const int key = key0 + (sb0 + sb) * 32 + (i >> 2) * 8 + g * 4 + (i & 3);
                    if (key < lo || key >= hi)
                        s[sb][i] = kNegInf;
                }
        }
        float mx = kNegInf;
#pragma unroll
        for (int sb = 0; sb < N; sb++)
#pragma unroll
            for (int i = 0; i < 16; i++)
                mx = fmaxf(mx, s[sb][i]);
        mx = pair_max(mx) * sc;
        const bool move = mx > m_ref + kLazyP;
        if (__builtin_amdgcn_ballot_w64(move) != 0) {
            const float m_new = move ? mx : m_ref;
            const float alpha = move ? __builtin_amdgcn_exp2f(m_ref - m_new) : 1.f;
            m_ref = m_new;
            l_run *= alpha;
#pragma unroll
            for (int cb = 0; cb < D / 32; cb++)
                acc[cb] *= alpha;
        }
        const float mc = m_ref == kNegInf ? 0.f : m_ref;
        bf16x2 pw[N][8];
#pragma unroll
        for (int sb = 0; sb < N; sb++)
#pragma unroll
            for (int i = 0; i < 16; i += 2) {
                pw[sb][i >> 1] = cvt_bf16x2(__builtin_amdgcn_exp2f(fmaf(s[sb][i], sc, -mc)),
                                            __builtin_amdgcn_exp2f(fmaf(s[sb][i + 1], sc, -mc)));
                l_run = __builtin_amdgcn_fdot2_f32_bf16(pw[sb][i >> 1], ones, l_run, false);
            }
#pragma unroll
        for (int sb = 0; sb < N; sb++)
#pragma unroll
            for (int ss = 0; ss < 2; ss++) {
                bf16x8 pf;
#pragma unroll
                for (int j = 0; j < 4; j++) {
                    pf[2 * j] = pw[sb][ss * 4 + j][0];
                    pf[2 * j + 1] = pw[sb][ss * 4 + j][1];
                }
#pragma unroll
                for (int cb = 0; cb < D / 32; cb++) {
                    const bf16x8 vf = read_vt_frag(
                        &sm.v[buf][(sb0 + sb) * 32 + ss * 16 + vt_row][vt_scol[cb]], D);
                    acc[cb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, pf, acc[cb], 0, 0, 0);
                }
            }
    };

    int buf = 0;
    for (int key = k0; key < k1; key += kBlockN, buf ^= 1) {
        dma_wait_barrier();                      // this tile is in, the other buffer is read
        if (key + kBlockN < k1)
            stage(buf ^ 1, key + kBlockN);
        if (live) {
            if (wk == 1)
                step(std::integral_constant<int, 2>{}, buf, 0, key);
            else
                step(std::integral_constant<int, 1>{}, buf, kg, key);
        }
    }

    // The two key halves joined through LDS (the tiles are read).
    if (wk == 2) {
        float *other = (float *)&sm + rb * 64 * (D / 2 + 2) + lane;
        static_assert(sizeof(PrefixSmem<D>) >= 2 * 64 * (D / 2 + 2) * sizeof(float), "LDS");
        __syncthreads();
        if (live && kg == 1) {
#pragma unroll
            for (int cb = 0; cb < D / 32; cb++)
#pragma unroll
                for (int i = 0; i < 16; i++)
                    other[(cb * 16 + i) * 64] = acc[cb][i];
            other[D / 2 * 64] = m_ref;
            other[(D / 2 + 1) * 64] = l_run;
        }
        __syncthreads();
        if (!live || kg != 0)
            return;
        const float mo = other[D / 2 * 64], M = fmaxf(m_ref, mo);
        const float Mc = M == kNegInf ? 0.f : M;
        const float fa = __builtin_amdgcn_exp2f(m_ref - Mc), fb = __builtin_amdgcn_exp2f(mo - Mc);
#pragma unroll
        for (int cb = 0; cb < D / 32; cb++)
#pragma unroll
            for (int i = 0; i < 16; i++)
                acc[cb][i] = fmaf(acc[cb][i], fa, other[(cb * 16 + i) * 64] * fb);
        l_run = fmaf(l_run, fa, other[(D / 2 + 1) * 64] * fb);
        m_ref = M;
    }
    if (!live)
        return;
    const float l = pair_sum(l_run);
    if (!row_valid)
        return;
    const int64_t row = ((int64_t)(a.slot0[kind] + c) * a.num_seqs + b) * a.hq + head;
    float *op = a.part + row * D + 4 * g;
#pragma unroll
    for (int cb = 0; cb < D / 32; cb++)
#pragma unroll
        for (int q = 0; q < 4; q++)
            *(f32x4 *)(op + cb * 32 + q * 8) = f32x4{acc[cb][4 * q], acc[cb][4 * q + 1],
                                                     acc[cb][4 * q + 2], acc[cb][4 * q + 3]};
    if (g == 0)
        *(f32x2 *)(a.ml + 2 * row) = f32x2{m_ref, l};
}

// WPH waves per (sequence, head), four waves per workgroup; a wave's halves
// of D / 4 lanes take the chunks of a branch in turn.
template <int D, int WPH>
__global__ __launch_bounds__(256) void prefix_combine_kernel(const PrefixArgs a) {
    constexpr int kLanes = D / 4, kGroups = 64 / kLanes, kStreams = kGroups * WPH;
    constexpr int kMost = 2 * kMaxPrefixChunks;
    __shared__ float s_w[4][kMost];
    __shared__ __attribute__((aligned(16))) float s_o[2][4][D];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int e = lane % kLanes, st = (wave % WPH) * kGroups + lane / kLanes;
    const int64_t job = (int64_t)blockIdx.x * (4 / WPH) + wave / WPH;
    const int64_t rows = (int64_t)a.num_seqs * a.hq;
    if (WPH == 1 && job >= rows)
        return;                                   // whole wave: no barrier below
    const int b = (int)(job / a.hq), h = (int)(job % a.hq);
    // the sequence's prefix: largest r with cu_grp[r] <= b (of several equal
    // ones the last, the others' groups are empty)
    int r = 0;
    for (int hi = a.num_prefixes - 1; r < hi;) {
        const int mid = (r + hi + 1) >> 1;
        if (a.cu_grp[mid] <= b)
            r = mid;
        else
            hi = mid - 1;
    }
    const int P = a.cu_pre[r + 1] - a.cu_pre[r], S = a.cu[b + 1] - a.cu[b];
    const float p = a.gate[b];
    const bool sel = p > decode_threshold(a);

    // (m, l) of one branch and its unnormalised output: this stream's part of
    // it in A
    auto branch = [&](int kp, int ko, float &M, float &lsum) {
        // written chunks of the two ranges
        int first[2], n[2];
        const int kinds[2] = {kp, ko};
#pragma unroll
        for (int i = 0; i < 2; i++) {
            const int kind = kinds[i], len = i == 0 ? P : S;
            int lo, hi;
            key_range(a, kind, P, S, lo, hi);
            const int base = chunk_base(a, kind, len), kc = a.kc[kind];
            first[i] = lo < hi ? (lo - base) / kc : 0;
            const int end = lo < hi ? min((hi - base + kc - 1) / kc, a.chunks[kind]) : 0;
            n[i] = max(0, end - first[i]);
            first[i] += a.slot0[kind];
        }
        const int total = n[0] + n[1];
        auto row_of = [&](int j) {
            const int slot = j < n[0] ? first[0] + j : first[1] + j - n[0];
            return (int64_t)slot * rows + job;
        };
        M = kNegInf;
        float *w = s_w[wave];
        float lc[kMost / 64];
#pragma unroll
        for (int i = 0; i < kMost / 64; i++) {
            const int j = lane + 64 * i;
            lc[i] = 0.f;
            if (j < total) {
                const f32x2 v = *(const f32x2 *)(a.ml + 2 * row_of(j));
                w[j] = v[0];
                M = fmaxf(M, v[0]);
                lc[i] = v[1];
            }
        }
#pragma unroll
        for (int sh = 1; sh < 64; sh <<= 1)
            M = fmaxf(M, __shfl_xor(M, sh, 64));
        const float Mc = M == kNegInf ? 0.f : M;
        lsum = 0.f;
#pragma unroll
        for (int i = 0; i < kMost / 64; i++) {
            const int j = lane + 64 * i;
            if (j < total) {
                const float wc = __builtin_amdgcn_exp2f(w[j] - Mc);
                w[j] = wc;
                lsum = fmaf(wc, lc[i], lsum);
            }
        }
#pragma unroll
        for (int sh = 1; sh < 64; sh <<= 1)
            lsum += __shfl_xor(lsum, sh, 64);
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        f32x4 A = {};
#pragma unroll 4
        for (int j = st; j < total; j += kStreams) {
            const f32x4 v = *(const f32x4 *)(a.part + row_of(j) * D + 4 * e);
            const float wc = w[j];
#pragma unroll
            for (int i = 0; i < 4; i++)
                A[i] = fmaf(wc, v[i], A[i]);
        }
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");   // w is rewritten by the next branch
#pragma unroll
        for (int i = 0; i < 4; i++)
#pragma unroll
            for (int sh = kLanes; sh < 64; sh <<= 1)
                A[i] += __shfl_xor(A[i], sh, 64);
        return A;
    };
    float ml = kNegInf, ll = 0.f, mg = kNegInf, lg = 0.f;
    f32x4 ol = branch(kPfxLocal, kOwnLocal, ml, ll), og = {};
    if (sel)                                      // (every wave of the head)
        og = branch(kPfxGlobal, kOwnGlobal, mg, lg);
    if constexpr (WPH > 1) {
        if (lane < kLanes) {
            *(f32x4 *)&s_o[0][wave][4 * e] = ol;
            *(f32x4 *)&s_o[1][wave][4 * e] = og;
        }
        __syncthreads();
        ol = f32x4{};
        og = f32x4{};
#pragma unroll
        for (int i = 0; i < 4; i++) {
            ol += *(const f32x4 *)&s_o[0][i][4 * e];
            og += *(const f32x4 *)&s_o[1][i][4 * e];
        }
    }
    if (wave % WPH != 0 || lane >= kLanes)
        return;
    if (sel && a.share) {                         // the window's keys, attended to once
        const float M = fmaxf(ml, mg), Mc = M == kNegInf ? 0.f : M;
        const float fl = __builtin_amdgcn_exp2f(ml - Mc), fg = __builtin_amdgcn_exp2f(mg - Mc);
        lg = fmaf(ll, fl, lg * fg);
#pragma unroll
        for (int i = 0; i < 4; i++)
            og[i] = fmaf(ol[i], fl, og[i] * fg);
    }
    auto norm = [&](f32x4 o, float lsum, const float *gain) {
        const float inv = lsum > 0.f ? 1.f / lsum : 0.f;
        float ss = 0.f;
#pragma unroll
        for (int i = 0; i < 4; i++) {
            o[i] *= inv;
            ss = fmaf(o[i], o[i], ss);
        }
#pragma unroll
        for (int sh = 1; sh < kLanes; sh <<= 1)
            ss += __shfl_xor(ss, sh, 64);
        const float rn = 1.f / sqrtf(ss / (float)D + a.eps);
#pragma unroll
        for (int i = 0; i < 4; i++)
            o[i] *= rn * (gain ? gain[h * D + 4 * e + i] : 1.f);
        return o;
    };
    f32x4 o = norm(ol, ll, a.gain_local);
    if (sel) {
        const f32x4 n = norm(og, lg, a.gain_global);
#pragma unroll
        for (int i = 0; i < 4; i++)
            o[i] = (1.f - p) * o[i] + p * n[i];
    }
    *(u32x2 *)(a.out + job * D + 4 * e) = u32x2{pack_bf16x2(o[0], o[1]), pack_bf16x2(o[2], o[3])};
}

template <int D>
hipError_t launch_d(const PrefixArgs &a, hipStream_t s) {
    hipLaunchKernelGGL((prefix_attn_kernel<D>), dim3(a.first[4] + (a.act || a.n_act)),
                       dim3(kPrefixThreads), 0, s, a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess)
        return e;
    const int64_t jobs = (int64_t)a.num_seqs * a.hq;
    if (a.chunks[kPfxGlobal] + a.chunks[kOwnGlobal] > kWidePrefixMerge)
        hipLaunchKernelGGL((prefix_combine_kernel<D, 4>), dim3(jobs), dim3(256), 0, s, a);
    else
        hipLaunchKernelGGL((prefix_combine_kernel<D, 1>), dim3((jobs + 3) / 4), dim3(256), 0, s, a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_decode_prefix(const PrefixArgs &a, hipStream_t s) {
    return a.head_dim == 128 ? launch_d<128>(a, s) : launch_d<64>(a, s);
}

}  // namespace logo
