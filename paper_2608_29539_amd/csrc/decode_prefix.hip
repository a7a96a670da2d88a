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
//                          the heads of one sequence).  Four waves of 32 rows.
//   prefix_combine_kernel  joins the chunks of each (sequence, head), applies
//                          ContextNorm and the fusion, rounds once to bf16.
//
// The decoding step keeps P in fp32, and so does this one but for 2^-16 of it: P
// goes into the PV product as the sum of two bf16 numbers, two products per
// fragment of V.  One would halve those products (64 sequences behind 32K tokens,
// all selected: 76 us a step, 89 with two; 32 behind 16K, 4 selected: 47 both
// ways) but leave an error as large as the output's rounding.  Everything else
// is fp32.
//
// Bounds (32 / 8 heads, d = 128).  32 sequences behind 16K tokens, 4 selected:
// reading 171 MB, 31 us + 5.6 of merge (5.5 TB/s from the last-level cache).
// 64 behind 32K, all selected: a wave's chain per tile (fragment reads, the
// running max, exponentials, products of 256 and 512 cycles), 87 us + 7.5 for 36
// GFLOP (54 with both parts of P); 64-key tiles and deeper or shallower prefetch
// took the same time.  Small steps: the prologue (4 us of dependent loads) and the
// merge's.
#include "cache_internal.h"
#include "cache_tiles.h"
#include "decode_common.h"
#include "logo_internal.h"

#include <type_traits>

namespace logo {
namespace {

constexpr int kPfWaves = kPrefixThreads / 64;
constexpr float kLazyP = 8.f;               // exp2-domain headroom of the running max

// Over the lanes l, l ^ 16, l ^ 32 and l ^ 48.
__device__ __forceinline__ float quad_max(float x) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return pair_max(fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1])));
}
__device__ __forceinline__ float quad_sum(float x) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return pair_sum(__uint_as_float(r[0]) + __uint_as_float(r[1]));
}

// Over a row of 16 lanes and over the wave, in every lane (rotations and quad
// swaps in the vector unit).
template <int Ctrl>
__device__ __forceinline__ float dpp_f(float x) {
    return __int_as_float(
        __builtin_amdgcn_update_dpp(0, __float_as_int(x), Ctrl, 0xF, 0xF, false));
}
__device__ __forceinline__ float row_sum(float x) {
    x += dpp_f<0x128>(x);   // row_ror:8
    x += dpp_f<0x124>(x);   // row_ror:4
    x += dpp_f<0x4E>(x);    // quad_perm [2,3,0,1]
    x += dpp_f<0xB1>(x);    // quad_perm [1,0,3,2]
    return x;
}
__device__ __forceinline__ float wave_sum(float x) { return quad_sum(row_sum(x)); }
__device__ __forceinline__ float wave_maxf(float x) {
    x = fmaxf(x, dpp_f<0x128>(x));
    x = fmaxf(x, dpp_f<0x124>(x));
    x = fmaxf(x, dpp_f<0x4E>(x));
    x = fmaxf(x, dpp_f<0xB1>(x));
    return quad_max(x);
}

// Largest over the wave, in every lane.
template <int Ctrl>
__device__ __forceinline__ int dpp_max(int x) {
    return max(x, __builtin_amdgcn_update_dpp(x, x, Ctrl, 0xF, 0xF, false));
}
__device__ __forceinline__ int wave_max(int x) {
    x = dpp_max<0x128>(x);   // row_ror:8
    x = dpp_max<0x124>(x);   // row_ror:4
    x = dpp_max<0x4E>(x);    // quad_perm [2,3,0,1]
    x = dpp_max<0xB1>(x);    // quad_perm [1,0,3,2]
    const auto r = __builtin_amdgcn_permlane16_swap((uint32_t)x, (uint32_t)x, false, false);
    x = max((int)r[0], (int)r[1]);
    const auto q = __builtin_amdgcn_permlane32_swap((uint32_t)x, (uint32_t)x, false, false);
    return max((int)q[0], (int)q[1]);
}

// Kinds of key range (the order of the work items).
enum { kPfxGlobal = 0, kOwnGlobal = 1, kPfxLocal = 2, kOwnLocal = 3 };

// Two weights as bf16 parts, x = hi + lo to 2^-16 of its value.
__device__ __forceinline__ void split_bf16x2(float x, float y, bf16x2 &hi, bf16x2 &lo) {
    hi = cvt_bf16x2(x, y);
    lo = cvt_bf16x2(x - (float)hi[0], y - (float)hi[1]);
}

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

// Tiles of kPfKeys keys in kPfStages buffers, loaded kPfStages - 1 ahead: with
// two workgroups per CU at d = 128, 96 KB of K and V on their way per CU.
constexpr int kPfKeys = 32;
constexpr int kPfStages = 4;
template <int D>
struct alignas(16) PrefixSmem {
    uint16_t k[kPfStages][kPfKeys][D];           // pieces permuted (piece_swz)
    uint16_t v[kPfStages][kPfKeys][D];           // segments permuted (seg_swz)
};

template <int D>
__global__ __launch_bounds__(kPrefixThreads, 2) void prefix_attn_kernel(const PrefixArgs a) {
    __shared__ PrefixSmem<D> sm;
    __shared__ int s_seq[kPrefixRows], s_lo[kPrefixRows], s_hi[kPrefixRows], s_cnt[kPfWaves];
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
    int t = 0, pair = item;
    if (tiles > 1) {
        const int u = item / (kQueues * tiles), rem = item % (kQueues * tiles);
        t = rem / kQueues;
        pair = u * kQueues + rem % kQueues;
    }
    const int pk = pair / nch, c = pair % nch, kvh = pk % a.hkv, r = pk / a.hkv;
    if (r >= (own ? a.num_seqs : a.num_prefixes))
        return;
    // (all of them read before the first is looked at)
    const int32_t *cu = own ? a.cu : a.cu_pre;
    const int64_t base = cu[r];
    const int len = cu[r + 1] - (int)base;
    const int g0 = a.cu_grp[own ? 0 : r], g1 = a.cu_grp[own ? 1 : r + 1];
    const float thr = decode_threshold(a), gate_r = a.gate[own ? r : 0];
    if (own && global && !(gate_r > thr))
        return;                                  // an unselected token: window only

    // the chunk's keys [k0, k1) and the tile's rows: s_seq[i] for the
    // sequences of ranks rank0, rank0 + 1, ... among those that see the chunk
    int k0 = chunk_base(a, kind, len) + c * kc;
    int k1 = min(len, k0 + kc);
    if (k0 >= k1)
        return;
    if (own) {
        int lo, hi;
        key_range(a, kind, 0, len, lo, hi);
        k0 = max(k0, lo);
        k1 = min(k1, hi);
        if (k0 >= k1)
            return;
    }

    // K / V tiles: a wave's kLoads loads of each, whose lanes read whole rows
    constexpr int kPc = D / 8, kLoads = kPfKeys * kPc / 64 / kPfWaves;
    const uint16_t *kt = own ? (global ? a.k_g : a.k) : (global ? a.kp_g : a.kp);
    const uint16_t *vt = own ? (global ? a.v_g : a.v) : (global ? a.vp_g : a.vp);
    const int row_bytes = a.hkv * D * 2;
    kt += (base * a.hkv + kvh) * (int64_t)D;
    vt += (base * a.hkv + kvh) * (int64_t)D;
    // A lane's byte offset inside a tile for the 1 KB of LDS that load ld fills;
    // rows at or past k1 read as zeros (they are masked).
    auto k_off = [&](int ld) {
        const int row = (ld * 64 + lane) / kPc;
        return row * row_bytes + ((lane % kPc) ^ piece_swz<D>(row)) * 16;
    };
    auto v_off = [&](int ld) {
        const int row = (ld * 64 + lane) / kPc, c16 = lane % kPc;
        return row * row_bytes + (((c16 >> 2) ^ seg_swz<D>(row)) * 4 + (c16 & 3)) * 16;
    };
    auto tile_at = [&](const uint16_t *t, int key) {
        return raw_rsrc((const char *)t + (int64_t)key * row_bytes, min(kPfKeys, k1 - key) * row_bytes);
    };
    int koff[kLoads], voff[kLoads];
#pragma unroll
    for (int i = 0; i < kLoads; i++) {
        koff[i] = k_off(i * kPfWaves + wave);
        voff[i] = v_off(i * kPfWaves + wave);
    }
    auto stage = [&](int buf, int key) {
        const uint32_t kd = lds_addr_of(&sm.k[buf][0][0]), vd = lds_addr_of(&sm.v[buf][0][0]);
        const u32x4 kr = tile_at(kt, key), vr = tile_at(vt, key);
#pragma unroll
        for (int i = 0; i < kLoads; i++) {
            const int at = (i * kPfWaves + wave) * 1024;
            lds_load16_at(kr, kd + at, koff[i]);
            lds_load16_at(vr, vd + at, voff[i]);
        }
    };
    auto fill = [&]() {
#pragma unroll
        for (int i = 0; i < kPfStages; i++)
            if (k0 + i * kPfKeys < k1)
                stage(i, k0 + i * kPfKeys);
    };

    // The first tiles are on their way while the rows are listed (not for a
    // group's later row tiles, which may have none).
    if (t == 0)
        fill();
    const int rank0 = t * kPrefixRows / a.group;
    int count = 0;
    if (own) {
        count = 1;
    } else {
        const int most = (t * kPrefixRows + kPrefixRows - 1) / a.group - rank0 + 1;
        for (int c0 = g0; c0 < g1; c0 += kPrefixThreads) {
            const int b = c0 + tid;
            bool in = b < g1 && (!global || a.gate[b] > thr);
            int lo = 0, hi = 0;
            if (in) {
                key_range(a, kind, len, a.cu[b + 1] - a.cu[b], lo, hi);
                lo = max(lo, k0);
                hi = min(hi, k1);
                in = lo < hi;
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
            if (in && at >= 0 && at < most) {
                s_seq[at] = b;
                s_lo[at] = lo;
                s_hi[at] = hi;
            }
            __syncthreads();
        }
    }
    const int64_t left = (int64_t)count * a.group - (int64_t)t * kPrefixRows;
    if (left <= 0) {
        __builtin_amdgcn_s_waitcnt(kWaitVmcnt0);   // (no load may outlive the workgroup's LDS)
        return;
    }
    if (t != 0)
        fill();
    const int nrows = left < kPrefixRows ? (int)left : kPrefixRows;

    // Waves of 32 rows; with 16 rows or fewer (the heads of one sequence, a
    // small group) every wave has all of them, and tiles of its own.
    const bool few = nrows <= 16;
    const int first_row = few ? 0 : wave * 32, lr = few ? lane & 15 : m;
    const bool live = first_row < nrows;
    // this lane's query row; rows past the last repeat it and are not stored
    const int ri = min(first_row + lr, nrows - 1);
    const bool row_valid = first_row + lr < nrows;
    const int flat = t * kPrefixRows + ri, rank = flat / a.group - rank0;
    const int b = own ? r : s_seq[rank];
    const int lo = own ? k0 : s_lo[rank], hi = own ? k1 : s_hi[rank];
    const int head = kvh * a.group + flat % a.group;
    const uint16_t *qp = (global ? a.q_g : a.q) + ((int64_t)b * a.hq + head) * D;
    // keys that every row of the wave sees: tiles inside need no mask
    const int all_lo = uni(wave_max(lo)), all_hi = -uni(wave_max(-hi));
    const float sc = a.scale_log2;
    const int64_t prow = ((int64_t)(a.slot0[kind] + c) * a.num_seqs + b) * a.hq + head;
    float m_ref = kNegInf, l_run = 0.f;
    // the running max of a tile's scores moves (rescaling O and l) when it is
    // exceeded by kLazyP; returns what the exponents subtract
    auto rescale = [&](float mx, auto &acc) {
        const bool move = mx > m_ref + kLazyP;
        if (__builtin_amdgcn_ballot_w64(move) != 0) {
            const float m_new = move ? mx : m_ref;
            const float alpha = move ? __builtin_amdgcn_exp2f(m_ref - m_new) : 1.f;
            m_ref = m_new;
            l_run *= alpha;
            for (auto &x : acc)
                x *= alpha;
        }
        return m_ref == kNegInf ? 0.f : m_ref;
    };
    constexpr int kAhead = kPfStages - 1;

    if (few) {
        // Wave w has tiles w, w + 4, ... in stage w of its own, which it reads
        // into registers whole and fills again before it multiplies: no
        // barriers, and the four waves' chains cover each other.  O^T = V^T P^T
        // in blocks of 16 d values; lane (row lr, kg): keys 4 kg + 0..3 of the
        // tile's halves, the product's order of keys.
        static_assert(kPfStages == kPfWaves, "a stage per wave");
        const int kg = lane >> 4;
        bf16x8 qf[D / 32];
#pragma unroll
        for (int x = 0; x < D / 32; x++)
            qf[x] = *(const bf16x8 *)(qp + x * 32 + kg * 8);
        const int vt_row = 4 * kg + ((lane & 15) >> 2), vt_col = 4 * (lane & 3);
        f32x4 acc[D / 16];
#pragma unroll
        for (int x = 0; x < D / 16; x++)
            acc[x] = f32x4{};
        // the wave's whole tile at `key`
        const uint32_t kd = lds_addr_of(&sm.k[wave][0][0]), vd = lds_addr_of(&sm.v[wave][0][0]);
        auto stage_own = [&](int key) {
            const u32x4 kr = tile_at(kt, key), vr = tile_at(vt, key);
#pragma unroll
            for (int ld = 0; ld < kPfKeys * kPc / 64; ld++) {
                lds_load16_at(kr, kd + ld * 1024, k_off(ld));
                lds_load16_at(vr, vd + ld * 1024, v_off(ld));
            }
        };
        dma_wait_barrier();                      // the first four tiles, the queries
#pragma unroll 1
        for (int key = k0 + wave * kPfKeys; key < k1; key += kPfWaves * kPfKeys) {
            __builtin_amdgcn_s_waitcnt(kWaitVmcnt0);
            asm volatile("" ::: "memory");
            bf16x8 kf[2][D / 32], vf[D / 16];
#pragma unroll
            for (int x = 0; x < D / 32; x++)
#pragma unroll
                for (int h = 0; h < 2; h++) {
                    const int row = h * 16 + lr;
                    kf[h][x] =
                        *(const bf16x8 *)&sm.k[wave][row][((x * 4 + kg) ^ piece_swz<D>(row)) * 8];
                }
#pragma unroll
            for (int x = 0; x < D / 16; x++) {
                const uint16_t *vr = &sm.v[wave][vt_row][((x / 2) ^ seg_swz<D>(vt_row)) * 32 +
                                                         (x % 2) * 16 + vt_col];
                vf[x] = lds_tr_pair(vr, vr + 16 * D);
            }
            // the stage is read before it is filled again
            __builtin_amdgcn_s_waitcnt(kWaitLgkmcnt0);
            asm volatile("" ::: "memory");
            if (key + kPfWaves * kPfKeys < k1)
                stage_own(key + kPfWaves * kPfKeys);
            f32x4 s[2] = {};
#pragma unroll
            for (int x = 0; x < D / 32; x++)
#pragma unroll
                for (int h = 0; h < 2; h++)
                    s[h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[h][x], qf[x], s[h], 0, 0, 0);
            if (key < all_lo || key + kPfKeys > all_hi) {
#pragma unroll
                for (int h = 0; h < 2; h++)
#pragma unroll
                    for (int i = 0; i < 4; i++) {
                        const int j = key + h * 16 + kg * 4 + i;
                        if (j < lo || j >= hi)
                            s[h][i] = kNegInf;
                    }
            }
            float mx = max2(max2(max2(s[0][0], s[0][1]), max2(s[0][2], s[0][3])),
                            max2(max2(s[1][0], s[1][1]), max2(s[1][2], s[1][3])));
            mx = quad_max(mx) * sc;
            const float mc = rescale(mx, acc);
            bf16x8 pf[2];                            // the weights' upper and lower parts
            float l2[2] = {};
#pragma unroll
            for (int h = 0; h < 2; h++)
#pragma unroll
                for (int i = 0; i < 4; i += 2) {
                    const float x = __builtin_amdgcn_exp2f(fmaf(s[h][i], sc, -mc));
                    const float y = __builtin_amdgcn_exp2f(fmaf(s[h][i + 1], sc, -mc));
                    bf16x2 p[2];
                    split_bf16x2(x, y, p[0], p[1]);
                    l2[i >> 1] += x + y;
#pragma unroll
                    for (int u = 0; u < 2; u++) {
                        pf[u][h * 4 + i] = p[u][0];
                        pf[u][h * 4 + i + 1] = p[u][1];
                    }
                }
            l_run += l2[0] + l2[1];
#pragma unroll
            for (int u = 0; u < 2; u++)
#pragma unroll
                for (int x = 0; x < D / 16; x++)
                    acc[x] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf[x], pf[u], acc[x], 0, 0, 0);
        }
        // The waves' (O, m, l) joined through LDS (the stages are read): wave w
        // takes its quarter of the blocks.
        constexpr int kVals = D / 4 + 2;         // floats per lane and wave
        static_assert(sizeof(PrefixSmem<D>) >= kPfWaves * 64 * kVals * sizeof(float), "LDS");
        float *mine = (float *)&sm + wave * 64 * kVals + lane;
        const float lw = quad_sum(l_run);
        __syncthreads();
#pragma unroll
        for (int x = 0; x < D / 16; x++)
#pragma unroll
            for (int i = 0; i < 4; i++)
                mine[(x * 4 + i) * 64] = acc[x][i];
        mine[D / 4 * 64] = m_ref;
        mine[(D / 4 + 1) * 64] = lw;
        __syncthreads();
        const float *all = (const float *)&sm + lane;
        float M = kNegInf, f[kPfWaves], l = 0.f;
#pragma unroll
        for (int w = 0; w < kPfWaves; w++) {
            f[w] = all[(w * kVals + D / 4) * 64];
            M = fmaxf(M, f[w]);
        }
        const float Mc = M == kNegInf ? 0.f : M;
#pragma unroll
        for (int w = 0; w < kPfWaves; w++) {
            f[w] = __builtin_amdgcn_exp2f(f[w] - Mc);
            l = fmaf(f[w], all[(w * kVals + D / 4 + 1) * 64], l);
        }
        constexpr int kOwn = D / 16 / kPfWaves;
#pragma unroll
        for (int x = 0; x < kOwn; x++) {
            f32x4 o = {};
#pragma unroll
            for (int w = 0; w < kPfWaves; w++)
#pragma unroll
                for (int i = 0; i < 4; i++)
                    o[i] = fmaf(f[w], all[(w * kVals + (wave * kOwn + x) * 4 + i) * 64], o[i]);
            if (row_valid)
                *(f32x4 *)(a.part + prow * D + (wave * kOwn + x) * 16 + 4 * kg) = o;
        }
        if (row_valid && kg == 0 && wave == 0)
            *(f32x2 *)(a.ml + 2 * prow) = f32x2{M, l};
        return;
    }

    bf16x8 qf[D / 16];
#pragma unroll
    for (int s = 0; s < D / 16; s++)
        qf[s] = *(const bf16x8 *)(qp + g * 8 + s * 16);
    const int vt_row = 4 * g + ((lane & 15) >> 2);
    const int vt_col = 16 * ((lane >> 4) & 1) + 4 * (lane & 3);
    int vt_scol[D / 32];
#pragma unroll
    for (int cb = 0; cb < D / 32; cb++)
        vt_scol[cb] = (cb ^ seg_swz<D>(vt_row)) * 32 + vt_col;
    f32x16 acc[D / 32];
#pragma unroll
    for (int cb = 0; cb < D / 32; cb++)
        acc[cb] = f32x16{};

    constexpr int kHalf = D / 32;
    auto k_frags = [&](int buf, int ss0, bf16x8 (&kf)[kHalf]) {
#pragma unroll
        for (int i = 0; i < kHalf; i++)
            kf[i] = *(const bf16x8 *)&sm.k[buf][m][(((ss0 + i) * 2 + g) ^ piece_swz<D>(m)) * 8];
    };
    auto v_frags = [&](int buf, int ss, bf16x8 (&vf)[D / 32]) {
#pragma unroll
        for (int cb = 0; cb < D / 32; cb++)
            vf[cb] = lds_tr_pair(&sm.v[buf][ss * 16 + vt_row][vt_scol[cb]],
                                 &sm.v[buf][ss * 16 + vt_row + 8][vt_scol[cb]]);
    };
    auto scores = [&](f32x16 s, int ss0, const bf16x8 (&kf)[kHalf]) {
#pragma unroll
        for (int i = 0; i < kHalf; i++)
            s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[i], qf[ss0 + i], s, 0, 0, 0);
        return s;
    };
    // Tile `buf` with its scores s; on return s has the next tile's scores,
    // whose products are issued between this one's exponentials (past the last
    // tile they are not used).  Fragments are read half a tile ahead of the
    // products that take them.
    auto step = [&](int buf, int key0, f32x16 &s) {
        const int nbuf = (buf + 1) % kPfStages;
        bf16x8 kf[2][kHalf], vf[2][D / 32];
        k_frags(nbuf, 0, kf[0]);
        __builtin_amdgcn_sched_barrier(0);
        if (key0 < all_lo || key0 + kPfKeys > all_hi) {
#pragma unroll
            for (int i = 0; i < 16; i++) {
                const int key = key0 + (i >> 2) * 8 + g * 4 + (i & 3);
                if (key < lo || key >= hi)
                    s[i] = kNegInf;
            }
        }
        float mx[4];
#pragma unroll
        for (int i = 0; i < 4; i++)
            mx[i] = max2(max2(s[i], s[i + 4]), max2(s[i + 8], s[i + 12]));
        const float top = pair_max(max2(max2(mx[0], mx[1]), max2(mx[2], mx[3]))) * sc;
        const float mc = rescale(top, acc);
        k_frags(nbuf, kHalf, kf[1]);
        v_frags(buf, 0, vf[0]);
        __builtin_amdgcn_sched_barrier(0);
        f32x16 next = scores(f32x16{}, 0, kf[0]);
        bf16x2 pw[2][8];                         // the weights' upper and lower parts
        float l2[2] = {};
        auto exps = [&](int i0) {
#pragma unroll
            for (int i = i0; i < i0 + 8; i += 2) {
                const float x = __builtin_amdgcn_exp2f(fmaf(s[i], sc, -mc));
                const float y = __builtin_amdgcn_exp2f(fmaf(s[i + 1], sc, -mc));
                split_bf16x2(x, y, pw[0][i >> 1], pw[1][i >> 1]);
                l2[(i >> 1) & 1] += x + y;
            }
        };
        exps(0);
        v_frags(buf, 1, vf[1]);
        __builtin_amdgcn_sched_barrier(0);
        next = scores(next, kHalf, kf[1]);
        exps(8);
        l_run += l2[0] + l2[1];
#pragma unroll
        for (int ss = 0; ss < 2; ss++)
#pragma unroll
            for (int u = 0; u < 2; u++) {
                bf16x8 pf;
#pragma unroll
                for (int j = 0; j < 4; j++) {
                    pf[2 * j] = pw[u][ss * 4 + j][0];
                    pf[2 * j + 1] = pw[u][ss * 4 + j][1];
                }
#pragma unroll
                for (int cb = 0; cb < D / 32; cb++)
                    acc[cb] =
                        __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[ss][cb], pf, acc[cb], 0, 0, 0);
            }
        s = next;
    };

    // (the queries are in before the loop, whose waits count the tiles' loads
    // alone; the first tiles with them)
    dma_wait_barrier();
    f32x16 s = {};
    if (live) {
        bf16x8 kf[kHalf];
        k_frags(0, 0, kf);
        s = scores(s, 0, kf);
        k_frags(0, kHalf, kf);
        s = scores(s, kHalf, kf);
    }
    int buf = 0;
    for (int key = k0; key < k1; key += kPfKeys, buf = (buf + 1) % kPfStages) {
        // the next tile is in, and the buffer of the one before this is read
        if (key + (kAhead - 1) * kPfKeys < k1)
            dma_wait_barrier_but<(kAhead - 2) * 2 * kLoads>();
        else
            dma_wait_barrier();
        if (key > k0 && key + kAhead * kPfKeys < k1)
            stage((buf + kAhead) % kPfStages, key + kAhead * kPfKeys);
        if (live)
            step(buf, key, s);
    }

    if (!live)
        return;
    const float l = pair_sum(l_run);
    if (!row_valid)
        return;
    float *op = a.part + prow * D + 4 * g;
#pragma unroll
    for (int cb = 0; cb < D / 32; cb++)
#pragma unroll
        for (int q = 0; q < 4; q++)
            *(f32x4 *)(op + cb * 32 + q * 8) = f32x4{acc[cb][4 * q], acc[cb][4 * q + 1],
                                                     acc[cb][4 * q + 2], acc[cb][4 * q + 3]};
    if (g == 0)
        *(f32x2 *)(a.ml + 2 * prow) = f32x2{m_ref, l};
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

    // One branch's written chunks: begin() issues the loads of their (m, l) and
    // of the stream's first kPre parts, finish() weights and adds them.
    constexpr int kPre = 4;
    struct Branch {
        int first[2], n[2], total;               // slots of the two ranges
        f32x2 ml[kMost / 64];
        f32x4 pre[kPre];
    };
    auto row_of = [&](const Branch &x, int j) {
        const int slot = j < x.n[0] ? x.first[0] + j : x.first[1] + j - x.n[0];
        return (int64_t)slot * rows + job;
    };
    auto begin = [&](int kp, int ko, Branch &x) {
        const int kinds[2] = {kp, ko};
#pragma unroll
        for (int i = 0; i < 2; i++) {
            const int kind = kinds[i], len = i == 0 ? P : S;
            int lo, hi;
            key_range(a, kind, P, S, lo, hi);
            const int base = chunk_base(a, kind, len), kc = a.kc[kind];
            const int c0 = lo < hi ? (lo - base) / kc : 0;
            const int end = lo < hi ? min((hi - base + kc - 1) / kc, a.chunks[kind]) : 0;
            x.n[i] = max(0, end - c0);
            x.first[i] = a.slot0[kind] + c0;
        }
        x.total = x.n[0] + x.n[1];
#pragma unroll
        for (int i = 0; i < kMost / 64; i++) {
            const int j = lane + 64 * i;
            x.ml[i] = j < x.total ? *(const f32x2 *)(a.ml + 2 * row_of(x, j)) : f32x2{kNegInf, 0.f};
        }
#pragma unroll
        for (int u = 0; u < kPre; u++) {
            const int j = st + u * kStreams;
            x.pre[u] = j < x.total ? *(const f32x4 *)(a.part + row_of(x, j) * D + 4 * e) : f32x4{};
        }
    };
    auto finish = [&](const Branch &x, float &M, float &lsum) {
        M = kNegInf;
#pragma unroll
        for (int i = 0; i < kMost / 64; i++)
            M = fmaxf(M, x.ml[i][0]);
        M = wave_maxf(M);
        const float Mc = M == kNegInf ? 0.f : M;
        float *w = s_w[wave];
        lsum = 0.f;
#pragma unroll
        for (int i = 0; i < kMost / 64; i++) {
            const float wc = __builtin_amdgcn_exp2f(x.ml[i][0] - Mc);
            w[lane + 64 * i] = wc;
            lsum = fmaf(wc, x.ml[i][1], lsum);
        }
        lsum = wave_sum(lsum);
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        f32x4 A = {};
        auto add = [&](float wc, const f32x4 v) {
#pragma unroll
            for (int i = 0; i < 4; i++)
                A[i] = fmaf(wc, v[i], A[i]);
        };
#pragma unroll
        for (int u = 0; u < kPre; u++)           // (past the last chunk: weight and part 0)
            if (st + u * kStreams < kMost)
                add(w[st + u * kStreams], x.pre[u]);
#pragma unroll 4
        for (int j = st + kPre * kStreams; j < x.total; j += kStreams)
            add(w[j], *(const f32x4 *)(a.part + row_of(x, j) * D + 4 * e));
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");   // w is rewritten by the next branch
#pragma unroll
        for (int i = 0; i < 4; i++)              // the wave's groups of lanes
            A[i] = D == 128 ? pair_sum(A[i]) : quad_sum(A[i]);
        return A;
    };
    Branch local, global;
    begin(kPfxLocal, kOwnLocal, local);
    if (sel)                                      // (every wave of the head)
        begin(kPfxGlobal, kOwnGlobal, global);
    float ml = kNegInf, ll = 0.f, mg = kNegInf, lg = 0.f;
    f32x4 ol = finish(local, ml, ll), og = {};
    if (sel)
        og = finish(global, mg, lg);
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
        ss = row_sum(ss);
        if (D == 128)                            // (32 lanes: two rows)
            ss += __shfl_xor(ss, 16, 64);
        // (a sequence without rows: zeros, also where eps is zero)
        const float rn = lsum == 0.f ? 0.f : 1.f / sqrtf(ss / (float)D + a.eps);
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
    // (no work item where no cache has any row: the merge writes the zeros)
    const int items = a.first[4] + (a.act || a.n_act);
    if (items > 0) {
        hipLaunchKernelGGL((prefix_attn_kernel<D>), dim3(items), dim3(kPrefixThreads), 0, s, a);
        hipError_t e = hipGetLastError();
        if (e != hipSuccess)
            return e;
    }
    const int64_t jobs = (int64_t)a.num_seqs * a.hq;
    // four waves per head where a head has many chunks and the heads alone do
    // not fill the card (64 sequences of 32 heads behind 32K tokens, 2048 heads:
    // the step 78.5 us with four, 76.7 with one)
    if (a.chunks[kPfxGlobal] + a.chunks[kOwnGlobal] > kWidePrefixMerge && jobs <= 1024)
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
