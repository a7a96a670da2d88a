// cache_evict.hip -- caches cut down to a budget of rows per sequence and KV
// head by the attention weight that each row has received.
//
// Of L rows n = min(L, budget) are kept: the last min(recent, n), and of the
// others the k with the largest scores (a NaN is the lowest, -0 equals +0, ties
// go to the lowest index), in ascending order.
//
// The k-th largest is found by radix selection on order-preserving 32-bit keys
// (11, 11 and 10 bits), and the rows above it and the first ones equal to it
// get their places by counting.  A workgroup has 8192 rows in registers.
//
//   evict_select_kernel  caches of up to 8192 rows: one workgroup per (sequence,
//                        KV head) does it all, with the histograms in LDS (up
//                        to 2048 rows of 256 threads, whose barriers and scans
//                        are shorter: 4 caches of 2048 rows 7.4 us, 10.1 with
//                        1024; a call that is waited for 27.8 and 30.5 us, one
//                        among others 13.1-13.5 with both: its enqueuing)
//   evict_hist_kernel    longer ones: a launch per digit, in which every part
//                        of 8192 rows adds up all parts' last histograms, picks
//                        the bin of the k-th and counts the next digit
//   evict_rank_kernel    picks the last digit and places its part's rows, the
//                        counts of the parts before it added up
//   evict_copy_kernel    copies the kept rows of K and V
//
// 4 heads of 131071 rows, an eighth kept: 27 us of selection (bound by the four
// launches' chains; one workgroup per head took 205) and 11 of copying; 128 of
// 32768: 44 and 101 us (5.3 TB/s read and written).
#include "attn_common.h"
#include "cache_internal.h"

namespace logo {
namespace {

constexpr int kEvPer = kEvPartRows / kEvThreads;           // rows per thread
constexpr int kEvBins = 2048;

// Order-preserving key of a score: a larger score has a larger key, NaN 0.
__device__ __forceinline__ uint32_t score_key(float x) {
    if (x != x)
        return 0;
    const uint32_t u = __float_as_uint(x + 0.f);          // -0 -> +0
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// Inclusive prefix over the wave's lanes, in the vector unit: lanes 1, 2, 4 and
// 8 to the left within rows of 16, then the last lanes of the rows before.
template <int Ctrl, int RowMask>
__device__ __forceinline__ uint32_t dpp_u(uint32_t x) {
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, Ctrl, RowMask, 0xF, false);
}
__device__ __forceinline__ uint32_t wave_scan(uint32_t x) {
    x += dpp_u<0x111, 0xF>(x);   // row_shr:1
    x += dpp_u<0x112, 0xF>(x);
    x += dpp_u<0x114, 0xF>(x);
    x += dpp_u<0x118, 0xF>(x);
    x += dpp_u<0x142, 0xA>(x);   // row_bcast:15 into rows 1 and 3
    x += dpp_u<0x143, 0xC>(x);   // row_bcast:31 into rows 2 and 3
    return x;
}

// What the waves exchange: sums of theirs in turn in two places, so that a
// scan needs one barrier (two scans later every wave has read the first).
template <int NT>
struct WaveSums {
    static constexpr int kWaves = NT / 64;
    uint32_t (*part)[kWaves];                            // [2] in LDS
    int at = 0;
    // (sum over the waves before this one, over all of them) of a value that
    // lane 63 of each wave gives
    __device__ __forceinline__ uint32_t exchange(uint32_t v, uint32_t &total) {
        const int wave = threadIdx.x >> 6;
        uint32_t *p = part[at];
        at ^= 1;
        if ((threadIdx.x & 63) == 63)
            p[wave] = v;
        __syncthreads();
        uint32_t before = 0;
        total = 0;
#pragma unroll
        for (int i = 0; i < kWaves; i++) {
            const uint32_t x = p[i];
            before += i < wave ? x : 0;
            total += x;
        }
        return before;
    }
    // exclusive prefix of v over the workgroup, and the total
    __device__ __forceinline__ uint32_t scan(uint32_t v, uint32_t &total) {
        const uint32_t incl = wave_scan(v);
        return exchange(incl, total) + incl - v;
    }
};

// One (sequence, KV head): n rows stay of L, k of the first `old` by score.
struct Choice {
    int b, h, base, L, n, rec, k, old;
    const float *score;
    __device__ __forceinline__ Choice(const EvictArgs &a, int problem) {
        b = problem / a.hkv;
        h = problem % a.hkv;
        base = a.cu[b];
        L = a.cu[b + 1] - base;
        n = min(L, a.budget);
        rec = min(a.recent, n);
        k = n - rec;
        old = L - rec;
        score = a.score + (int64_t)h * a.n + base;
    }
    __device__ __forceinline__ bool by_score() const { return k > 0 && k < old; }
};

// A part's rows in registers, each wave 512 consecutive ones: row
// part * kEvPartRows + wave * 512 + j * 64 + lane.
struct Rows {
    float x[kEvPer];
    int first, old;
    __device__ __forceinline__ int row(int j) const { return first + j * 64; }
    __device__ __forceinline__ bool in(int j) const { return row(j) < old; }
    __device__ __forceinline__ Rows(const Choice &c, int part) {
        first = part * kEvPartRows + (threadIdx.x >> 6) * (64 * kEvPer) + (threadIdx.x & 63);
        old = c.old;
#pragma unroll
        for (int j = 0; j < kEvPer; j++)
            x[j] = in(j) ? c.score[row(j)] : 0.f;
    }
};

// The digits found so far: keys that agree with `prefix` under `mask`, `left`
// of them (the largest) stay.
struct Digits {
    uint32_t prefix = 0, mask = 0, left = 0;
    __device__ __forceinline__ static int shift(int level) { return level == 0 ? 21 : level == 1 ? 10 : 0; }
    __device__ __forceinline__ static uint32_t width(int level) { return level == 2 ? 1023 : 2047; }
    __device__ __forceinline__ void take(int level, uint32_t bin, uint32_t in_bin) {
        prefix |= bin << shift(level);
        mask |= width(level) << shift(level);
        left = in_bin;
    }
};

// Histogram of digit `level` of the rows that agree with the digits so far.
template <int NT>
__device__ __forceinline__ void count_digit(const Rows &r, const Digits &d, int level,
                                            uint32_t *s_hist) {
    for (int i = threadIdx.x; i < kEvBins; i += NT)
        s_hist[i] = 0;
    __syncthreads();
#pragma unroll
    for (int j = 0; j < kEvPer; j++) {
        const uint32_t key = score_key(r.x[j]);
        if (r.in(j) && (key & d.mask) == d.prefix)
            atomicAdd(&s_hist[(key >> Digits::shift(level)) & Digits::width(level)], 1u);
    }
    __syncthreads();
}

// The bin in which the `left`-th largest lies, from this thread's bins (c[i]:
// bin 2047 - N tid - i); s_pick: the bin and how many of it stay.
template <int NT, int N>
__device__ __forceinline__ void pick_bin(const uint32_t (&c)[N], uint32_t left, WaveSums<NT> &sums,
                                         uint32_t *s_pick) {
    static_assert(N * NT == kEvBins, "every bin has a thread");
    uint32_t mine = 0, total;
#pragma unroll
    for (int i = 0; i < N; i++)
        mine += c[i];
    uint32_t above = sums.scan(mine, total);
#pragma unroll
    for (int i = 0; i < N; i++) {
        if (above < left && left <= above + c[i]) {
            s_pick[0] = kEvBins - 1 - N * threadIdx.x - i;
            s_pick[1] = left - above;
        }
        above += c[i];
    }
    __syncthreads();
}

// Places of a part's rows: all of them, or those above the pivot and the
// first `need` equal to it; gt0, eq0: such rows before the part.  The masks of
// 64 rows stay in scalar registers between the count and the placing.
template <int NT>
__device__ __forceinline__ void place(const EvictArgs &a, const Choice &c, const Rows &r, bool all,
                                      uint32_t pivot, uint32_t need, uint32_t gt0, uint32_t eq0,
                                      uint32_t off, WaveSums<NT> &sums) {
    uint64_t gm[kEvPer], em[kEvPer];
    uint32_t gt = 0, eq = 0;                               // of this wave
    const int left = c.old - uni(r.first);                 // (lane 0's row)
#pragma unroll
    for (int j = 0; j < kEvPer; j++) {
        const int n = left - j * 64;
        const uint64_t real = n >= 64 ? ~0ull : n > 0 ? (1ull << n) - 1 : 0ull;
        const uint32_t key = score_key(r.x[j]);
        gm[j] = real & (all ? ~0ull : __ballot(key > pivot));
        em[j] = real & (all ? 0ull : __ballot(key == pivot));
        gt += (uint32_t)__popcll(gm[j]);
        eq += (uint32_t)__popcll(em[j]);
    }
    uint32_t total;
    const uint32_t ex = uni(sums.exchange(gt | eq << 16, total));
    gt0 = uni(gt0) + (ex & 0xFFFFu);
    eq0 = uni(eq0) + (ex >> 16);
    const int room = a.cap - (int)off;                     // (n, for a capacity as documented)
    int32_t *idx = a.keep_idx + (int64_t)c.h * a.cap + off;
    float *sc = a.score_out + (int64_t)c.h * a.cap + off;
    auto lower = [](uint64_t mask) {                       // bits below this lane
        return __builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32),
                                         __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0));
    };
    const uint64_t me = 1ull << (threadIdx.x & 63);
#pragma unroll
    for (int j = 0; j < kEvPer; j++) {
        const uint32_t eb = eq0 + lower(em[j]);
        const uint32_t at = gt0 + lower(gm[j]) + min(eb, need);
        if (((gm[j] & me) || ((em[j] & me) && eb < need)) && (int)at < room) {
            idx[at] = c.base + r.row(j);
            sc[at] = r.x[j];
        }
        gt0 += (uint32_t)__popcll(gm[j]);
        eq0 += (uint32_t)__popcll(em[j]);
    }
}

// Rows that the sequences before this one keep; cu_keep; the newest rows, of
// which workgroup `part` of `parts` places its share.
template <int NT>
__device__ __forceinline__ uint32_t place_recent(const EvictArgs &a, const Choice &c, int part,
                                                 int parts) {
    const int tid = threadIdx.x;
    uint32_t mine = 0;                                     // (every wave adds them up itself)
    for (int i = tid & 63; i < c.b; i += 64)
        mine += min(a.cu[i + 1] - a.cu[i], a.budget);
    const uint32_t off = __builtin_amdgcn_readlane(wave_scan(mine), 63);
    if (c.h == 0 && part == 0 && tid == 0) {
        if (c.b == 0)
            a.cu_keep[0] = 0;
        a.cu_keep[c.b + 1] = (int)off + c.n;
    }
    const int64_t out = (int64_t)c.h * a.cap + off + c.k;
    const int room = a.cap - (int)off - c.k;
    // (unsigned: a step past the end may pass 2^31)
    const uint32_t end = max(0, min(c.rec, room));
    for (uint32_t i = part * NT + tid; i < end; i += parts * NT) {
        a.keep_idx[out + i] = c.base + c.old + (int)i;
        a.score_out[out + i] = c.score[c.old + i];
    }
    return off;
}

template <int NT>
__global__ __launch_bounds__(NT) void evict_select_kernel(const EvictArgs a) {
    constexpr int N = kEvBins / NT;
    __shared__ uint32_t s_hist[kEvBins], s_part[2][NT / 64], s_pick[2];
    const int tid = threadIdx.x;
    WaveSums<NT> sums{s_part};
    const Choice c(a, blockIdx.x);
    const Rows r(c, 0);
    const uint32_t off = place_recent<NT>(a, c, 0, 1);
    Digits d;
    d.left = c.k;
    if (c.by_score()) {
#pragma unroll 1
        for (int level = 0; level < 3; level++) {
            count_digit<NT>(r, d, level, s_hist);
            uint32_t bins[N];
#pragma unroll
            for (int i = 0; i < N; i++)
                bins[i] = s_hist[kEvBins - 1 - N * tid - i];
            pick_bin<NT, N>(bins, d.left, sums, s_pick);
            d.take(level, s_pick[0], s_pick[1]);
        }
    }
    if (c.k > 0)
        place<NT>(a, c, r, c.k == c.old, d.prefix, d.left, 0, 0, off, sums);
}

// Two 16-bit bins per word: word 1023 - t holds thread t's bins.
__device__ __forceinline__ uint32_t *hist_of(const EvictArgs &a, int level, int problem, int part) {
    return a.hist + (((int64_t)(level & 1) * a.num_seqs * a.hkv + problem) * a.parts + part) *
                        (kEvBins / 2);
}
// This thread's bins over all parts with rows by score, and over those before
// `part`.
struct Bins {
    uint32_t sum[2] = {0, 0}, before0 = 0, before1 = 0;
    __device__ __forceinline__ Bins(const EvictArgs &a, const Choice &c, int level, int problem,
                                    int part) {
        const int n = (c.old + kEvPartRows - 1) / kEvPartRows;
        const uint32_t *w = hist_of(a, level, problem, 0) + (kEvBins / 2 - 1 - threadIdx.x);
#pragma unroll 8
        for (int i = 0; i < n; i++) {
            const uint32_t v = w[(int64_t)i * (kEvBins / 2)];
            sum[0] += v >> 16;
            sum[1] += v & 0xFFFFu;
            before0 += i < part ? v >> 16 : 0u;
            before1 += i < part ? v & 0xFFFFu : 0u;
        }
    }
};

// LEVEL 0, 1, 2: the digits before it are picked (the last from the
// histograms, an earlier one as part 0 of its launch wrote it), the part's
// rows above the last pick are counted, and its digit LEVEL.
template <int LEVEL>
__global__ __launch_bounds__(kEvThreads) void evict_hist_kernel(const EvictArgs a) {
    __shared__ uint32_t s_hist[kEvBins], s_part[2][kEvThreads / 64], s_pick[2];
    const int tid = threadIdx.x;
    WaveSums<kEvThreads> sums{s_part};
    const int problem = blockIdx.x / a.parts, part = blockIdx.x % a.parts;
    const Choice c(a, problem);
    if (!c.by_score() || (int64_t)part * kEvPartRows >= c.old)
        return;
    const Rows r(c, part);
    Digits d;
    d.left = c.k;
    if constexpr (LEVEL == 2)
        d.take(0, a.picks[problem * 2], a.picks[problem * 2 + 1]);
    if constexpr (LEVEL > 0) {
        const Bins w(a, c, LEVEL - 1, problem, part);
        pick_bin<kEvThreads, 2>(w.sum, d.left, sums, s_pick);
        if (LEVEL == 1 && part == 0 && tid < 2)
            a.picks[problem * 2 + tid] = s_pick[tid];
        const Digits last = d;
        d.take(LEVEL - 1, s_pick[0], s_pick[1]);
        // the part's rows above it
        uint32_t gt = 0, total;
#pragma unroll
        for (int j = 0; j < kEvPer; j++) {
            const uint32_t key = score_key(r.x[j]);
            gt += (uint32_t)__popcll(__ballot(r.in(j) && (key & last.mask) == last.prefix &&
                                              (key & d.mask) > d.prefix));
        }
        sums.exchange(gt, total);
        if (tid == 0) {
            uint32_t *above = a.above + (int64_t)problem * a.parts + part;
            *above = (LEVEL == 1 ? 0u : *above) + total;
        }
    }
    count_digit<kEvThreads>(r, d, LEVEL, s_hist);
    hist_of(a, LEVEL, problem, part)[kEvBins / 2 - 1 - tid] =
        s_hist[kEvBins - 1 - 2 * tid] << 16 | s_hist[kEvBins - 2 - 2 * tid];
    if (LEVEL == 2 && part == 0 && tid < 2)
        a.picks[a.num_seqs * a.hkv * 2 + problem * 2 + tid] = s_pick[tid];
}

__global__ __launch_bounds__(kEvThreads) void evict_rank_kernel(const EvictArgs a) {
    __shared__ uint32_t s_part[2][kEvThreads / 64], s_pick[2];
    const int tid = threadIdx.x;
    WaveSums<kEvThreads> sums{s_part};
    const int problem = blockIdx.x / a.parts, part = blockIdx.x % a.parts;
    const Choice c(a, problem);
    const uint32_t off = place_recent<kEvThreads>(a, c, part, a.parts);
    if (c.k == 0 || (int64_t)part * kEvPartRows >= c.old)
        return;
    const Rows r(c, part);
    Digits d;
    uint32_t gt0 = 0, eq0 = 0;
    if (c.by_score()) {
        const uint32_t *picks = a.picks + problem * 2;
        d.take(0, picks[0], picks[1]);
        picks += a.num_seqs * a.hkv * 2;
        d.take(1, picks[0], picks[1]);
        const Bins w(a, c, 2, problem, part);
        pick_bin<kEvThreads, 2>(w.sum, d.left, sums, s_pick);
        // rows of the parts before this one: above the pick of each digit,
        // and equal to the pivot
        const uint32_t b0 = kEvBins - 1 - 2 * tid, bin = s_pick[0];
        uint32_t gt = (b0 > bin ? w.before0 : 0u) + (b0 - 1 > bin ? w.before1 : 0u);
        for (int i = tid; i < part; i += kEvThreads)
            gt += a.above[(int64_t)problem * a.parts + i];
        sums.scan(gt, gt0);
        sums.scan(b0 == bin ? w.before0 : b0 - 1 == bin ? w.before1 : 0u, eq0);
        d.take(2, bin, s_pick[1]);
    } else {
        gt0 = (uint32_t)part * kEvPartRows;
    }
    place<kEvThreads>(a, c, r, c.k == c.old, d.prefix, d.left, gt0, eq0, off, sums);
}

template <int D>
__global__ __launch_bounds__(256) void evict_copy_kernel(const EvictArgs a) {
    constexpr int kLanes = D / 8;                          // 16 bytes each
    const int e = threadIdx.x % kLanes;
    const int64_t x = ((int64_t)blockIdx.x * 256 + threadIdx.x) / kLanes;
    const int64_t t = x / a.hkv;
    const int h = (int)(x % a.hkv);
    if (t >= min(a.cu_keep[a.num_seqs], a.cap))
        return;
    const int64_t src = ((int64_t)a.keep_idx[(int64_t)h * a.cap + t] * a.hkv + h) * D + e * 8;
    const int64_t dst = (t * a.hkv + h) * D + e * 8;
#pragma unroll
    for (int i = 0; i < 4; i++)
        if (a.in[i])
            *(u32x4 *)(a.out[i] + dst) = *(const u32x4 *)(a.in[i] + src);
}

}  // namespace

hipError_t launch_cache_evict(const EvictArgs &a, hipStream_t s) {
    const dim3 grid_s(a.num_seqs * a.hkv * a.parts), block(kEvThreads);
    hipError_t e;
    if (a.small) {
        hipLaunchKernelGGL((evict_select_kernel<kEvSmallThreads>), grid_s, dim3(kEvSmallThreads),
                           0, s, a);
        e = hipGetLastError();
    } else if (a.parts == 1) {
        hipLaunchKernelGGL((evict_select_kernel<kEvThreads>), grid_s, block, 0, s, a);
        e = hipGetLastError();
    } else {
        hipLaunchKernelGGL((evict_hist_kernel<0>), grid_s, block, 0, s, a);
        if ((e = hipGetLastError()) != hipSuccess)
            return e;
        hipLaunchKernelGGL((evict_hist_kernel<1>), grid_s, block, 0, s, a);
        if ((e = hipGetLastError()) != hipSuccess)
            return e;
        hipLaunchKernelGGL((evict_hist_kernel<2>), grid_s, block, 0, s, a);
        if ((e = hipGetLastError()) != hipSuccess)
            return e;
        hipLaunchKernelGGL(evict_rank_kernel, grid_s, block, 0, s, a);
        e = hipGetLastError();
    }
    if (e != hipSuccess || (!a.in[0] && !a.in[2]) || a.rows == 0)
        return e;
    const int per = 256 / (a.head_dim / 8);                // rows per workgroup
    const dim3 grid(((int64_t)a.rows * a.hkv + per - 1) / per);
    if (a.head_dim == 128)
        hipLaunchKernelGGL((evict_copy_kernel<128>), grid, dim3(256), 0, s, a);
    else
        hipLaunchKernelGGL((evict_copy_kernel<64>), grid, dim3(256), 0, s, a);
    return hipGetLastError();
}

}  // namespace logo
