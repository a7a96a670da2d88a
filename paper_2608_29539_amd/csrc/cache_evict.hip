// cache_evict.hip -- caches cut down to a budget of rows per sequence and KV
// head by the attention weight that each row has received.
//
// Of L rows n = min(L, budget) are kept: the last min(recent, n), and of the
// others the k with the largest scores (a NaN is the lowest, -0 equals +0, ties
// go to the lowest index), in ascending order.
//
//   evict_select_kernel  one workgroup per (sequence, KV head): the k-th
//                        largest score by radix selection on order-preserving
//                        32-bit keys (histograms of 11, 11 and 10 bits in LDS),
//                        then one pass that ranks the rows above it and the
//                        first ones equal to it
//   evict_copy_kernel    copies the kept rows of K and V
#include "attn_common.h"
#include "logo_internal.h"

namespace logo {
namespace {

constexpr int kEvThreads = 1024;
constexpr int kEvWaves = kEvThreads / 64;
constexpr int kEvBins = 2048;

// Order-preserving key of a score: a larger score has a larger key, NaN 0.
__device__ __forceinline__ uint32_t score_key(float x) {
    if (x != x)
        return 0;
    const uint32_t u = __float_as_uint(x + 0.f);          // -0 -> +0
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// Exclusive prefix of v over the workgroup, and the total.
__device__ __forceinline__ uint32_t block_scan(uint32_t v, uint32_t *s_part, uint32_t &total) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    uint32_t incl = v;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const uint32_t x = __shfl_up(incl, d, 64);
        if (lane >= d)
            incl += x;
    }
    if (lane == 63)
        s_part[wave] = incl;
    __syncthreads();
    uint32_t before = 0;
    total = 0;
#pragma unroll
    for (int i = 0; i < kEvWaves; i++) {
        const uint32_t x = s_part[i];
        before += i < wave ? x : 0;
        total += x;
    }
    __syncthreads();
    return before + incl - v;
}

__global__ __launch_bounds__(kEvThreads) void evict_select_kernel(const EvictArgs a) {
    __shared__ uint32_t s_hist[kEvBins], s_part[kEvWaves], s_pick[2];
    const int tid = threadIdx.x;
    const int b = blockIdx.x / a.hkv, h = blockIdx.x % a.hkv;
    // rows that the sequences before this one keep
    uint32_t off = 0;
    {
        uint32_t mine = 0;
        for (int i = tid; i < b; i += kEvThreads)
            mine += min(a.cu[i + 1] - a.cu[i], a.budget);
        block_scan(mine, s_part, off);
    }
    const int64_t base = a.cu[b];
    const int L = a.cu[b + 1] - (int)base;
    const int n = min(L, a.budget), rec = min(a.recent, n), k = n - rec, old = L - rec;
    if (h == 0 && tid == 0) {
        if (b == 0)
            a.cu_keep[0] = 0;
        a.cu_keep[b + 1] = (int)off + n;
    }
    const float *sc = a.score + (int64_t)h * a.n + base;
    const int64_t out = (int64_t)h * a.cap + off;
    const int room = a.cap - (int)off;                     // (n, for a capacity as documented)

    uint32_t pivot = 0, need = 0;                          // the k-th key, rows equal to it kept
    if (k > 0 && k < old) {
        uint32_t prefix = 0, mask = 0, left = k;
        for (int pass = 0; pass < 3; pass++) {
            const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0;
            const uint32_t width = pass == 2 ? 1023 : 2047;
            for (int i = tid; i < kEvBins; i += kEvThreads)
                s_hist[i] = 0;
            __syncthreads();
            for (int i = tid; i < old; i += kEvThreads) {
                const uint32_t key = score_key(sc[i]);
                if ((key & mask) == prefix)
                    atomicAdd(&s_hist[(key >> shift) & width], 1u);
            }
            __syncthreads();
            // bins from the largest: this thread's two
            const uint32_t c0 = s_hist[kEvBins - 1 - 2 * tid], c1 = s_hist[kEvBins - 2 - 2 * tid];
            uint32_t total;
            const uint32_t above = block_scan(c0 + c1, s_part, total);
            if (above < left && left <= above + c0 + c1) {
                const bool first = left <= above + c0;
                s_pick[0] = kEvBins - 1 - 2 * tid - (first ? 0 : 1);
                s_pick[1] = left - above - (first ? 0 : c0);
            }
            __syncthreads();
            prefix |= s_pick[0] << shift;
            mask |= width << shift;
            left = s_pick[1];
            __syncthreads();
        }
        pivot = prefix;
        need = left;
    }
    if (k > 0) {
        const bool all = k == old;
        uint32_t gt0 = 0, eq0 = 0;                         // rows before this step
        for (int i0 = 0; i0 < old; i0 += kEvThreads) {
            const int i = i0 + tid;
            const float x = i < old ? sc[i] : 0.f;
            const uint32_t key = score_key(x);
            const bool gt = i < old && (all || key > pivot), eq = i < old && !all && key == pivot;
            uint32_t total;
            const uint32_t ex = block_scan((gt ? 1u : 0u) | (eq ? 0x10000u : 0u), s_part, total);
            const uint32_t gb = gt0 + (ex & 0xFFFFu), eb = eq0 + (ex >> 16);
            const uint32_t at = gb + min(eb, need);
            if ((gt || (eq && eb < need)) && (int)at < room) {
                a.keep_idx[out + at] = (int)base + i;
                a.score_out[out + at] = x;
            }
            gt0 += total & 0xFFFFu;
            eq0 += total >> 16;
        }
    }
    for (int i = tid; i < rec; i += kEvThreads)
        if (k + i < room) {
            a.keep_idx[out + k + i] = (int)base + old + i;
            a.score_out[out + k + i] = sc[old + i];
        }
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
    hipLaunchKernelGGL(evict_select_kernel, dim3(a.num_seqs * a.hkv), dim3(kEvThreads), 0, s, a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || (!a.in[0] && !a.in[2]) || a.cap == 0)
        return e;
    const int rows = 256 / (a.head_dim / 8);               // per workgroup
    const dim3 grid(((int64_t)a.cap * a.hkv + rows - 1) / rows);
    if (a.head_dim == 128)
        hipLaunchKernelGGL((evict_copy_kernel<128>), grid, dim3(256), 0, s, a);
    else
        hipLaunchKernelGGL((evict_copy_kernel<64>), grid, dim3(256), 0, s, a);
    return hipGetLastError();
}

}  // namespace logo
