// decode_common.h -- device code shared by the decoding steps (decode.hip,
// decode_prefix.hip, cache_score.hip): the routing decision and the list of
// selected sequences.  gfx950 only.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace logo {
namespace {

// The token's routing decision z_b = gate[b] > thr (fp32, strict: a NaN
// gate or threshold selects nothing), taken identically by every workgroup
// that needs it.  A: arguments with sel_mode, thr_dev and thr_host.
template <class A>
__device__ __forceinline__ float decode_threshold(const A &a) {
    return a.sel_mode == 2 ? a.thr_dev[0] : a.thr_host;
}

// The compacted list of selected sequences (ascending) and the count, each
// where it is asked for: one workgroup of NT threads, ballot + mbcnt ranks
// and a carry over chunks of NT sequences.
template <int NT, class A>
__device__ void build_active_list(const A &a) {
    __shared__ int s_cnt[NT / 64];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const float thr = decode_threshold(a);
    int carry = 0;
    for (int c0 = 0; c0 < a.num_seqs; c0 += NT) {
        const int b = c0 + tid;
        const bool z = b < a.num_seqs && a.gate[b] > thr;
        const uint64_t m = __ballot(z);
        const int below = (int)__builtin_amdgcn_mbcnt_hi((uint32_t)(m >> 32),
                                                        __builtin_amdgcn_mbcnt_lo((uint32_t)m, 0));
        if (lane == 0)
            s_cnt[wave] = (int)__popcll(m);
        __syncthreads();
        int before = carry, total = 0;
        for (int i = 0; i < NT / 64; i++) {
            if (i < wave)
                before += s_cnt[i];
            total += s_cnt[i];
        }
        if (z && a.act)
            a.act[before + below] = b;
        carry += total;
        __syncthreads();                         // s_cnt is rewritten by the next chunk
    }
    if (tid == 0 && a.n_act)
        a.n_act[0] = carry;
}

}  // namespace
}  // namespace logo
