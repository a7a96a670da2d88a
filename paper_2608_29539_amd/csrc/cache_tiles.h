// cache_tiles.h -- device helpers of the kernels that read caches
// (decode_prefix.hip, cache_score.hip): tiles of K and V rows in LDS filled by
// direct loads from addresses of the lanes' own, their layouts, waits.  gfx950
// only.
#pragma once

#include "attn_common.h"

namespace logo {
namespace {

// The larger of two: the middle of them and +inf (fmaxf makes the compiler
// quiet its operands first, an instruction each).
__device__ __forceinline__ float max2(float a, float b) {
    return __builtin_amdgcn_fmed3f(a, b, __builtin_inff());
}

// One 16-byte-per-lane load from a lane's own address to LDS (lane i writes
// the 16 bytes at lds + 16 i); see lds_load16_at.
__device__ __forceinline__ void lds_gather16(const void *src, uint32_t lds) {
    const uint32_t lds_addr = __builtin_amdgcn_readfirstlane(lds);
    uint32_t saved;
    asm volatile(
        "s_mov_b32 %0, m0\n\t"
        "s_mov_b32 m0, %1\n\t"
        "s_nop 0\n\t"
        "global_load_lds_dwordx4 %2, off\n\t"
        "s_mov_b32 m0, %0"
        : "=&s"(saved)
        : "s"(lds_addr), "v"(src)
        : "memory");
}

// kWaitVmcnt0 for lgkmcnt (LDS reads) only.
constexpr int kWaitLgkmcnt0 = 0xC07F;

// Unpadded rows of D / 8 16-byte pieces: piece c of row r is stored at
// c ^ piece_swz(r), so that the 16-byte reads of one piece from 16 rows hit
// distinct banks (rows of D = 64 fill half of the 256-byte bank window: the
// two rows that share one take the same permutation).
template <int D>
__device__ __forceinline__ constexpr int piece_swz(int r) {
    return D == 128 ? r % 16 : (r / 2) % 8;
}

// Rows of V as the transposed read (lds_tr_pair) takes them: segment j (32
// columns, 64 bytes) of row r is stored at j ^ seg_swz(r), so that the read of
// one segment from four consecutive rows hits distinct 64-byte bank groups of
// the 256-byte bank window (which holds 128 / D rows).
template <int D>
__device__ __forceinline__ constexpr int seg_swz(int r) {
    return (r / (128 / D)) % (D / 32);
}

}  // namespace
}  // namespace logo
