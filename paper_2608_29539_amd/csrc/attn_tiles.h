// attn_tiles.h -- the K and V tiles of the forward attention kernels in LDS:
// their layout, the loads that fill them and the transposed read of V.
// gfx950 only.
#pragma once

#include "attn_common.h"
#include "logo_internal.h"

namespace logo {
namespace {

// LDS tiles, both [key][d].  K rows are padded by 16 B so that the 16-byte
// fragment reads of 8 consecutive rows hit distinct banks.  V rows are not
// padded; instead the 64-byte segments of a row are permuted (segment j of
// row r is stored at j ^ vswz(r)) so that the transpose reads, which take
// one 64-byte segment from each of 4 consecutive rows per half-wave, hit 4
// distinct 64-byte bank groups of the 256-byte bank window.
constexpr int kKPad = 8;
template <int D>
__device__ __forceinline__ constexpr int vswz(int r) {
    // rows per 256-byte bank window: 128 / D; segments per row: D / 32
    return (r / (128 / D)) % (D / 32);
}

// K/V tiles go global -> LDS directly (buffer_load_dwordx4 ... lds): each
// wave-instruction writes 64 consecutive 16-byte LDS slots (lane i at
// M0 + 16 i), so a padded tile is filled as a sequence of 1 KB slot runs; a
// lane whose slot is row padding re-loads the row's last chunk (never read).
// The per-lane byte offsets inside a tile are fixed and computed once.
template <int D, int W>
struct Dma {
    static constexpr int kSlotsK = (D + kKPad) * 2 / 16;     // 16-byte slots per K row
    static constexpr int kSlotsV = D * 2 / 16;
    static constexpr int kInstK = kSlotsK;                   // 64 rows x slots / 64 lanes
    static constexpr int kInstV = kSlotsV;
    static constexpr int kPerWaveK = (kInstK + W - 1) / W;
    static constexpr int kPerWaveV = (kInstV + W - 1) / W;
    int voff_k[kPerWaveK];
    int voff_v[kPerWaveV];
};

template <int D, int W>
__device__ __forceinline__ void dma_plan(Dma<D, W> &d, int wave, int lane, int row_bytes) {
#pragma unroll
    for (int i = 0; i < Dma<D, W>::kPerWaveK; i++) {
        const int slot = (i * W + wave) * 64 + lane;
        const int row = slot / Dma<D, W>::kSlotsK, col = min(slot % Dma<D, W>::kSlotsK, D / 8 - 1);
        d.voff_k[i] = row * row_bytes + col * 16;
    }
#pragma unroll
    for (int i = 0; i < Dma<D, W>::kPerWaveV; i++) {
        // LDS slot (row, chunk p) receives the chunk whose segment maps to p's
        const int slot = (i * W + wave) * 64 + lane;
        const int row = slot / Dma<D, W>::kSlotsV, p = slot % Dma<D, W>::kSlotsV;
        const int col = ((p >> 2) ^ vswz<D>(row)) * 4 + (p & 3);
        d.voff_v[i] = row * row_bytes + col * 16;
    }
}

// Descriptor of one tile: base = its first key row of this KV head, size =
// the rows that exist, so rows at or past the sequence end read as zeros
// (masked keys with zero values keep masked-out products finite).  Raw
// buffer descriptor words: base address (48 bits, stride 0), size in bytes,
// flags.
__device__ __forceinline__ u32x4 tile_rsrc(const uint16_t *kv, int T, int k0, int row_bytes) {
    const int rows = min(kBlockN, T - k0);
    return raw_rsrc((const char *)kv + (long long)k0 * row_bytes, rows > 0 ? rows * row_bytes : 0);
}

template <int D, int W>
__device__ __forceinline__ void dma_k(uint16_t *dst, const Dma<D, W> &d, const uint16_t *kv_k,
                                      int T, int k0, int row_bytes, int wave) {
    const u32x4 r = tile_rsrc(kv_k, T, k0, row_bytes);
#pragma unroll
    for (int i = 0; i < Dma<D, W>::kPerWaveK; i++) {
        const int inst = i * W + wave;
        if (inst < Dma<D, W>::kInstK)
            lds_load16(r, (char *)dst + inst * 1024, d.voff_k[i]);
    }
}
template <int D, int W>
__device__ __forceinline__ void dma_v(uint16_t *dst, const Dma<D, W> &d, const uint16_t *kv_v,
                                      int T, int k0, int row_bytes, int wave) {
    const u32x4 r = tile_rsrc(kv_v, T, k0, row_bytes);
#pragma unroll
    for (int i = 0; i < Dma<D, W>::kPerWaveV; i++) {
        const int inst = i * W + wave;
        if (inst < Dma<D, W>::kInstV)
            lds_load16(r, (char *)dst + inst * 1024, d.voff_v[i]);
    }
}

// V^T operand of the O^T MFMA straight from the row-major V tile with the
// gfx950 LDS transpose read: within each 16-lane group, lane 4b+e receives
// element e of the 4-element rows addressed by lanes b, b+4, b+8, b+12.
// Lane i of group q addresses row (key0 + 4*(q/2) + i/4), columns
// (c0 + 16*(q%2) + 4*(i%4)) .. +3, so lane l ends up holding column c0 + l%32
// for keys key0 + 4*(l/32) + 0..3 (first read) and, 8 rows further, + 8..11
// (second read): the 8 keys of its MFMA k-slice, in the order the S^T
// accumulator (and so P^T) holds them.
__device__ __forceinline__ bf16x8 read_vt_frag(const uint16_t *vrow_lane, int row_stride) {
    return lds_tr_pair(vrow_lane, vrow_lane + 8 * row_stride);
}

// Unpadded rows of D / 8 16-byte pieces: piece c of row r is stored at
// c ^ piece_swz(r), so that the 16-byte reads of one piece from 16 rows hit
// distinct banks (rows of D = 64 fill half of the 256-byte bank window: the
// two rows that share one take the same permutation).
template <int D>
__device__ __forceinline__ constexpr int piece_swz(int r) {
    return D == 128 ? r % 16 : (r / 2) % 8;
}

}  // namespace
}  // namespace logo
