// The GQA attention kernels over a cache held in 8 bits: conversion, the few-row
// kernel's LDS layout of the 32-key E4M3 tiles and its MFMA operand reads, and the
// scales of the many-row kernel's tiles.
//
// Codes become bf16 two an instruction (v_cvt_scalef32_pk_bf16_fp8, at the rate of
// an FMA), with the block's scale, a power of two, applied by the same instruction:
// a code times its scale is exactly a bf16 number (under the scale bytes 1 and 2 the
// nearest one, as the smallest codes lie between bf16's steps there), so everything
// behind the conversion is the bf16 kernels' arithmetic over the dequantised cache.
// Bytes above 246, whose largest codes bf16 cannot hold, are taken as 246 and 0 as 1,
// so that only NaN codes are not finite, whatever byte a block has that no row sees.
// In the few-row kernel one wave reads a tile and converts it at its operand reads; the
// many-row kernel's four waves share a tile and convert it once, on its way to LDS.
#pragma once

#include "attn_common.h"

namespace pkv {

// XOR swizzles of a row's 16-byte chunk index (16 codes) by its key, for LDS reads
// whose lanes must spread over the 16 bank groups of 16 bytes.
//   K: an operand read takes one logical chunk from 16 consecutive keys.  Rows of
//      128 (64) bytes: 2 (4) keys a bank line, so 8 (4) keys share a place in it.
//   V: a transposed read takes two neighbouring chunks from 8 keys, {0..3, 8..11}
//      or those plus 4: bit 0 of the chunk stays, the pair moves.
template <int D>
__device__ inline int swz_k8(int key) {
    return D == 128 ? (key >> 1) & 7 : (key >> 2) & 3;
}
template <int D>
__device__ inline int swz_v8(int key) {
    return D == 128 ? (((key >> 1) & 1) | ((key >> 2) & 2)) << 1 : ((key >> 3) & 1) << 1;
}

// Per-lane LDS byte offsets of the 32x32x16 MFMA operands within a tile.
//   K (A of S^T = K Q^T): chunk 2c + hl of key j holds the lane's 8 channels of
//       k-steps 2c and 2c + 1, so a k-step contracts channels 32c + 16 hl + 8 (ks & 1)
//       .. +7 (q8_channel); the queries are loaded in that order.
//   V^T (A of O^T = V^T P^T), 16-key step st, channel block db: vofs[db] + st * 16 * D.
//       The 16 lanes of a group give the addresses of 8 keys x 16 channels, in the
//       key order of the P^T accumulators, and each receives one channel's 8 keys.
template <int D>
__device__ inline void gqa_operand_offsets_q8(int lane, int (&kofs)[D / 32], int (&vofs)[D / 32]) {
    const int j = lane & 31, hl = lane >> 5;
#pragma unroll
    for (int c = 0; c < D / 32; ++c) kofs[c] = j * D + (((c * 2 + hl) ^ swz_k8<D>(j)) << 4);
    const int g = lane >> 4, sl = lane & 15;
    const int row = sl >> 1;
    const int key = (row >> 2) * 8 + (g >> 1) * 4 + (row & 3);
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
        vofs[db] = key * D + (((db * 2 + (g & 1)) ^ swz_v8<D>(key)) << 4) + (sl & 1) * 8;
}
__device__ inline int q8_channel(int ks, int hl) { return (ks >> 1) * 32 + hl * 16 + (ks & 1) * 8; }

// Eight codes as bf16, times scale (a power of two).
__device__ __forceinline__ bf16x8 q8_to_bf16(uint32_t lo, uint32_t hi, float scale) {
    const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false);
    const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true);
    const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false);
    const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true);
    return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// The scale byte e that counts for a stored one.
__device__ __forceinline__ uint32_t q8_exponent(uint32_t e) { return max(min(e, 246u), 1u); }

typedef int i32x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ u32x2 q8_v_read(const uint8_t* base) {
    return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr8_b64_v2i32(PKV_LDS(i32x2, base)));
}

// 0x80 in every byte that is a NaN code (0x7f or 0xff).
__device__ __forceinline__ uint32_t q8_nan_bytes(uint32_t w) {
    return ((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u;
}

// Kernel argument: empty where the cache is not in 8 bits.
template <bool Q8>
struct ScaleArg {};
template <>
struct ScaleArg<true> : BlockScales {};

// What a wave that stages one tensor's tiles needs of the tables for the next 128 of them,
// in the order in which the loop visits them: pages (clamped into the pool) and scales, two
// registers of 64 lanes each.  Loading it again stalls the loop for two dependent loads,
// once in about 120 tiles.
struct CodeWindow {
    const int32_t* row;      // the sequence's row of the tensor's block table
    const uint8_t* scales;   // of the layer and head
    int64_t page_stride, block_stride;   // of the scales
    int block_shift, top;
    int first, last;         // tiles first .. last - 1
    int p0, p1;
    float s0, s1;

    __device__ __forceinline__ void init(const AttnArgs& a, const BlockScales& s, bool of_v, int seq, int layer, int kvh) {
        row = (of_v && a.v_block_table ? a.v_block_table : a.block_table) + (int64_t)seq * a.max_pages;
        const int64_t* const stride = of_v ? s.v_stride : s.k_stride;
        scales = (of_v ? s.v : s.k) + layer * stride[0] + kvh * stride[1];
        page_stride = stride[2];
        block_stride = stride[3];
        block_shift = s.block_shift;
        top = (int)(a.n_pages - 1);
    }
    // key_of(i): first key of tile i < n_tiles.
    template <typename F>
    __device__ __forceinline__ void load(const AttnArgs& a, int from, int n_tiles, F key_of) {
        first = from;
        last = from + 64;
        p0 = p1 = 0;
        s0 = s1 = 0.f;
        if (n_tiles <= 0) return;
        auto lookup = [&](int i, int& page, float& scale) __attribute__((always_inline)) {
            const int key = key_of(min(i, n_tiles - 1));   // (below the slots that the table covers)
            page = min(max(row[key >> a.page_shift], 0), top);
            const int block = (key & ((1 << a.page_shift) - 1)) >> block_shift;
            scale = __uint_as_float(q8_exponent(scales[page * page_stride + block * block_stride]) << 23);
        };
        const int i = from + (int)__lane_id();
        lookup(i, p0, s0);
        if (n_tiles > last) {
            last = from + 128;
            lookup(i + 64, p1, s1);
        }
    }
    // Of tile i, which the window holds.
    __device__ __forceinline__ int64_t page(int i) const {
        const int l = (i - first) & 63;
        const int x0 = __builtin_amdgcn_readlane(p0, l), x1 = __builtin_amdgcn_readlane(p1, l);
        return i - first < 64 ? x0 : x1;
    }
    __device__ __forceinline__ float scale(int i) const {
        const int l = (i - first) & 63;
        const int x0 = __builtin_amdgcn_readlane(__float_as_int(s0), l), x1 = __builtin_amdgcn_readlane(__float_as_int(s1), l);
        return __int_as_float(i - first < 64 ? x0 : x1);
    }
};

}  // namespace pkv
