// The GQA attention kernels over a cache held in 8 bits: the LDS layout of the
// 32-key E4M3 tiles, the MFMA operand reads and the blocks' scales.
//
// A tile stays in its codes from HBM to the operand registers and is turned into
// bf16 there, two codes an instruction (v_cvt_scalef32_pk_bf16_fp8, at the rate
// of an FMA), with the block's scale, a power of two, applied by the same
// instruction: a code times its scale is exactly a bf16 number, so everything
// behind the operands is the bf16 kernels' arithmetic over the dequantised cache.
// Converting once a workgroup instead (bf16 tiles in LDS) would move 2.5 times the
// LDS bytes, which the bf16 kernels are near the limit of.
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

typedef int i32x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ u32x2 q8_v_read(const uint8_t* base) {
    return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr8_b64_v2i32(PKV_LDS(i32x2, base)));
}

// 0x80 in every byte that is a NaN code (0x7f or 0xff).
__device__ __forceinline__ uint32_t q8_nan_bytes(uint32_t w) {
    return ((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u;
}
// Values of 8 keys of one channel in a tile with masked keys: a NaN code weighs
// nothing in `value` and 1 in `nan`, for a product with the keys' visibility that
// tells which rows see it (0 * NaN would reach the rows that do not).
__device__ __forceinline__ void q8_split_nan(u32x2 w, float scale, bf16x8& value, bf16x8& nan) {
    const uint32_t m0 = (q8_nan_bytes(w[0]) >> 7) * 0xffu, m1 = (q8_nan_bytes(w[1]) >> 7) * 0xffu;
    value = q8_to_bf16(w[0] & ~m0, w[1] & ~m1, scale);
    nan = q8_to_bf16(m0 & 0x38383838u, m1 & 0x38383838u, 1.0f);   // 0x38: 1.0
}

// Kernel argument: empty where the cache is not in 8 bits.
template <bool Q8>
struct ScaleArg {};
template <>
struct ScaleArg<true> : BlockScales {};

// The scales of up to 256 tiles in the order in which the loop visits them, K's
// exponent in the low byte and V's in the next, in four registers of 64 lanes (as
// PageWindow).  Loading it again stalls the loop for two dependent loads, once in
// 256 tiles.
struct ScaleWindow {
    int first, last;        // tiles first .. last - 1
    int e0, e1, e2, e3;

    // key_of(i): first key of tile i < n_tiles.  Table entries are clamped into the pool.
    template <typename F>
    __device__ __forceinline__ void load(const AttnArgs& a, const BlockScales& s, int seq, int layer, int kvh, int from,
                                         int n_tiles, F key_of) {
        const int32_t* const k_row = a.block_table + (int64_t)seq * a.max_pages;
        const int32_t* const v_row = a.v_block_table ? a.v_block_table + (int64_t)seq * a.max_pages : k_row;
        const uint8_t* const k = s.k + layer * s.k_stride[0] + kvh * s.k_stride[1];
        const uint8_t* const v = s.v + layer * s.v_stride[0] + kvh * s.v_stride[1];
        auto lookup = [&](int i) __attribute__((always_inline)) {
            const int key = key_of(min(i, n_tiles - 1));   // (below the slots that the table covers)
            const int entry = key >> a.page_shift;
            const int block = (key & ((1 << a.page_shift) - 1)) >> s.block_shift;
            const int top = (int)(a.n_pages - 1);
            const int kp = min(max(k_row[entry], 0), top), vp = min(max(v_row[entry], 0), top);
            return k[kp * s.k_stride[2] + block * s.k_stride[3]] | (v[vp * s.v_stride[2] + block * s.v_stride[3]] << 8);
        };
        first = from;
        last = from + 64;
        e0 = e1 = e2 = e3 = 0;
        if (n_tiles <= 0) return;
        const int i = from + (int)__lane_id();
        e0 = lookup(i);
        if (n_tiles > last) {
            last = from + 256;
            e1 = lookup(i + 64);
            e2 = lookup(i + 128);
            e3 = lookup(i + 192);
        }
    }
    __device__ __forceinline__ bool holds(int lo, int hi) const { return lo >= first && hi < last; }
    // Both exponents of tile i (one that the window holds), in a scalar register.
    __device__ __forceinline__ uint32_t at(int i) const {
        const int r = (i - first) >> 6, l = (i - first) & 63;
        const int x0 = __builtin_amdgcn_readlane(e0, l), x1 = __builtin_amdgcn_readlane(e1, l);
        const int x2 = __builtin_amdgcn_readlane(e2, l), x3 = __builtin_amdgcn_readlane(e3, l);
        return (uint32_t)(r == 0 ? x0 : r == 1 ? x1 : r == 2 ? x2 : x3);
    }
};
__device__ __forceinline__ float q8_k_scale(uint32_t e) { return __uint_as_float((e & 0xffu) << 23); }
__device__ __forceinline__ float q8_v_scale(uint32_t e) { return __uint_as_float((e >> 8) << 23); }

}  // namespace pkv
