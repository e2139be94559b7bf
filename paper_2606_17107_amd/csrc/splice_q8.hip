// Reposition + splice into a cache held in 8 bits: re-rotate a chunk's keys by
// delta = dst_pos - src_pos as splice.hip does, quantise keys and values to E4M3
// codes with one power-of-two scale per block of slots, KV head, layer and tensor,
// and write codes and scales into the paged destination.
//
// For a block that receives the rows x_t and keeps the rows that it held before in
// other slots below the sequence's length:
//     need = the smallest e in [1, 246] with max |x_t| <= 448 * 2^(e - 127)
//     e    = need, or max(need, old e) if the block keeps a row
//     code = E4M3(x_t * 2^(127 - e))  to the nearest, ties to even
// and where e grew, kept codes become E4M3(code * 2^(old e - e)).  Products with
// powers of two are exact, so each stored value is rounded once; a kept row loses
// nothing but what falls below E4M3's smallest step.  A NaN or an infinity is
// stored as NaN (E4M3 has no infinity) and does not enter the maximum.  246 is the
// last e under which every code is finite in bf16; finite magnitudes above
// 448 * 2^119 (2.98e38) get the largest code.
//
// Design (a stream of 2 or 4 bytes read and 1 written per element):
//   * A wave owns 32 slots of one (layer, tensor, KV head): 8 lanes a row at head
//     size 128, two 8-channel chunks a lane (the two halves of its rotary pairs), all
//     of its rows in registers as fp32 between the maximum and the codes, so the
//     source is read once.  Blocks of 64 and 128 slots are 2 and 4 waves of one
//     workgroup that exchange their maxima through LDS; with blocks of 32 slots the
//     four waves of a workgroup take four heads.
//   * A block is written by one owner, the first segment (by number) that touches
//     it; the owner gathers the rows of all segments that end or begin there, so that
//     chunks spliced back to back in one call share a block's scale.  Every wave finds
//     the segments by looking through the records, 64 at a time.
//   * cos and sin are formed as exactly as fp32 holds them: an E4M3 code depends on the
//     rotated value's last bits only near a rounding boundary, and there the fp32
//     rotation decides as exactly as it can.
//   * Measured (8 KV heads of 128): 4096 tokens into 32 layers 138 us a call, 808 MB at 5.9
//     TB/s, what a copy of such rows reaches; 277 when every row was loaded once for the
//     maximum and once for the codes; the same from fp32 into 16 layers 119 us, 671 MB at
//     5.7 TB/s.  16 contexts of 4052 tokens in 4 layers, whose source stays in the L2s, 184
//     us for 531 MB written: vector instructions take 72% of the cycles (168 us where no row
//     turns), and a third of the workgroups, sized by the longest of three chunks, have no
//     block (154 us in a grid of 7 block places a chunk instead of 18; 161 us for one chunk
//     a context).  One token in each of 64 contexts 7 us, 5 in the kernel: a chain of loads.
#include <math.h>

#include "attn_columns.h"

namespace pkv {
namespace {

constexpr int kWaves = 4;
constexpr int kSub = 32;           // slots per wave
constexpr int kPairs = 64;         // most rotary pairs of a row
constexpr int kTop = 0x7f600000;   // fp32 bits of 448 * 2^119, the largest magnitude that is stored
constexpr int64_t kMaxGridX = 0xffffffffll / (kWaves * 64);   // blocks: HIP refuses 2^32 threads in one dimension

struct Freqs {
    double w[kPairs];
};

// Grid: x = (block of the segment, part of the heads), y = segment, z = (layer,
// tensor).  A workgroup is its waves' worth of heads of one block; with blocks of 32
// slots and fewer heads than waves, of several consecutive blocks.
struct StoreGeo {
    int spots;             // x extent over the parts: groups of blocks of the longest segment
    int parts;             // workgroups that share the heads of a slot
    int heads;             // heads per workgroup
    int blocks;            // blocks per workgroup: waves / (waves per block x heads)
    int tensors;           // 2, or 1 without values
    int rope_c0, rope_nc;  // rotary chunks of 8 channels: first, number
};

typedef short s16x2 __attribute__((ext_vector_type(2)));
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));

// Codes of four values divided by a power of two (the conversion applies it: one
// instruction for two values, like the unscaled one).
__device__ inline uint32_t pack4(float a, float b, float c, float d, float scale) {
    s16x2 v = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(s16x2{0, 0}, a, b, scale, false);
    v = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(v, c, d, scale, true);
    return __builtin_bit_cast(uint32_t, v);
}
__device__ inline uint32_t pack4_bf16(uint32_t lo, uint32_t hi, float scale) {
    s16x2 v = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(s16x2{0, 0}, __builtin_bit_cast(bf16x2, lo), scale, false);
    v = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(v, __builtin_bit_cast(bf16x2, hi), scale, true);
    return __builtin_bit_cast(uint32_t, v);
}
__device__ inline float exp2_int(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }   // -126 <= e <= 127

// cos and sin of delta * omega to fp32's last bit or nearly: the angle is formed and
// reduced by pi/2 in fp64, r = rh + rl in two fp32 parts, and the Taylor series are
// summed in fp32 with their leading terms kept apart from the corrections (errors below
// 0.09 of a unit in the last place beside the rounding of the result, which is the nearest
// number for all but 0.3% of the sines and 0.6% of the cosines; terms below 2^-29 left out).
// fp64 series would hold 24 more registers in constants.
__device__ inline void turn(double delta, double omega, float& c, float& s) {
    const double x = delta * omega;
    const double k = rint(x * 0.63661977236758134308);            // 2/pi
    double r = fma(-k, 1.5707963267948966192, x);                // pi/2, leading part
    r = fma(-k, 6.123233995736766036e-17, r);                    // pi/2, trailing part
    const int q = (int)fma(-4.0, floor(k * 0.25), k);            // k mod 4
    const float rh = (float)r, rl = (float)(r - (double)rh);
    const float z = rh * rh, ze = fmaf(rh, rh, -z), hz = 0.5f * z;   // rh^2 = z + ze
    // sin r = rh - rh^3/3! + (rh^3 (z/5! - z^2/7! + z^3/9!) + rl (1 - z/2))
    const float cube = rh * z, cube_e = fmaf(rh, ze, fmaf(rh, z, -cube));
    constexpr float k3 = -0.166666671633720398f, k3_e = 4.96705373e-9f;   // -1/3! = k3 + k3_e
    const float third = cube * k3, third_e = fmaf(cube_e, k3, fmaf(cube, k3, -third));
    float ps = fmaf(z, 2.75573192e-6f, -1.98412698e-4f);
    ps = fmaf(z, ps, 8.33333333e-3f);
    ps = fmaf(z, ps, k3_e);
    const float lead = rh + third, lead_e = (rh - lead) + third;
    const float sr = lead + (lead_e + fmaf(cube, ps, third_e + fmaf(-hz, rl, rl)));
    // cos r = (1 - z/2) + (what that rounding lost - (ze + 2 rh rl)/2 + z^2 (1/4! - z/6! + z^2/8! - z^3/10!))
    float pc = fmaf(z, -2.75573192e-7f, 2.48015873e-5f);
    pc = fmaf(z, pc, -1.38888889e-3f);
    pc = fmaf(z, pc, 4.16666667e-2f);
    const float w = 1.f - hz, lost = (1.f - w) - hz;
    const float cr = w + fmaf(z * z, pc, fmaf(-0.5f, ze + 2.f * rh * rl, lost));
    const float sa = (q & 1) ? cr : sr;
    const float ca = (q & 1) ? sr : cr;
    s = (q & 2) ? -sa : sa;
    c = ((q + 1) & 2) ? -ca : ca;
}

// Eight channels of a source row as they are loaded, and as fp32.
template <bool F32>
struct Raw8 {
    u32x4 a, b;
    __device__ __forceinline__ void load(const char* p) {
        a = __builtin_nontemporal_load((const u32x4*)p);
        b = __builtin_nontemporal_load((const u32x4*)(p + 16));
    }
    __device__ __forceinline__ float get(int i) const { return __uint_as_float(i < 4 ? a[i & 3] : b[i & 3]); }
};
template <>
struct Raw8<false> {
    u32x4 a;
    __device__ __forceinline__ void load(const char* p) { a = *(const u32x4*)p; }
    __device__ __forceinline__ float get(int i) const {
        return __uint_as_float(i & 1 ? a[i >> 1] & 0xffff0000u : a[i >> 1] << 16);
    }
};

// The value of lane l ^ 1.
__device__ inline uint32_t swap1(uint32_t v) { return (uint32_t)dpp<0xb1>((int)v, (int)v); }   // quad_perm [1, 0, 3, 2]

// D: head size.  SUBS: waves (of 32 slots) per scale block.  INTER: interleaved pairs.
// LISTED: instead of records, sequence s appends rows a.rows[s][0 .. a.n_rows[s]) of the
// source behind its a.kv_len[s] slots, as they are.
template <int D, int SUBS, bool F32, bool INTER, bool LISTED>
__global__ __launch_bounds__(kWaves * 64, D == 64 ? 5 : F32 ? 3 : 4) void store_kernel(StoreArgs a, StoreGeo g, Freqs ft) {
    constexpr int LPT = D / 16;           // lanes per row
    constexpr int TPS = 64 / LPT;         // rows per step
    constexpr int STEPS = kSub / TPS;
    constexpr int BT = SUBS * kSub;       // slots per scale block
    constexpr int EB = F32 ? 4 : 2;
    __shared__ int top_lds[2][kWaves], any_lds[2][kWaves];
    __shared__ __attribute__((aligned(16))) float coef_lds[kWaves][2 * kPairs];   // cos of all pairs, then sin

    // The first look at the records (below) is under way before this segment's own is here.
    const int lane = threadIdx.x & 63;
    StoreSegment look{};
    if constexpr (!LISTED) look = a.segs[min(lane, a.n_segs - 1)];
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int seg_i = blockIdx.y;
    StoreSegment mine;
    if constexpr (LISTED) {
        const int at = a.kv_len[seg_i];
        mine = StoreSegment{0, seg_i, min(a.n_rows[seg_i], a.max_rows), at, at};
    } else {
        mine = a.segs[seg_i];
    }
    const int spot = g.parts == 1 ? (int)blockIdx.x : (int)(blockIdx.x / (uint32_t)g.parts);
    const int part = (int)blockIdx.x - spot * g.parts;
    const int tensor = g.tensors == 2 ? blockIdx.z & 1 : 0, layer = g.tensors == 2 ? blockIdx.z >> 1 : blockIdx.z;
    const bool is_k = tensor == 0;
    const int sub = wave % SUBS, member = wave / SUBS;   // heads fastest
    const int in_group = g.blocks == 1 ? 0 : member / g.heads;
    const int head_i = part * g.heads + member - in_group * g.heads;
    const bool working = head_i < a.n_kv_heads;   // the other waves only meet the barriers
    const int head = working ? head_i : 0;

    const bool teller = blockIdx.x == 0 && blockIdx.z == 0 && threadIdx.x == 0;   // reports what is out of range
    auto flag = [&]() __attribute__((always_inline)) {
        if (a.err_flag) *a.err_flag = 1;
    };
    if (mine.n_tokens <= 0) return;
    const int64_t past = (int64_t)mine.dst_pos0 + mine.n_tokens;
    if (teller && (mine.seq < 0 || mine.seq >= a.n_seqs || mine.dst_pos0 < 0 || past > a.dst_capacity ||
                   (LISTED ? a.n_src <= 0 : mine.src_slot0 < 0 || mine.src_slot0 > a.n_src - mine.n_tokens)))
        flag();
    if (mine.seq < 0 || mine.seq >= a.n_seqs || a.n_src <= 0 || (LISTED && mine.dst_pos0 < 0)) return;
    const int cap = (int)a.dst_capacity;   // at most 2^30: slots and block ends are int32
    const int end = (int)min(past, (int64_t)cap);
    const int live = min(a.kv_len[mine.seq], cap);

    // This lane's chunks of 8 channels: rotary lanes hold a chunk and its partner.
    const int cl = lane % LPT, row0 = lane / LPT;
    const int half_r = is_k ? g.rope_nc >> 1 : 0;
    const bool rope = cl < half_r;
    int ca, cb;
    if (rope) {
        ca = g.rope_c0 + cl;
        cb = ca + half_r;
    } else if (is_k) {
        const int i0 = cl - half_r, i1 = i0 + ((D / 8 - g.rope_nc) >> 1);
        ca = i0 < g.rope_c0 ? i0 : i0 + g.rope_nc;
        cb = i1 < g.rope_c0 ? i1 : i1 + g.rope_nc;
    } else {
        ca = cl;
        cb = cl + LPT;
    }
    // Chunks of lanes 2m and 2m + 1 are neighbours, the first at an even place: 16 bytes of codes.
    const bool pairs = !is_k || (g.rope_c0 % 2 == 0 && g.rope_nc % 4 == 0);
    const char* const src = (is_k ? a.src_k : a.src_v) + ((int64_t)layer * (is_k ? a.src_k_stride[0] : a.src_v_stride[0]) +
                                                          (int64_t)head * (is_k ? a.src_k_stride[1] : a.src_v_stride[1])) * EB;
    const uint32_t src_row = (uint32_t)((is_k ? a.src_k_stride[2] : a.src_v_stride[2]) * EB);   // at most 16 MiB
    uint8_t* const dst = (is_k ? a.dst_k : a.dst_v) + (int64_t)layer * (is_k ? a.dst_k_stride[0] : a.dst_v_stride[0]) +
                         (int64_t)head * (is_k ? a.dst_k_stride[1] : a.dst_v_stride[1]);
    const uint32_t dst_row = (uint32_t)(is_k ? a.dst_k_stride[2] : a.dst_v_stride[2]);
    const int64_t dst_page = is_k ? a.dst_k_page_stride : a.dst_v_page_stride;
    const int32_t* const table =
        (!is_k && a.v_block_table ? a.v_block_table : a.block_table) + (int64_t)mine.seq * a.max_pages;
    uint8_t* const scales = (is_k ? a.k_scale : a.v_scale) + (int64_t)layer * (is_k ? a.k_scale_stride[0] : a.v_scale_stride[0]) +
                            (int64_t)head * (is_k ? a.k_scale_stride[1] : a.v_scale_stride[1]);

    // The segment's blocks, a grid's worth apart (one, unless a segment is longer than the stated bound).
    const int b0 = max(mine.dst_pos0, 0) / BT + spot * g.blocks + in_group, b_end = (end + BT - 1) / BT;
    int turn_no = 0;
#pragma unroll 1
    for (int b = b0; b < b_end; b += g.spots * g.blocks) {
        const int slot0 = b * BT;                     // the block's first slot
        const int first = slot0 + sub * kSub + row0;  // this lane's slots: first, + TPS, ..
        const int block_end = min(slot0 + BT, cap);
        const int page = table[slot0 >> a.page_shift];
        const bool in_pool = page >= 0 && page < a.n_pages;
        const int64_t at = (int64_t)(in_pool ? page : 0);
        const int inside = slot0 & ((1 << a.page_shift) - 1);
        uint8_t* const scale_at = scales + at * (is_k ? a.k_scale_stride[2] : a.v_scale_stride[2]) +
                                  (inside / BT) * (is_k ? a.k_scale_stride[3] : a.v_scale_stride[3]);
        uint8_t* const rows = dst + at * dst_page + (int64_t)(inside + sub * kSub) * dst_row;

        // Which record fills which slot: this segment's own, then the others that touch the block, by
        // number (a slot that two records name goes to the first); one below this segment's owns the
        // block.  The own rows are under way while the others are looked for, 64 records at a time.
        int rec[STEPS];   // the record's place among those that touch the block, -1 none
#pragma unroll
        for (int t = 0; t < STEPS; ++t) rec[t] = -1;
        // Take the slots of a record, as its `place`-th; returns the address of its first row in the block
        // (a row that exists, where it has none) and sets *lo to that row's slot.
        auto assign = [&](const StoreSegment& s, int place, int* lo_slot) __attribute__((always_inline)) {
            // the block's slots [lo, hi) that the record fills from rows that exist
            const int64_t shift = (int64_t)s.dst_pos0 - s.src_slot0;   // slot - source slot
            const int lo = (int)min(max(max((int64_t)slot0, (int64_t)s.dst_pos0), shift), (int64_t)block_end);
            const int64_t rows_end = LISTED ? past : shift + a.n_src;
            const int hi = (int)max(min(min((int64_t)block_end, (int64_t)s.dst_pos0 + s.n_tokens), rows_end), (int64_t)slot0);
#pragma unroll
            for (int t = 0; t < STEPS; ++t) {
                const int slot = first + t * TPS;
                if (slot >= lo && slot < hi && rec[t] < 0) rec[t] = place;
            }
            *lo_slot = lo;
            return src + (lo < hi ? (uint64_t)(lo - shift) * src_row : 0);
        };
        Raw8<F32> raw[STEPS][2];
        {
            int lo;
            const char* const p = assign(mine, 0, &lo);
            if constexpr (LISTED) {
                int row[STEPS];
#pragma unroll
                for (int t = 0; t < STEPS; ++t)
                    row[t] = rec[t] == 0 ? a.rows[(int64_t)seg_i * a.max_rows + (first + t * TPS - mine.dst_pos0)] : 0;
#pragma unroll
                for (int t = 0; t < STEPS; ++t) {
                    const bool is = row[t] >= 0 && row[t] < a.n_src;
                    if (!is) {
                        rec[t] = -1;
                        flag();
                    }
                    const char* const at = src + (is ? (uint64_t)(uint32_t)row[t] * src_row : 0);
                    raw[t][0].load(at + ca * 8 * EB);
                    raw[t][1].load(at + cb * 8 * EB);
                }
            } else {
#pragma unroll
                for (int t = 0; t < STEPS; ++t) {
                    const uint32_t off = rec[t] == 0 ? (uint32_t)(first + t * TPS - lo) * src_row : 0u;
                    raw[t][0].load(p + (off + ca * 8 * EB));
                    raw[t][1].load(p + (off + cb * 8 * EB));
                }
            }
        }
        const int old = (int)*scale_at;
        auto hit = [&](const StoreSegment& s, int j) __attribute__((always_inline)) {
            return j < a.n_segs && j != seg_i && s.seq == mine.seq && s.n_tokens > 0 && s.dst_pos0 < block_end &&
                   (int64_t)s.dst_pos0 + s.n_tokens > slot0;
        };
        auto others = [&](int j0) __attribute__((always_inline)) {   // those among records j0 .. j0 + 63
            if (a.n_segs > 64) look = a.segs[min(j0 + lane, a.n_segs - 1)];
            return __builtin_amdgcn_ballot_w64(hit(look, j0 + lane));
        };
        int records = 1;
        bool owner = true, moved = mine.dst_pos0 != mine.src_pos0;
#pragma unroll 1
        for (int j0 = 0; !LISTED && j0 < a.n_segs && owner; j0 += 64) {
#pragma unroll 1
            for (uint64_t hits = others(j0); hits; hits &= hits - 1) {
                const int h = j0 + __builtin_ctzll(hits);
                owner = h > seg_i;
                if (!owner) break;
                const StoreSegment s = a.segs[h];
                int lo;
                const char* const p = assign(s, records, &lo);
#pragma unroll
                for (int t = 0; t < STEPS; ++t) {
                    if (rec[t] == records) {
                        const uint32_t off = (uint32_t)(first + t * TPS - lo) * src_row;
                        raw[t][0].load(p + (off + ca * 8 * EB));
                        raw[t][1].load(p + (off + cb * 8 * EB));
                    }
                }
                ++records;
                moved = moved || s.dst_pos0 != s.src_pos0;
            }
        }
        if (!owner) continue;   // uniform over the workgroup

        bool gets = false, keeps = false;
        bool kept[STEPS];
#pragma unroll
        for (int t = 0; t < STEPS; ++t) {
            kept[t] = working && rec[t] < 0 && first + t * TPS < min(live, block_end);
            gets |= rec[t] >= 0;
            keeps |= kept[t];
        }
        int any = (__builtin_amdgcn_ballot_w64(gets) != 0 ? 1 : 0) | (__builtin_amdgcn_ballot_w64(keeps) != 0 ? 2 : 0);
        int e = 0;

        // From the rows to their codes.  PACKED: no row turns, and they stay in bf16, which takes half
        // the instructions; otherwise they become fp32.  (Two copies of the code rather than a choice at
        // each step, which would hold both forms in registers.)
        auto quantise = [&](auto packed_tag) __attribute__((always_inline)) {
            constexpr bool PACKED = decltype(packed_tag)::value;
            // the fp32 bits of the largest finite magnitude
            int top;
            float x[PACKED ? 1 : STEPS][16];
            if constexpr (PACKED) {
                auto largest = [&](auto all_tag) __attribute__((always_inline)) {
                    u16x2 m = {0, 0};
#pragma unroll
                    for (int t = 0; t < STEPS; ++t)
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            u16x2 v = __builtin_bit_cast(u16x2, rec[t] >= 0 ? raw[t][i >> 2].a[i & 3] & 0x7fff7fffu : 0u);
                            if (!decltype(all_tag)::value) {
                                v[0] = v[0] < 0x7f80 ? v[0] : 0;
                                v[1] = v[1] < 0x7f80 ? v[1] : 0;
                            }
                            m = __builtin_elementwise_max(m, v);
                        }
                    return max((int)m[0], (int)m[1]);
                };
                top = largest(std::true_type{});
                if (__builtin_amdgcn_ballot_w64(top >= 0x7f80) != 0) top = largest(std::false_type{});
                top <<= 16;
            } else {
#pragma unroll
                for (int t = 0; t < STEPS; ++t)
#pragma unroll
                    for (int i = 0; i < 16; ++i) x[t][i] = raw[t][i >> 3].get(i & 7);
                // Turn the rows of a record, the r-th that touches the block.
                auto turn_rows = [&](const StoreSegment& s, int r) __attribute__((always_inline)) {
                    if (!is_k || s.dst_pos0 == s.src_pos0) return;   // uniform
                    // lane l evaluates pair l; the others' come through LDS (a wave's accesses are in order)
                    float c1, s1;
                    turn((double)s.dst_pos0 - (double)s.src_pos0, ft.w[lane], c1, s1);
                    asm volatile("" ::: "memory");
                    coef_lds[wave][lane] = c1;
                    coef_lds[wave][kPairs + lane] = s1;
                    __builtin_amdgcn_wave_barrier();
                    asm volatile("" ::: "memory");
                    float c[8], sn[8];
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        // HALF: pairs 8 cl ..; INTERLEAVED: 4 pairs of each of the lane's chunks
                        const int pair = (INTER ? (h ? (half_r + cl) * 4 : cl * 4) : cl * 8 + 4 * h) & (kPairs - 1);
                        const f32x4 cv = *(const f32x4*)&coef_lds[wave][pair];
                        const f32x4 sv = *(const f32x4*)&coef_lds[wave][kPairs + pair];
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            c[4 * h + i] = cv[i];
                            sn[4 * h + i] = sv[i];
                        }
                    }
#pragma unroll
                    for (int t = 0; t < STEPS; ++t) {
                        if (!rope || rec[t] != r) continue;
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            // Rounded as the formula stands, products and sum: which of two codes a value
                            // beside a rounding boundary gets is then the same as in a plain fp32 program.
                            // (An FMA for one product errs as often, on other values; 16 contexts of 4052
                            // tokens in 4 layers: 180 us, 184 as it is.)
#pragma clang fp contract(off)
                            const int ia = INTER ? 2 * i : i, ib = INTER ? 2 * i + 1 : i + 8;
                            const float u = x[t][ia], v = x[t][ib];
                            x[t][ia] = u * c[i] - v * sn[i];
                            x[t][ib] = u * sn[i] + v * c[i];
                        }
                    }
                };
                turn_rows(mine, 0);
                // The other records' rows, found once more.
#pragma unroll 1
                for (int j0 = 0, r = 1; !LISTED && r < records && j0 < a.n_segs; j0 += 64)
#pragma unroll 1
                    for (uint64_t hits = others(j0); hits; hits &= hits - 1, ++r)
                        turn_rows(a.segs[j0 + __builtin_ctzll(hits)], r);
                float m = 0.f;
#pragma unroll
                for (int t = 0; t < STEPS; ++t) {
                    float n = 0.f;
#pragma unroll
                    for (int i = 0; i < 16; ++i) n = fmaxf(n, fabsf(x[t][i]));   // (passes over a NaN)
                    m = rec[t] >= 0 ? fmaxf(m, n) : m;
                }
                if (__builtin_amdgcn_ballot_w64(m == INFINITY) != 0) {
                    m = 0.f;
#pragma unroll
                    for (int t = 0; t < STEPS; ++t)
#pragma unroll
                        for (int i = 0; i < 16; ++i)
                            m = fmaxf(m, rec[t] >= 0 && fabsf(x[t][i]) < INFINITY ? fabsf(x[t][i]) : 0.f);
                }
                top = (int)__float_as_uint(m);
            }
            top = wave_max_u(top);
            if constexpr (SUBS > 1) {
                // (two sets of words: a wave may be one block ahead)
                if (lane == 0) {
                    top_lds[turn_no][wave] = top;
                    any_lds[turn_no][wave] = any;
                }
                __syncthreads();
#pragma unroll
                for (int w = 0; w < SUBS; ++w) {
                    top = max(top, top_lds[turn_no][wave / SUBS * SUBS + w]);
                    any |= any_lds[turn_no][wave / SUBS * SUBS + w];
                }
            }
            if (!working || !in_pool || !(any & 1)) return;
            // 448 = 1.75 * 2^8 is the largest code.
            const bool beyond = __builtin_amdgcn_readfirstlane(top) > kTop;
            top = min(top, kTop);
            const int need = (top >> 23) - 8 + ((top & 0x7fffff) > 0x600000 ? 1 : 0);   // at most 246
            e = max(need, 1);
            if (any & 2) e = min(max(e, old), 246);   // (a byte above 246 means 246, one of 0 means 1)
            const float scale = __uint_as_float((uint32_t)e << 23);   // 2^(e - 127)
#pragma unroll
            for (int t = 0; t < STEPS; ++t) {
                if (rec[t] < 0) continue;
                uint8_t* const p = rows + (row0 + t * TPS) * dst_row;
                u32x2 w[2];
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    if constexpr (PACKED) {
                        const u32x4 y = raw[t][h].a;
                        w[h] = u32x2{pack4_bf16(y[0], y[1], scale), pack4_bf16(y[2], y[3], scale)};
                    } else {
                        const float* y = x[t] + 8 * h;
                        w[h] = u32x2{pack4(y[0], y[1], y[2], y[3], scale), pack4(y[4], y[5], y[6], y[7], scale)};
                    }
                }
                if (__builtin_expect(beyond, 0)) {   // the codes of finite values that came out as NaN become the largest
#pragma unroll
                    for (int h = 0; h < 2; ++h)
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            uint32_t lost = ((w[h][i] & 0x7f7f7f7fu) + 0x01010101u) >> 7 & 0x01010101u;   // 1 in each NaN byte
#pragma unroll
                            for (int k = 0; k < 4; ++k) {
                                uint32_t bits;
                                if constexpr (PACKED) bits = k & 1 ? raw[t][h].a[2 * i + k / 2] : raw[t][h].a[2 * i + k / 2] << 16;
                                else bits = __float_as_uint(x[t][8 * h + 4 * i + k]);
                                lost &= ~(((bits & 0x7f800000u) + 0x00800000u) >> 31 << 8 * k);   // NaN or infinite itself
                            }
                            w[h][i] -= lost;
                        }
                }
                if (pairs) {
                    // lanes 2m and 2m + 1 hold neighbouring chunks of either half of the row: one
                    // takes both of the first half, the other both of the second
                    const bool odd = lane & 1;
                    const uint32_t g0 = swap1(odd ? w[0][0] : w[1][0]), g1 = swap1(odd ? w[0][1] : w[1][1]);
                    const u32x4 v = odd ? u32x4{g0, g1, w[1][0], w[1][1]} : u32x4{w[0][0], w[0][1], g0, g1};
                    __builtin_nontemporal_store(v, (u32x4*)(p + (odd ? cb - 1 : ca) * 8));
                } else {
                    __builtin_nontemporal_store(w[0], (u32x2*)(p + ca * 8));
                    __builtin_nontemporal_store(w[1], (u32x2*)(p + cb * 8));
                }
            }
        };
        if constexpr (F32) {
            quantise(std::false_type{});
        } else {
            if (moved && is_k) quantise(std::false_type{});   // uniform over the workgroup
            else quantise(std::true_type{});
        }
        turn_no ^= 1;   // (a skipped block has no barrier)
        if (working && !in_pool && sub == 0 && lane == 0) flag();
        if (!working || !in_pool || !(any & 1)) continue;
        if ((any & 2) && e > old) {
            // 2^(old - e): codes below 2^-18 of the largest one vanish, so no smaller factor is needed
            const float down = exp2_int(max(max(old, 1) - e, -126));
#pragma unroll
            for (int t = 0; t < STEPS; ++t) {
                if (!kept[t]) continue;
                uint8_t* const p = rows + (row0 + t * TPS) * dst_row;
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    u32x2* const q = (u32x2*)(p + (h ? cb : ca) * 8);
                    u32x2 w = *q;
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[i], false);
                        const auto hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[i], true);
                        w[i] = pack4(lo[0] * down, lo[1] * down, hi[0] * down, hi[1] * down, 1.0f);
                    }
                    *q = w;
                }
            }
        }
        if (sub == 0 && lane == 0 && (!(any & 2) || e != old)) *scale_at = (uint8_t)e;
    }
}

template <int D, int SUBS>
void launch_geo(const StoreArgs& a, const StoreGeo& g, const Freqs& f, dim3 grid, hipStream_t stream) {
    const dim3 block(kWaves * 64);
    if (a.elem_bytes == 4) {
        if (a.rows) hipLaunchKernelGGL((store_kernel<D, SUBS, true, false, true>), grid, block, 0, stream, a, g, f);
        else if (a.rope_style) hipLaunchKernelGGL((store_kernel<D, SUBS, true, true, false>), grid, block, 0, stream, a, g, f);
        else hipLaunchKernelGGL((store_kernel<D, SUBS, true, false, false>), grid, block, 0, stream, a, g, f);
    } else {
        if (a.rows) hipLaunchKernelGGL((store_kernel<D, SUBS, false, false, true>), grid, block, 0, stream, a, g, f);
        else if (a.rope_style) hipLaunchKernelGGL((store_kernel<D, SUBS, false, true, false>), grid, block, 0, stream, a, g, f);
        else hipLaunchKernelGGL((store_kernel<D, SUBS, false, false, false>), grid, block, 0, stream, a, g, f);
    }
}

}  // namespace

namespace {

dim3 make_geo(const StoreArgs& a, StoreGeo& g, bool& fits) {
    const int bt = a.block_tokens, per_wg = kWaves / (bt / kSub);
    g.parts = (a.n_kv_heads + per_wg - 1) / per_wg;
    // (the waves of a workgroup that meet at a barrier take one block together)
    g.heads = per_wg;
    if (bt == kSub && a.n_kv_heads < per_wg) g.heads = a.n_kv_heads == 3 ? 4 : a.n_kv_heads;
    g.blocks = bt == kSub ? per_wg / g.heads : 1;
    const int64_t longest = a.max_seg_tokens < a.dst_capacity ? a.max_seg_tokens : a.dst_capacity;
    const int64_t blocks = (longest + bt - 2) / bt + 1;   // that so many slots can touch
    g.spots = (int)((blocks + g.blocks - 1) / g.blocks);
    g.tensors = a.src_v ? 2 : 1;
    g.rope_c0 = a.rope_offset / 8;
    g.rope_nc = a.rope_dim / 8;
    const int64_t x = (int64_t)g.spots * g.parts, z = (int64_t)a.n_layers * g.tensors;
    fits = x <= kMaxGridX && z <= 65535;
    return dim3((unsigned)x, (unsigned)a.n_segs, (unsigned)z);
}

}  // namespace

bool store_fits(const StoreArgs& a) {
    StoreGeo g;
    bool fits;
    make_geo(a, g, fits);
    return fits;
}

hipError_t launch_store(const StoreArgs& a, hipStream_t stream) {
    StoreGeo g;
    bool fits;
    const dim3 grid = make_geo(a, g, fits);
    if (!fits) return hipErrorInvalidValue;
    const int subs = a.block_tokens / kSub;
    Freqs f;
    if (a.rows) {   // nothing is turned
        for (int i = 0; i < kPairs; ++i) f.w[i] = 0.0;
    } else if (a.omega) {
        for (int i = 0; i < kPairs; ++i) f.w[i] = i < a.rope_dim / 2 ? a.omega[i] : 0.0;
    } else {
        for (int i = 0; i < kPairs; ++i) f.w[i] = i < a.rope_dim / 2 ? pow(a.theta, -2.0 * i / a.rope_dim) : 0.0;
    }
    if (a.head_dim == 64) {
        if (subs == 1) launch_geo<64, 1>(a, g, f, grid, stream);
        else if (subs == 2) launch_geo<64, 2>(a, g, f, grid, stream);
        else launch_geo<64, 4>(a, g, f, grid, stream);
    } else {
        if (subs == 1) launch_geo<128, 1>(a, g, f, grid, stream);
        else if (subs == 2) launch_geo<128, 2>(a, g, f, grid, stream);
        else launch_geo<128, 4>(a, g, f, grid, stream);
    }
    return hipGetLastError();
}

}  // namespace pkv
