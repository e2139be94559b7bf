// GQA suffix attention for few query rows over a cache held in 8 bits: token-by-token
// generation and short suffixes (paper Sec. 5 "Linear-time TTFT"; Sec. 4 erratum).
//
// The work is shared out as in attn_gqa_rows.hip: workgroups take equal runs of the
// tile axis (attn_columns.h), the waves of a workgroup take its tiles in turn, each
// through LDS stages of its own without a barrier, and are merged at the end.  What
// differs is the tile loop.  A tile of codes is half the bytes of a bf16 one, and a
// wave has half the time for it, which the steps of a tile one after another
// (scores, maximum, probabilities, values) exceed.  So, as in the many-row kernel, the
// score MFMAs of the next tile are interleaved with the probabilities of this one, and
// this one's value MFMAs with the maxima of the next one's scores; codes are turned
// into bf16 one operand ahead of their MFMA.
//
// Bound by the latency of a tile's steps and by HBM: 16 caches of 8448..12544 slots, 32
// heads over 8 KV heads of 128, one query each, 79 us a call, 70 of them in this kernel
// (4.9 TB/s, VALU 23% and MFMA 11% busy) and 5 in the merge; 63 us a call with every page
// in L2; 130 over the bf16 cache.  The first form, one step after another, took 96.
#include <type_traits>

#include "attn_columns.h"
#include "attn_gqa_tile_q8.h"

namespace pkv {
namespace {

// Waves of a workgroup (one a CU) and LDS stages of a wave: two waves a SIMD hide each
// other's latencies, and the loads in flight are the same as with half the waves and twice
// the stages (32 heads over 4 KV heads of 128, 16 caches of 8448..12544 slots: 45.2 us a
// call with four waves of 4 stages, 43.6 with these; 8 KV heads, one cache of 32768: 25.6
// and 25.0; 2 KV heads of 64: 29.7 with four waves of 8, 27.6 with eight of 4, 25.2 with
// these).
constexpr int kRowWaves = 8;
constexpr int kRowStages = 2;
constexpr int kAhead = 3;   // LDS operand reads issued this many operands ahead of their MFMA

__device__ inline int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }

// What the wave's next 64 tiles need of the tables, tile first + l in lane l: the pages of
// K and V (clamped into the pool) and the exponents of their scales, K's in the low byte
// and V's in the next.  Loading it stalls the loop for two dependent loads, once in
// about 60 tiles.
struct TileWindow {
    int first;
    int k_page, v_page, exps;

    template <typename F>
    __device__ __forceinline__ void load(const AttnArgs& a, const BlockScales& s, int seq, int layer, int kvh, int from,
                                         int n_tiles, F key_of) {
        first = from;
        k_page = v_page = exps = 0;
        if (n_tiles <= 0) return;
        const int key = key_of(min(from + (int)__lane_id(), n_tiles - 1));   // (below the slots that the table covers)
        const int64_t entry = (int64_t)seq * a.max_pages + (key >> a.page_shift);
        const int block = (key & ((1 << a.page_shift) - 1)) >> s.block_shift;
        const int top = (int)(a.n_pages - 1);
        k_page = min(max(a.block_table[entry], 0), top);
        v_page = a.v_block_table ? min(max(a.v_block_table[entry], 0), top) : k_page;
        const uint8_t* const k = s.k + layer * s.k_stride[0] + kvh * s.k_stride[1];
        const uint8_t* const v = s.v + layer * s.v_stride[0] + kvh * s.v_stride[1];
        exps = (int)(q8_exponent(k[k_page * s.k_stride[2] + block * s.k_stride[3]]) |
                     q8_exponent(v[v_page * s.v_stride[2] + block * s.v_stride[3]]) << 8);
    }
    __device__ __forceinline__ bool holds(int i) const { return i < first + 64; }   // (tiles are visited in order)
    __device__ __forceinline__ int of(int reg, int i) const { return __builtin_amdgcn_readlane(reg, (i - first) & 63); }
};

__device__ __forceinline__ float q8_k_scale(uint32_t e) { return __uint_as_float((e & 0xffu) << 23); }
__device__ __forceinline__ float q8_v_scale(uint32_t e) { return __uint_as_float((e >> 8) << 23); }

template <int D>
__global__ __launch_bounds__(kRowWaves * 64, 2) void attn_gqa_rows_q8_kernel(AttnArgs a, ColPlan p, BlockScales sa) {
    constexpr int NW = kRowWaves;
    constexpr int NS = kRowStages;
    constexpr int BN = kColTile;           // keys per tile
    constexpr int CH = D / 16;             // 16-byte chunks per row
    constexpr int KBLK = BN * CH / 64;     // LDS-DMA loads per K (or V) tile
    constexpr int KPB = 64 / CH;           // keys per LDS-DMA load
    constexpr int SP = D == 128 ? 2 : 1;   // LDS-DMA loads after which the swizzles repeat
    constexpr int KS = D / 16;             // MFMA k-steps over channels
    constexpr int KR = KS / 2;             // K operand reads: two k-steps each
    constexpr int DB = D / 32;             // 32-channel output blocks
    constexpr int TE = BN * D;             // bytes of one K or V tile
    constexpr int ROWS = 32;               // rows per workgroup
    static_assert((NS & (NS - 1)) == 0 && (2 * NS + 1) * KBLK < 64, "loads in flight within the vmcnt range");
    static_assert(ROWS * D * 4 <= 2 * NS * TE, "a wave's O^T fits its own stages");

    // Per wave: K stages, then V stages; after the loop, its O^T.
    __shared__ __attribute__((aligned(16))) uint8_t stage_lds[NW * 2 * NS * TE];
    __shared__ float row_max_lds[NW][ROWS], row_sum_lds[NW][ROWS];

    const uint32_t column = col_decode(p);
    const int tid = threadIdx.x;
    const int wave = uniform(tid >> 6);
    const int lane = tid & 63;
    const int j = lane & 31;
    const int hl = lane >> 5;
    const int lkey = lane / CH, phys = lane % CH;
    uint8_t* const my_lds = stage_lds + wave * 2 * NS * TE;
    auto kst = [&](int i) __attribute__((always_inline)) -> uint8_t* { return my_lds + (i & (NS - 1)) * TE; };
    auto vst = [&](int i) __attribute__((always_inline)) -> uint8_t* { return my_lds + (NS + (i & (NS - 1))) * TE; };

    int kofs[KR], vofs[DB];
    gqa_operand_offsets_q8<D>(lane, kofs, vofs);
    const float sc2 = fabsf(a.scale == 0.f ? 1.f : a.scale) * kLog2e;   // the sign, or the 0, goes into the queries

    // Touch the tensors that the sequence bounds lead to, so that their address
    // translations are fetched while the bounds are.
    const uint32_t touch = (uint32_t)a.q_pos[0] ^ *(const uint32_t*)a.q ^ (uint32_t)a.block_table[0];
    ColSeqs cs{};
    uint32_t x = 0, x1 = 1;
    if (p.columns) {
        cs = col_seqs(a, p);
        const uint64_t lo = (uint64_t)column * cs.col, axis = (uint64_t)cs.total * p.streams;
        if (lo >= axis) return;   // uniform
        x = (uint32_t)lo;
        x1 = (uint32_t)min(lo + cs.col, axis);
    } else if (column >= (uint32_t)p.streams * (uint32_t)a.n_seqs) {
        return;
    }
    asm volatile("" ::"v"(touch));

    while (x < x1) {
        ColSegment sg;
        if (p.columns) {
            sg = col_segment(cs, p, x, x1, column);
            x += sg.length;
            if (sg.first == sg.last) continue;   // uniform
        } else {
            sg.seq = (int)(column / (uint32_t)p.streams);   // by sequence: neighbours take about equally long
            sg.stream = (int)(column - (uint32_t)sg.seq * (uint32_t)p.streams);
            sg.first = 0;
            sg.last = sg.tiles = 1;
            sg.piece = 0;
            sg.pieces = 1;
            x = x1;
        }
        const int layer = sg.stream / a.n_kv_heads;
        const int kvh = sg.stream - layer * a.n_kv_heads;
        const SeqInfo si = p.columns ? col_seq_info(cs, sg.seq) : seq_info(a, sg.seq);
        const int M = si.nq * p.G;
        if (M <= 0) continue;

        // The lane's row and its Q^T operands (the same in every wave).
        const bool row_ok = j < M;
        const int qi = row_ok ? j / p.G : 0;
        const int pos = a.q_pos[si.q0 + qi], qpos = row_ok ? pos : -1;
        u32x4 qw[KS];
        {
            // rows past M repeat the first (never written)
            const int head = kvh * p.G + (row_ok ? j - qi * p.G : 0);
            const uint16_t* qrow = (const uint16_t*)a.q + (int64_t)layer * a.q_stride[0] +
                                   (int64_t)(si.q0 + qi) * a.q_stride[1] + (int64_t)head * a.q_stride[2];
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) qw[ks] = *(const u32x4*)(qrow + q8_channel(ks, hl));
        }
        int row_start, row_end;
        visible_range(qpos, si.kvl, a.window, row_start, row_end);   // (0, 0) for rows past M
        // Every wave holds every row, so these are the workgroup's bounds.
        const int e_min = wave_min_u(row_ok ? row_end : 0x7fffffff);
        const int e_max = wave_max_u(row_end);
        const int s_min = wave_min_u(row_ok ? row_start : 0x7fffffff);
        const int s_max = wave_max_u(row_start);
        const int lo = s_min == 0x7fffffff ? 0 : s_min / BN * BN;
        const int hi = min(si.kvl, e_max);
        const int real = hi > lo ? (hi - lo + BN - 1) / BN : 0;
        const int t_begin = uniform(col_real_tile(sg.first, sg.tiles, real)) + wave;   // this wave: t_begin, + NW, ...
        const int t_end = uniform(col_real_tile(sg.last, sg.tiles, real));
        const int n_tiles = t_end > t_begin ? (t_end - t_begin + NW - 1) / NW : 0;
        auto key_of = [&](int i) __attribute__((always_inline)) { return lo + (t_begin + i * NW) * BN; };

        const char* const kbase = (const char*)a.k + (int64_t)layer * a.k_stride[0] + (int64_t)kvh * a.k_stride[1];
        const char* const vbase = (const char*)a.v + (int64_t)layer * a.v_stride[0] + (int64_t)kvh * a.v_stride[1];
        const int64_t krow = a.k_stride[2], vrow = a.v_stride[2];   // bytes between keys
        TileWindow win;
        win.load(a, sa, sg.seq, layer, kvh, 0, n_tiles, key_of);
        const int page_mask = (1 << a.page_shift) - 1;

        // LDS-DMA of one tile of one tensor.  Lane l of load b fills LDS chunk
        // slot 64 b + l: key KPB b + l / CH, physical chunk l % CH, holding logical
        // chunk phys ^ swizzle(key).  A tile that runs past the last visible key
        // re-reads that key for the missing rows (masked later).
        uint32_t kchunk[SP], vchunk[SP];
#pragma unroll
        for (int b = 0; b < SP; ++b) {
            kchunk[b] = (uint32_t)(phys ^ swz_k8<D>(b * KPB + lkey)) * 16u;
            vchunk[b] = (uint32_t)(phys ^ swz_v8<D>(b * KPB + lkey)) * 16u;
        }
        auto issue = [&](const char* tile, int64_t row_bytes, int t0, uint8_t* dst, auto v_tag) __attribute__((always_inline)) {
            constexpr bool V = decltype(v_tag)::value;
            const uint32_t lds0 = lds_addr_of(dst);
            if (t0 + BN <= hi) {
                const uint32_t lane_off = (uint32_t)(lkey * row_bytes);
                uint64_t at = uniform_u64((uint64_t)(uintptr_t)tile);
#pragma unroll
                for (int b = 0; b < KBLK; ++b) {
                    lds_dma16(lds0 + b * 1024, (const void*)at, lane_off + (V ? vchunk[b % SP] : kchunk[b % SP]));
                    at += (uint64_t)(KPB * row_bytes);
                    asm volatile("" : "+s"(at));   // step by step: KBLK hoisted offsets would spill scalar registers
                }
            } else {
                int key0 = lkey;
                asm volatile("" : "+v"(key0));   // once per item at most: keep its addresses out of the set-up
#pragma unroll
                for (int b = 0; b < KBLK; ++b)
                    lds_dma16(lds0 + b * 1024, tile, (uint32_t)(min(b * KPB + key0, hi - 1 - t0) * row_bytes) +
                                                        (V ? vchunk[b % SP] : kchunk[b % SP]));
            }
        };
        auto issue_k = [&](int i) __attribute__((always_inline)) {
            const int t0 = key_of(i);
            issue(kbase + win.of(win.k_page, i) * a.k_page_stride + (t0 & page_mask) * krow, krow, t0, kst(i), std::false_type{});
        };
        auto issue_v = [&](int i) __attribute__((always_inline)) {
            const int t0 = key_of(i);
            issue(vbase + win.of(win.v_page, i) * a.v_page_stride + (t0 & page_mask) * vrow, vrow, t0, vst(i), std::true_type{});
        };
#pragma unroll 1
        for (int i = 0; i < min(NS, n_tiles); ++i) {
            issue_k(i);
            issue_v(i);
        }

        // The scale's sign, or a scale of 0, applied to the queries: exact, and the scores' largest is
        // their maximum whatever the scale.
        bf16x8 qf[KS];
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            u32x4 w = qw[ks];
            if (a.scale < 0.f) {
#pragma unroll
                for (int i = 0; i < 4; ++i) w[i] ^= 0x80008000u;
            }
            qf[ks] = __builtin_bit_cast(bf16x8, w);
            if (a.scale == 0.f) {
#pragma unroll
                for (int i = 0; i < 8; ++i) qf[ks][i] = (__bf16)((float)qf[ks][i] * 0.f);
            }
        }

        f32x16 o[DB];
#pragma unroll
        for (int db = 0; db < DB; ++db) o[db] = f32x16{};
        // The reference maximum starts below every finite score but finite, so that scores
        // of -inf (hidden keys among them) have weights exp2(-inf) = 0.
        float m_run = -__FLT_MAX__, l_run = 0.f;
        auto lds_reads_done = []() __attribute__((always_inline)) {
            __builtin_amdgcn_s_waitcnt(15 | (7 << 4) | (0 << 8) | (3 << 14));
            asm volatile("" ::: "memory");
        };
        auto masked = [&](int t0) __attribute__((always_inline)) { return t0 + BN > e_min || t0 < s_max; };
        auto hide = [&](int t0, f32x16& s) __attribute__((always_inline)) {
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int key = t0 + (r >> 2) * 8 + hl * 4 + (r & 3);
                if (key >= row_end || key < row_start) s[r] = -INFINITY;
            }
        };
        // Largest score of a row (lanes l and l + 32 hold its keys); a NaN is passed over.
        auto both = [&](float m) __attribute__((always_inline)) {
            const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(m), __float_as_uint(m), false, false);
            return fmaxf(__uint_as_float(sw[0]), __uint_as_float(sw[1]));
        };
        // The reference moves when a tile's maximum exceeds it by more than kLazy, so most
        // tiles leave O alone (probabilities stay below 2^kLazy).
        constexpr float kLazy = 8.0f;
        auto move_max = [&](float mx) __attribute__((always_inline)) {
            const float msc = mx * sc2;
            const bool up = msc > m_run + kLazy;
            if (__builtin_amdgcn_ballot_w64(up) != 0) {
                const float m_new = up ? msc : m_run;
                const float alpha = __builtin_amdgcn_exp2f(m_run - m_new);
                l_run *= alpha;
#pragma unroll
                for (int db = 0; db < DB; ++db) o[db] *= alpha;
                m_run = m_new;
            }
        };
        auto k_value = [&](const u32x4& w, int ks, uint32_t es) __attribute__((always_inline)) {
            return q8_to_bf16(w[(ks & 1) * 2], w[(ks & 1) * 2 + 1], q8_k_scale(es));
        };
        auto probability = [&](float s) __attribute__((always_inline)) {
            return __builtin_amdgcn_exp2f(fmaf(s, sc2, -m_run));
        };

        // Scores of the tile in K stage ks_src; with CUR, interleaved with the probabilities of cur (into
        // pb): groups of one k-step's MFMA, its share of the exponentials, the next operand's conversion and
        // the read kAhead reads ahead.
        auto seg1 = [&](const uint8_t* ks_src, uint32_t es, f32x16& cur, f32x16& nxt, bf16x8 (&pb)[2],
                        auto cur_tag) __attribute__((always_inline)) {
            constexpr bool CUR = decltype(cur_tag)::value;
            constexpr int A = kAhead < KR ? kAhead : KR;
            constexpr int PER_K = 16 / KS;
            u32x4 kop[KR];
#pragma unroll
            for (int q = 0; q < A; ++q) kop[q] = *(const u32x4*)(ks_src + kofs[q]);
            __builtin_amdgcn_sched_barrier(0);
            bf16x8 kf = k_value(kop[0], 0, es);
#pragma unroll
            for (int q = 0; q < KS; ++q) {
                nxt = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, qf[q], q == 0 ? f32x16{} : nxt, 0, 0, 0);
                if (CUR) {
#pragma unroll
                    for (int r = q * PER_K; r < (q + 1) * PER_K; ++r) cur[r] = probability(cur[r]);
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        if ((q + 1) * PER_K == 8 * (h + 1)) {
                            f32x8 pv8;
#pragma unroll
                            for (int e = 0; e < 8; ++e) pv8[e] = cur[h * 8 + e];
                            pb[h] = __builtin_convertvector(pv8, bf16x8);
                        }
                    }
                }
                if (q % 2 == 1 && q / 2 + A < KR) kop[q / 2 + A] = *(const u32x4*)(ks_src + kofs[q / 2 + A]);
                if (q + 1 < KS) kf = k_value(kop[(q + 1) / 2], q + 1, es);
                __builtin_amdgcn_sched_barrier(0);
            }
        };
        // O^T += V^T P^T of the tile in V stage vs_src, interleaved with the row sums of pb (the
        // probabilities as they enter PV: the rounding of a key that dominates its row cancels) and, with
        // NXT, the maximum of nxt's scores.
        auto seg2 = [&](const uint8_t* vs_src, uint32_t es, const bf16x8 (&pb)[2], const f32x16& nxt,
                        auto nxt_tag) __attribute__((always_inline)) {
            constexpr bool NXT = decltype(nxt_tag)::value;
            constexpr int NQ = 2 * DB;
            constexpr int A = kAhead < NQ ? kAhead : NQ;
            constexpr int PER_M = 16 / NQ, PER_D = 8 / NQ;
            const bf16x2 ones = {(__bf16)1.0f, (__bf16)1.0f};
            u32x2 vop[NQ];
            auto read = [&](int q) __attribute__((always_inline)) { return q8_v_read(vs_src + vofs[q % DB] + (q / DB) * 16 * D); };
#pragma unroll
            for (int q = 0; q < A; ++q) vop[q] = read(q);
            __builtin_amdgcn_sched_barrier(0);
            float m0 = -INFINITY, m1 = -INFINITY, l0 = 0.f, l1 = 0.f;
            bf16x8 vf = q8_to_bf16(vop[0][0], vop[0][1], q8_v_scale(es));
#pragma unroll
            for (int q = 0; q < NQ; ++q) {
                o[q % DB] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, pb[q / DB], o[q % DB], 0, 0, 0);
                if (NXT) {
#pragma unroll
                    for (int r = q * PER_M; r < (q + 1) * PER_M; r += 2) {
                        m0 = fmaxf(m0, nxt[r]);
                        m1 = fmaxf(m1, nxt[r + 1]);
                    }
                }
#pragma unroll
                for (int d = q * PER_D; d < (q + 1) * PER_D; ++d) {
                    const bf16x8 pp = pb[d >> 2];
                    const int e = (d & 3) * 2;
                    if (d & 1) l1 = __builtin_amdgcn_fdot2_f32_bf16((bf16x2){pp[e], pp[e + 1]}, ones, l1, false);
                    else l0 = __builtin_amdgcn_fdot2_f32_bf16((bf16x2){pp[e], pp[e + 1]}, ones, l0, false);
                }
                if (q + A < NQ) vop[q + A] = read(q + A);
                if (q + 1 < NQ) vf = q8_to_bf16(vop[q + 1][0], vop[q + 1][1], q8_v_scale(es));
                __builtin_amdgcn_sched_barrier(0);
            }
            l_run += l0 + l1;
            return fmaxf(m0, m1);
        };
        // A masked tile must not bring NaN values (0 * NaN): its NaN codes are cleared in V stage vs_src, and
        // come back, to the rows that see them, at the end of the item.
        bool left_out = false;
        auto leave_out_nan = [&](uint8_t* vs_src) __attribute__((always_inline)) {
            u32x4 w[TE / 1024];
            uint32_t nans = 0;
#pragma unroll
            for (int n = 0; n < TE / 1024; ++n) {
                w[n] = *(const u32x4*)(vs_src + (n * 64 + lane) * 16);
#pragma unroll
                for (int e = 0; e < 4; ++e) nans |= q8_nan_bytes(w[n][e]);
            }
            if (__builtin_amdgcn_ballot_w64(nans != 0) == 0) return;
            left_out = true;
#pragma unroll
            for (int n = 0; n < TE / 1024; ++n) {
#pragma unroll
                for (int e = 0; e < 4; ++e) w[n][e] &= ~((q8_nan_bytes(w[n][e]) >> 7) * 0xffu);
                *(u32x4*)(vs_src + (n * 64 + lane) * 16) = w[n];
            }
            asm volatile("" ::: "memory");
        };

        // Loads retire in order: K(0), V(0), .., K(NS-1), V(NS-1), K(NS) once tile 0's scores are read, then
        // K(i+1+NS) and V(i+NS) in step i, which needs K(i+1) and V(i).  With `rem` tiles behind tile i, those
        // issued later are the K of at most NS - 1 of the tiles behind i + 1 and the V of NS - 1 behind i.
        auto wait_step = [&](int rem) __attribute__((always_inline)) {
            if (rem >= NS) {
                wait_vmcnt<2 * (NS - 1) * KBLK>();
            } else {
                static_for<0, NS>([&](auto k_tag) {
                    constexpr int K = decltype(k_tag)::value;
                    if (rem == K) wait_vmcnt<(K + (K > 0 ? K - 1 : 0)) * KBLK>();
                });
            }
            asm volatile("" ::: "memory");
        };
        uint32_t es_cur = 0;   // exponents of the tile whose scores are held
        auto all_probabilities = [&](const f32x16& s, bf16x8 (&pb)[2]) __attribute__((always_inline)) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                f32x8 pv8;
#pragma unroll
                for (int e = 0; e < 8; ++e) pv8[e] = probability(s[h * 8 + e]);
                pb[h] = __builtin_convertvector(pv8, bf16x8);
            }
        };
        auto maximum = [&](const f32x16& s) __attribute__((always_inline)) {
            float mx = s[0];
#pragma unroll
            for (int r = 1; r < 16; ++r) mx = fmaxf(mx, s[r]);
            return mx;
        };
        // Tile i's probabilities and values, and the scores of tile i + 1; tile i has no hidden key.
        auto step = [&](int i, f32x16& cur, f32x16& nxt) __attribute__((always_inline)) {
            wait_step(n_tiles - 1 - i);
            const uint32_t es = win.of(win.exps, i + 1);
            bf16x8 pb[2];
            seg1(kst(i + 1), es, cur, nxt, pb, std::true_type{});
            lds_reads_done();
            if (i + 1 + NS < n_tiles) issue_k(i + 1 + NS);
            if (masked(key_of(i + 1))) hide(key_of(i + 1), nxt);
            const float mx = seg2(vst(i), es_cur, pb, nxt, std::true_type{});
            lds_reads_done();
            if (i + NS < n_tiles) issue_v(i + NS);
            es_cur = es;
            move_max(both(mx));
        };
        // The same for any tile, the last one too, without overlap.
        auto plain = [&](int i, f32x16& cur) __attribute__((always_inline)) {
            wait_step(n_tiles - 1 - i);
            bf16x8 pb[2];
            all_probabilities(cur, pb);
            if (masked(key_of(i))) leave_out_nan(vst(i));
            seg2(vst(i), es_cur, pb, cur, std::false_type{});
            lds_reads_done();
            if (i + 1 >= n_tiles) return;
            es_cur = win.of(win.exps, i + 1);
            bf16x8 none[2];
            seg1(kst(i + 1), es_cur, cur, cur, none, std::false_type{});
            lds_reads_done();
            if (i + 1 + NS < n_tiles) issue_k(i + 1 + NS);
            if (i + NS < n_tiles) issue_v(i + NS);
            if (masked(key_of(i + 1))) hide(key_of(i + 1), cur);
            move_max(both(maximum(cur)));
        };
        if (n_tiles > 0) {
            f32x16 s_a, s_b;
            bf16x8 none[2];
            es_cur = win.of(win.exps, 0);
            if (n_tiles >= NS) wait_vmcnt<(2 * NS - 1) * KBLK>();
            else static_for<1, NS>([&](auto k_tag) {
                constexpr int K = decltype(k_tag)::value;
                if (n_tiles == K) wait_vmcnt<(2 * K - 1) * KBLK>();
            });
            asm volatile("" ::: "memory");
            seg1(kst(0), es_cur, s_b, s_a, none, std::false_type{});
            lds_reads_done();
            if (NS < n_tiles) issue_k(NS);
            if (masked(key_of(0))) hide(key_of(0), s_a);
            move_max(both(maximum(s_a)));
            // Tiles with hidden keys come first (a window's start) and last.
#pragma unroll 1
            for (int i = 0; i < n_tiles; ++i) {
                auto more_tiles = [&]() __attribute__((always_inline)) {
                    if (!win.holds(i + 1 + NS)) win.load(a, sa, sg.seq, layer, kvh, i, n_tiles, key_of);
                };
                // A loop of their own, two steps a round: where the two kinds of step meet, and where the
                // scores change places, whole tiles of registers would be moved.
#pragma unroll 1
                for (; i + 1 < n_tiles && !masked(key_of(i)); ++i) {
                    more_tiles();
                    step(i, s_a, s_b);
                    if (!(++i + 1 < n_tiles && !masked(key_of(i)))) {
                        s_a = s_b;
                        break;
                    }
                    more_tiles();
                    step(i, s_b, s_a);
                }
                more_tiles();
                plain(i, s_a);
            }
            if (left_out) {   // where the NaN values are times the keys' visibility, over the masked tiles once more
#pragma unroll 1
                for (int i = 0; i < n_tiles; ++i) {
                    const int t0 = key_of(i);
                    if (!masked(t0)) continue;
                    win.load(a, sa, sg.seq, layer, kvh, i, n_tiles, key_of);
                    issue_v(i);
                    wait_vmcnt<0>();
                    asm volatile("" ::: "memory");
#pragma unroll 1
                    for (int st = 0; st < 2; ++st) {
                        f32x8 seen;
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            const int key = t0 + st * 16 + (e >> 2) * 8 + hl * 4 + (e & 3);
                            seen[e] = key < row_end && key >= row_start ? 1.0f : 0.0f;
                        }
                        const bf16x8 sees = __builtin_convertvector(seen, bf16x8);
#pragma unroll
                        for (int db = 0; db < DB; ++db) {
                            const u32x2 w = q8_v_read(vst(i) + vofs[db] + st * 16 * D);
                            const bf16x8 nan = q8_to_bf16((q8_nan_bytes(w[0]) >> 7) * 0x38u, (q8_nan_bytes(w[1]) >> 7) * 0x38u, 1.0f);
                            const f32x16 n = __builtin_amdgcn_mfma_f32_32x32x16_bf16(nan, sees, f32x16{}, 0, 0, 0);
#pragma unroll
                            for (int r = 0; r < 16; ++r) o[db][r] = n[r] > 0.f ? __builtin_nanf("") : o[db][r];
                            __builtin_amdgcn_sched_barrier(0);
                        }
                    }
                    lds_reads_done();
                }
            }
        }

        // Merge the waves: O^T to this wave's stages (row-major fp32,
        // 16-byte chunks XOR-swizzled by row), maxima and sums beside.
        constexpr int OC = D / 4;   // 16-byte fp32 chunks per row
        float* const my_o = (float*)my_lds;
        const float l_tot = l_run + __shfl_xor(l_run, 32);
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
            for (int b = 0; b < 4; ++b)
                *(f32x4*)(my_o + j * D + ((db * 8 + b * 2 + hl) ^ (j & (OC - 1))) * 4) =
                    f32x4{o[db][4 * b], o[db][4 * b + 1], o[db][4 * b + 2], o[db][4 * b + 3]};
        if (hl == 0) {
            row_max_lds[wave][j] = m_run;
            row_sum_lds[wave][j] = l_tot;
        }
        __syncthreads();
        col_merge_rows<NW, ROWS, D>(a, p, sg, si, layer, kvh * p.G, p.G, M, (const float*)stage_lds, 2 * NS * TE / 4,
                                    &row_max_lds[0][0], &row_sum_lds[0][0]);
        __syncthreads();   // the stages are free for the next item
    }
}

}  // namespace

hipError_t launch_attn_gqa_rows_q8(const AttnArgs& a, const ColPlan& p, const BlockScales& scales, dim3 grid,
                                   hipStream_t stream) {
    if (a.head_dim == 64)
        hipLaunchKernelGGL((attn_gqa_rows_q8_kernel<64>), grid, dim3(kRowWaves * 64), 0, stream, a, p, scales);
    else
        hipLaunchKernelGGL((attn_gqa_rows_q8_kernel<128>), grid, dim3(kRowWaves * 64), 0, stream, a, p, scales);
    return hipGetLastError();
}

}  // namespace pkv
