// Attention for trees of drafted tokens: the second of two steps.
//
// A drafted row sees the slots of its cache and, among the drafted rows of its
// sequence, its ancestors and itself; those rows' keys lie beside the cache until they
// are accepted.  The first step is suffix attention over the cache, whose kernels read
// every key once for all rows of the tree and leave normalised partials and their
// log2-sum-exps in the workspace.  This step joins a row's partials with its visible
// drafted rows by one running softmax: a partial enters like a key whose score is its
// log-sum-exp, with the partial's output in the place of a value.
//
// A tree's row sees few drafted rows (its depth, not the size of the tree), so a wave,
// which holds one row of one head, lists the set bits of the row's mask and loads only
// those keys and values: scores, sums and outputs stay in fp32 registers.  Head sizes
// 64 and 128: CH = D/8 lanes share a key (or a partial), KG = 64 / CH groups of lanes
// take U keys each at a time, and are merged at the end.  Latent rows (576 channels):
// the whole wave shares a key, whose first 512 channels are its value.
// The step is a chain of memory round trips (bounds; log-sum-exps, mask and query;
// partials, keys and values), so what does not depend on each other is asked for together:
// 3.5 us for one tree of 8 rows of 14 heads, 6.4 for 16 of 8 of 32. Beyond that it is bound by
// the records it reads (16 trees of up to 32 rows of 32 heads, 11.4 us).
#include "attn_columns.h"
#include "attn_gqa_tile.h"

namespace pkv {
namespace {

constexpr int kJoinWaves = 4;
constexpr int kJoinKeys = 2;

// Eight values as they lie in memory, and as floats.
template <typename T>
struct Raw8;
template <>
struct Raw8<float> {
    f32x4 a, b;
    __device__ __forceinline__ void load(const char* p) {
        a = *(const f32x4*)p;
        b = *(const f32x4*)(p + 16);
    }
    __device__ __forceinline__ void get(float (&x)[8]) const {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            x[e] = a[e];
            x[4 + e] = b[e];
        }
    }
};
template <>
struct Raw8<uint16_t> {
    u32x4 a;
    __device__ __forceinline__ void load(const char* p) { a = *(const u32x4*)p; }
    __device__ __forceinline__ void get(float (&x)[8]) const {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            x[2 * e] = __uint_as_float(a[e] << 16);
            x[2 * e + 1] = __uint_as_float(a[e] & 0xffff0000u);
        }
    }
};
__device__ __forceinline__ float load1(const float* p) { return *p; }
__device__ __forceinline__ float load1(const uint16_t* p) { return __uint_as_float((uint32_t)*p << 16); }

// Sum over the CH lanes that share a key, the same in each of them.
template <int CTRL>
__device__ __forceinline__ float dpp_add(float v) {
    return v + __uint_as_float((uint32_t)dpp<CTRL>(0, (int)__float_as_uint(v)));
}
template <int CH>
__device__ __forceinline__ float group_sum(float v) {
    if constexpr (CH == 8) {
        constexpr int kSwap1 = 0xb1, kSwap2 = 0x4e, kHalfMirror = 0x141;   // quad_perm [1,0,3,2], [2,3,0,1]; lane 7 - i of 8
        return dpp_add<kHalfMirror>(dpp_add<kSwap2>(dpp_add<kSwap1>(v)));
    } else {
        v = dpp_add<kDppRor + 1>(dpp_add<kDppRor + 2>(dpp_add<kDppRor + 4>(dpp_add<kDppRor + 8>(v))));
        if constexpr (CH == 16) return v;
        float r[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) r[k] = __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(v), 16 * k));
        return (r[0] + r[1]) + (r[2] + r[3]);
    }
}
__device__ __forceinline__ float lane_value(float v, int lane) {
    return __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(v), lane));
}
template <int CTRL>
__device__ __forceinline__ float dpp_max(float v) {
    return fmaxf(v, __uint_as_float((uint32_t)dpp<CTRL>((int)__float_as_uint(v), (int)__float_as_uint(v))));
}
__device__ __forceinline__ float wave_max_f(float v) {   // a NaN counts for nothing
    v = dpp_max<kDppRor + 1>(dpp_max<kDppRor + 2>(dpp_max<kDppRor + 4>(dpp_max<kDppRor + 8>(v))));
    return fmaxf(fmaxf(lane_value(v, 0), lane_value(v, 16)), fmaxf(lane_value(v, 32), lane_value(v, 48)));
}
// v of this lane and of the one in the other half (32) or the neighbouring row of 16 lanes.
template <int W>
__device__ __forceinline__ void both(float v, float& x, float& y) {
    const uint32_t u = __float_as_uint(v);
    const auto r = W == 32 ? __builtin_amdgcn_permlane32_swap(u, u, false, false) : __builtin_amdgcn_permlane16_swap(u, u, false, false);
    x = __uint_as_float(r[0]);
    y = __uint_as_float(r[1]);
}
// Sums over the same two lanes: of v in the lower, of w in the upper one.
template <int W>
__device__ __forceinline__ float scatter_sum(float v, float w) {
    const uint32_t a = __float_as_uint(v), b = __float_as_uint(w);
    const auto r = W == 32 ? __builtin_amdgcn_permlane32_swap(a, b, false, false) : __builtin_amdgcn_permlane16_swap(a, b, false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

template <typename T, int D>
__global__ __launch_bounds__(kJoinWaves * 64) void tree_join(AttnArgs a, DraftArgs d, int seq0) {
    constexpr bool MLA = D == 576;
    constexpr int DV = MLA ? 512 : D;
    constexpr int CH = DV / 8;          // lanes per key
    constexpr int KG = 64 / CH;         // groups of lanes
    constexpr int U = kJoinKeys;        // keys (partials) of a group at a time
    // The arguments of the set-up are asked for together, not one round trip after another.
    asm volatile("" ::"s"(a.cu_q), "s"(a.total_q), "s"(a.max_q), "s"(a.n_heads), "s"(a.n_kv_heads), "s"(a.n_layers), "s"(a.n_splits),
                 "s"(a.ws_lse), "s"(a.ws_o), "s"(a.q), "s"(a.q_stride[0]), "s"(a.q_stride[1]), "s"(a.q_stride[2]), "s"(a.window));
    asm volatile("" ::"s"(d.mask), "s"(d.mask_words), "s"(d.k), "s"(d.v), "s"(d.k_stride[0]), "s"(d.k_stride[1]), "s"(d.k_stride[2]),
                 "s"(d.v_stride[0]), "s"(d.v_stride[1]), "s"(d.v_stride[2]), "s"(a.scale));
    const int lane = threadIdx.x & 63;
    const int kg = lane / CH, c = lane % CH;
    const uint32_t unit = blockIdx.x * kJoinWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int i = (int)(unit / (uint32_t)a.n_heads), head = (int)(unit - (uint32_t)i * (uint32_t)a.n_heads);
    const int seq = seq0 + (int)blockIdx.y;
    const int layer = (int)blockIdx.z;
    int q0 = 0, nq = a.total_q;
    if (a.cu_q) {
        q0 = a.cu_q[seq];
        nq = a.cu_q[seq + 1] - q0;
    }
    if (q0 < 0 || nq < 0 || (int64_t)q0 + nq > a.total_q) nq = 0;   // as seq_info
    if (i >= nq || i >= a.max_q) return;
    const int kvh = head / (a.n_heads / a.n_kv_heads);
    const int64_t row = q0 + i;
    const int64_t items = (int64_t)a.n_layers * a.total_q * a.n_heads;
    const int64_t item = ((int64_t)layer * a.total_q + row) * a.n_heads + head;

    // The first records' log-sum-exps, one a lane; the query; 64 columns of the mask, one a lane.
    const int ns = a.n_splits;
    float lse = lane < ns ? a.ws_lse[lane * items + item] : -INFINITY;
    const char* const qrow = (const char*)((const T*)a.q + (int64_t)layer * a.q_stride[0] + row * a.q_stride[1] + (int64_t)head * a.q_stride[2]);
    Raw8<T> q_raw;
    q_raw.load(qrow + c * (8 * sizeof(T)));
    const float q_rope = MLA ? load1((const T*)qrow + 512 + c) : 0.f;
    const int64_t pos = a.window > 0 ? a.q_pos[row] : 0;
    auto columns = [&](int b) __attribute__((always_inline)) -> uint64_t {   // columns 64 b .. of the row's mask
        const int col = b * 64 + lane;
        bool seen = col < nq;                                                 // no rows behind the sequence
        if (d.mask) {
            const int w = col >> 5;
            const uint32_t word = w < d.mask_words ? d.mask[row * d.mask_words + w] : 0u;
            seen = seen && ((word >> (col & 31)) & 1);
        } else {
            seen = seen && col <= i;
        }
        if (a.window > 0 && seen) seen = a.q_pos[q0 + col] > pos - a.window;
        return __builtin_amdgcn_ballot_w64(seen);
    };
    uint64_t seen = columns(0);

    constexpr int EB = sizeof(T);
    const char* const k0 = (const char*)d.k + ((int64_t)layer * d.k_stride[0] + (int64_t)kvh * d.k_stride[1] + q0 * d.k_stride[2]) * EB;
    const char* const v0 = (const char*)d.v + ((int64_t)layer * d.v_stride[0] + (int64_t)kvh * d.v_stride[1] + q0 * d.v_stride[2]) * EB;
    const uint32_t k_row = (uint32_t)d.k_stride[2] * EB, v_row = (uint32_t)d.v_stride[2] * EB;   // (64 MiB at most)
    const float sc2 = a.scale * kLog2e;
    // The places of the set bits: entry x in lane x.  (Lanes without a bit send theirs behind.)
    auto list_of = [&](uint64_t bits) __attribute__((always_inline)) {
        const int rank = __builtin_amdgcn_mbcnt_hi((uint32_t)(bits >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)bits, 0));
        const int to = (bits >> lane) & 1 ? rank : __builtin_popcountll(bits) + lane - rank;
        return __builtin_amdgcn_ds_permute(to * 4, lane);
    };
    auto entry = [&](int list, int x) __attribute__((always_inline)) {
        return KG == 1 ? __builtin_amdgcn_readlane(list, x & 63) : __builtin_amdgcn_ds_bpermute(x * 4, list);
    };
    // Entries x0 + KG u + kg of a list, u < U, in each group of lanes.  Behind the list's
    // end its last entry is loaded again (and weighs nothing); a u of which no group has an entry is left out.
    Raw8<T> k_raw[U], v_raw[U];
    float k_rope[U];
    auto load_keys = [&](int list, int count, int b, int x0) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (x0 + u * KG < count) {   // uniform
                const uint32_t r = b * 64 + entry(list, min(x0 + u * KG + kg, count - 1));
                const char* const k = k0 + (uint64_t)r * k_row;
                k_raw[u].load(k + c * (8 * EB));
                if constexpr (MLA) k_rope[u] = load1((const T*)k + 512 + c);
                else v_raw[u].load(v0 + (uint64_t)r * v_row + c * (8 * EB));
            }
        }
    };
    int list = list_of(seen), count = __builtin_popcountll(seen);

    // The cache's partials: weights relative to the largest of 64 records, each group of
    // lanes sums its share.  A NaN log-sum-exp makes the sum NaN, and so the row.
    float m = -INFINITY, l = 0.f, acc[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) acc[e] = 0.f;
    const uint64_t rec_bytes = (uint64_t)items * (DV * 4);
    int recs, n_recs;        // records with a weight (a list), how many, and the weights by record
    float w;
    auto weigh = [&](float lse) __attribute__((always_inline)) {
        const uint64_t used = __builtin_amdgcn_ballot_w64(lse != -INFINITY);
        recs = list_of(used);
        n_recs = __builtin_popcountll(used);
        const float m_new = fmaxf(m, wave_max_f(lse));
        w = lse == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(lse - m_new);
        return m_new;
    };
    Raw8<float> x[U];
    float wu[U];
    auto load_records = [&](int s0, int x0) __attribute__((always_inline)) {
        const char* const o0 = (const char*)(a.ws_o + (s0 * items + item) * DV + c * 8);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (x0 + u * KG < n_recs) {
                const int at = x0 + u * KG + kg;
                const int rec = entry(recs, min(at, n_recs - 1));
                const float weight = __uint_as_float((uint32_t)entry((int)__float_as_uint(w), rec));
                wu[u] = at < n_recs ? weight : 0.f;
                x[u].load(o0 + (uint32_t)rec * rec_bytes);
            }
        }
    };
    auto add_records = [&](int x0) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (x0 + u * KG < n_recs) {
                const bool in = x0 + u * KG + kg < n_recs;
                float v[8];
                x[u].get(v);
                l += wu[u];
#pragma unroll
                for (int e = 0; e < 8; ++e) acc[e] = fmaf(wu[u], in ? v[e] : 0.f, acc[e]);
            }
        }
    };
    m = weigh(lse);
    load_records(0, 0);
    load_keys(list, count, 0, 0);
    add_records(0);
    for (int x0 = KG * U; x0 < n_recs; x0 += KG * U) {
        load_records(0, x0);
        add_records(x0);
    }
    for (int s0 = 64; s0 < ns; s0 += 64) {   // (many splits, by the caller's choice)
        lse = s0 + lane < ns ? a.ws_lse[(int64_t)(s0 + lane) * items + item] : -INFINITY;
        const float m_new = weigh(lse);
        const float keep = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - m_new);
        l *= keep;
#pragma unroll
        for (int e = 0; e < 8; ++e) acc[e] *= keep;
        m = m_new;
        for (int x0 = 0; x0 < n_recs; x0 += KG * U) {
            load_records(s0, x0);
            add_records(x0);
        }
    }

    // The drafted rows it sees.
    float q[8];
    q_raw.get(q);
    auto add_keys = [&](int count, int x0) __attribute__((always_inline)) {
        float s[U], top = m;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            s[u] = -INFINITY;
            if (x0 + u * KG < count) {
                float k[8], x = MLA ? q_rope * k_rope[u] : 0.f;
                k_raw[u].get(k);
#pragma unroll
                for (int e = 0; e < 8; ++e) x = fmaf(q[e], k[e], x);
                x = group_sum<CH>(x) * sc2;
                if (x0 + u * KG + kg < count) s[u] = x;
                top = fmaxf(top, s[u]);
            }
        }
        const float keep = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - top);
        l *= keep;
#pragma unroll
        for (int e = 0; e < 8; ++e) acc[e] *= keep;
        m = top;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (x0 + u * KG < count) {
                const bool weighs = s[u] != -INFINITY;   // (a score of -inf: nothing, whatever the value)
                const float p = weighs ? __builtin_amdgcn_exp2f(s[u] - top) : 0.f;
                float v[8];
                if constexpr (MLA) k_raw[u].get(v);
                else v_raw[u].get(v);
                l += p;
#pragma unroll
                for (int e = 0; e < 8; ++e) acc[e] = fmaf(p, weighs ? v[e] : 0.f, acc[e]);
            }
        }
    };
    if (count > 0) add_keys(count, 0);
    for (int b = 0;;) {
        for (int x0 = b == 0 ? KG * U : 0; x0 < count; x0 += KG * U) {
            load_keys(list, count, b, x0);
            add_keys(count, x0);
        }
        if (++b * 64 >= (d.mask ? nq : i + 1)) break;
        seen = columns(b);
        list = list_of(seen);
        count = __builtin_popcountll(seen);
    }

    // The groups of lanes hold disjoint entries: their sums, relative to the largest
    // maximum, are added and dealt out at once, so that a lane ends with `OUT` channels.
    constexpr int OUT = MLA ? 8 : 2;
    if constexpr (!MLA) {
        float x, y, top;
        both<32>(m, x, y);
        both<16>(fmaxf(x, y), x, y);
        top = fmaxf(x, y);
        if constexpr (CH == 8) top = dpp_max<kDppRor + 8>(top);
        const float r = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - top);
        m = top;
        both<32>(l * r, x, y);
        both<16>(x + y, x, y);
        l = x + y;
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[e] = scatter_sum<32>(acc[e] * r, acc[4 + e] * r);
#pragma unroll
        for (int e = 0; e < 2; ++e) acc[e] = scatter_sum<16>(acc[e], acc[2 + e]);
        if constexpr (CH == 8) {
            l = dpp_add<kDppRor + 8>(l);
            acc[0] = dpp_add<kDppRor + 8>(acc[0]);
            acc[1] = dpp_add<kDppRor + 8>(acc[1]);
            if (lane & 8) return;   // the row's other half has the same
        }
    }
    const float inv = row_inverse(l);
    // Channels of the lane: the upper half and the odd rows of lanes hold the later ones.
    const int at = c * 8 + (MLA ? 0 : (lane >> 5) * 4 + ((lane >> 4) & 1) * 2);
    T* const dst = (T*)a.out + (int64_t)layer * a.o_stride[0] + row * a.o_stride[1] + (int64_t)head * a.o_stride[2] + at;
    if constexpr (sizeof(T) == 4) {
        typedef float f32x2 __attribute__((ext_vector_type(2)));
        *(f32x2*)dst = f32x2{acc[0] * inv, acc[1] * inv};
    } else {
        uint32_t o[OUT / 2];
#pragma unroll
        for (int e = 0; e < OUT / 2; ++e) o[e] = bf_rne(acc[2 * e] * inv) | (bf_rne(acc[2 * e + 1] * inv) << 16);
        if constexpr (MLA) *(u32x4*)dst = u32x4{o[0], o[1], o[2], o[3]};
        else *(uint32_t*)dst = o[0];
    }
    if (a.lse_out && lane == 0) a.lse_out[item] = row_lse2(m, l) * kLn2;
}

// The weight in a tile of a drafted row that is not seen, or whose score is -inf (of others: +0 or more).
constexpr float kUnseen = -0.f;

// The same for many rows of bf16 heads: a workgroup takes 128 (row, head-in-group) rows
// of one KV head, 32 a wave, and the drafted rows 32 at a time through LDS and the
// matrix cores, in the layouts of the many-row attention kernels (S^T = K Q^T, then
// O^T += V^T P^T with probabilities rounded to bf16, as over the cache).  Above, a thousand
// rows of a head cost about 0.7 us, most of it instructions; here keys, values and masks are
// read once for 128 rows.
// A value that is no finite number is left out of the tile (0 * inf would reach rows
// that do not see it) and added by hand to the rows that do, also where the weight of a
// row that sees it vanishes (NaN then, as above).
template <int D>
__global__ __launch_bounds__(256, 2) void tree_join_tiles(AttnArgs a, DraftArgs d, int seq0) {
    constexpr int BN = 32, KS = D / 16, DB = D / 32, CH = D / 8;
    constexpr int PER = BN * CH / 256;     // 16-byte chunks of a tile a thread stages
    __shared__ __attribute__((aligned(16))) uint16_t k_lds[BN * D], v_lds[BN * D];
    __shared__ uint32_t odd_keys[2];       // keys of the tile with values that were left out
    const int tid = threadIdx.x, lane = tid & 63, j = lane & 31, hl = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int seq = seq0 + (int)blockIdx.y, layer = (int)blockIdx.z / a.n_kv_heads, kvh = (int)blockIdx.z - layer * a.n_kv_heads;
    int q0 = 0, nq = a.total_q;
    if (a.cu_q) {
        q0 = a.cu_q[seq];
        nq = a.cu_q[seq + 1] - q0;
    }
    if (q0 < 0 || nq < 0 || (int64_t)q0 + nq > a.total_q) nq = 0;   // as seq_info
    const int G = a.n_heads / a.n_kv_heads, M = min(nq, a.max_q) * G, m0 = (int)blockIdx.x * 128;
    if (m0 >= M) return;   // uniform
    const int m = m0 + wave * 32 + j;
    const bool row_ok = m < M;
    const int i = row_ok ? m / G : 0, head = kvh * G + (row_ok ? m - i * G : 0);   // rows past M repeat row 0 (never written)
    const int64_t row = q0 + i;
    const int64_t items = (int64_t)a.n_layers * a.total_q * a.n_heads;
    const int64_t item = ((int64_t)layer * a.total_q + row) * a.n_heads + head;

    // The first tile's keys and values, the query.
    const uint16_t* const k0 = (const uint16_t*)d.k + (int64_t)layer * d.k_stride[0] + (int64_t)kvh * d.k_stride[1] + q0 * d.k_stride[2];
    const uint16_t* const v0 = (const uint16_t*)d.v + (int64_t)layer * d.v_stride[0] + (int64_t)kvh * d.v_stride[1] + q0 * d.v_stride[2];
    u32x4 k_raw[PER], v_raw[PER];
    auto load_tile = [&](int t) __attribute__((always_inline)) {
#pragma unroll
        for (int n = 0; n < PER; ++n) {
            const int key = (tid + n * 256) / CH, c = (tid + n * 256) % CH, r = t * BN + key;
            const bool in = r < nq;
            const u32x4 k = *(const u32x4*)(k0 + (int64_t)(in ? r : 0) * d.k_stride[2] + c * 8);
            const u32x4 v = *(const u32x4*)(v0 + (int64_t)(in ? r : 0) * d.v_stride[2] + c * 8);
            const u32x4 none = {0u, 0u, 0u, 0u};
            k_raw[n] = in ? k : none;
            v_raw[n] = in ? v : none;
        }
    };
    load_tile(0);
    bf16x8 qf[KS];
    {
        const uint16_t* const qrow = (const uint16_t*)a.q + (int64_t)layer * a.q_stride[0] + row * a.q_stride[1] + (int64_t)head * a.q_stride[2];
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) qf[ks] = __builtin_bit_cast(bf16x8, *(const u32x4*)(qrow + ks * 16 + hl * 8));
    }
    const int64_t pos = a.window > 0 ? a.q_pos[row] : 0;
    if (tid < 2) odd_keys[tid] = 0;

    // The cache's partials, relative to the largest log-sum-exp.  Element 4b + e of o[db]
    // is channel 32 db + 8 b + 4 hl + e of row j; both halves of a row hold all records.
    f32x16 o[DB];
#pragma unroll
    for (int db = 0; db < DB; ++db) o[db] = f32x16{};
    float mx = -INFINITY, l = 0.f;
    for (int s = 0; s < a.n_splits; ++s) mx = fmaxf(mx, a.ws_lse[s * items + item]);
#pragma unroll 1
    for (int s = 0; s < a.n_splits; ++s) {
        const float lse = a.ws_lse[s * items + item];
        const bool used = lse != -INFINITY;
        if (__builtin_amdgcn_ballot_w64(used) == 0) continue;
        const float w = used ? __builtin_amdgcn_exp2f(lse - mx) : 0.f;
        if (!used) continue;   // (its output was not written)
        const float* const x = a.ws_o + (s * items + item) * D + hl * 4;
        l += w;
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
            for (int b = 0; b < 4; ++b) {
                const f32x4 v = *(const f32x4*)(x + db * 32 + b * 8);
#pragma unroll
                for (int e = 0; e < 4; ++e) o[db][4 * b + e] = fmaf(w, v[e], o[db][4 * b + e]);
            }
    }
    if (hl != 0) l = 0.f;   // counted once: the halves hold different drafted rows

    int kofs[KS], vofs[DB];
    gqa_operand_offsets<D>(lane, kofs, vofs);
    const float sc2 = a.scale * kLog2e;
    // Drafted rows that the workgroup can see: with a mask all, in a chain those up to its last row.
    const int last_row = (min(M, m0 + 128) - 1) / G;
    const int tiles = ((d.mask ? nq : last_row + 1) + BN - 1) / BN;
#pragma unroll 1
    for (int t = 0; t < tiles; ++t) {
        __syncthreads();   // every wave is done with the tile before
        if (tid == 0) odd_keys[(t + 1) & 1] = 0;
#pragma unroll
        for (int n = 0; n < PER; ++n) {
            const int key = (tid + n * 256) / CH, c = (tid + n * 256) % CH;
            u32x4 v = v_raw[n];
            bool odd = false;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const bool lo = (v[e] & 0x7f80u) == 0x7f80u, hi = (v[e] & 0x7f800000u) == 0x7f800000u;
                odd = odd || lo || hi;
                v[e] &= (lo ? 0xffff0000u : ~0u) & (hi ? 0xffffu : ~0u);
            }
            if (odd) atomicOr(&odd_keys[t & 1], 1u << key);
            *(u32x4*)(k_lds + key * D + ((c ^ swz_k<D>(key)) << 3)) = k_raw[n];
            *(u32x4*)(v_lds + key * D + ((c ^ swz_v<D>(key)) << 3)) = v;
        }
        // Which of the tile's rows this row sees.
        uint32_t word;
        if (d.mask) word = t < d.mask_words ? d.mask[row * d.mask_words + t] : 0u;
        else word = i >= t * BN + 31 ? ~0u : i >= t * BN ? (2u << (i - t * BN)) - 1 : 0u;
        if (nq - t * BN < 32) word &= (1u << (nq - t * BN)) - 1;   // no rows behind the sequence
        if (!row_ok) word = 0;
        if (a.window > 0) {
            for (int c = 0; c < BN; ++c)   // (a position past the sequence's end is not read)
                if (t * BN + c < nq && a.q_pos[q0 + t * BN + c] <= pos - a.window) word &= ~(1u << c);
        }
        __syncthreads();
        if (t + 1 < tiles) load_tile(t + 1);
        if (__builtin_amdgcn_ballot_w64(word != 0) == 0) continue;   // (the barriers are behind)

        f32x16 s = f32x16{};
#pragma unroll
        for (int ks = 0; ks < KS; ++ks)
            s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, *(const u32x4*)(k_lds + kofs[ks])), qf[ks], s, 0, 0, 0);
        // Element r holds drafted row 8 (r / 4) + 4 hl + r % 4 of the tile.
        float top = -INFINITY;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            s[r] = (word >> ((r >> 2) * 8 + hl * 4 + (r & 3))) & 1 ? s[r] * sc2 : -INFINITY;
            top = fmaxf(top, s[r]);
        }
        float x, y;
        both<32>(top, x, y);
        const float m_new = fmaxf(mx, fmaxf(x, y));
        const float keep = mx == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(mx - m_new);
        l *= keep;
#pragma unroll
        for (int db = 0; db < DB; ++db) o[db] *= keep;
        mx = m_new;
        bf16x8 pb[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            f32x8 p;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int r = h * 8 + e;
                s[r] = s[r] == -INFINITY ? kUnseen : __builtin_amdgcn_exp2f(s[r] - m_new);
                p[e] = s[r];
            }
            pb[h] = __builtin_convertvector(p, bf16x8);
        }
        // The sum takes the probabilities as they enter the product.
        const bf16x2 ones = {(__bf16)1.0f, (__bf16)1.0f};
#pragma unroll
        for (int e = 0; e < 16; e += 2)
            l = __builtin_amdgcn_fdot2_f32_bf16((bf16x2){pb[e >> 3][e & 7], pb[e >> 3][(e & 7) + 1]}, ones, l, false);
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int db = 0; db < DB; ++db)
                o[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(gqa_v_operand<D>(v_lds + vofs[db] + h * 16 * D), pb[h], o[db], 0, 0, 0);
        // Values that were left out, key by key.
        uint32_t odd = (uint32_t)__builtin_amdgcn_readfirstlane((int)odd_keys[t & 1]);
        while (odd) {
            const int key = __builtin_ctz(odd);
            odd &= odd - 1;
            float mine = 0.f;
#pragma unroll
            for (int r = 0; r < 16; ++r) mine = r == (key >> 3) * 4 + (key & 3) ? s[r] : mine;
            const float other = __shfl_xor(mine, 32);
            const float p = hl == ((key >> 2) & 1) ? mine : other;
            const bool weighs = __float_as_uint(p) != __float_as_uint(kUnseen);
            const uint16_t* const v = v0 + (int64_t)(t * BN + key) * d.v_stride[2] + hl * 4;
#pragma unroll
            for (int db = 0; db < DB; ++db)
#pragma unroll
                for (int b = 0; b < 4; ++b)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float z = load1(v + db * 32 + b * 8 + e);
                        if (weighs && !(fabsf(z) < INFINITY)) o[db][4 * b + e] += p * z;
                    }
        }
    }

    const float l_tot = l + __shfl_xor(l, 32);
    if (!row_ok) return;
    const float inv = row_inverse(l_tot);
    uint16_t* const dst = (uint16_t*)a.out + (int64_t)layer * a.o_stride[0] + row * a.o_stride[1] + (int64_t)head * a.o_stride[2];
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int b = 0; b < 4; ++b) {
            u32x2 w;
            w[0] = bf_rne(o[db][4 * b] * inv) | (bf_rne(o[db][4 * b + 1] * inv) << 16);
            w[1] = bf_rne(o[db][4 * b + 2] * inv) | (bf_rne(o[db][4 * b + 3] * inv) << 16);
            *(u32x2*)(dst + db * 32 + b * 8 + hl * 4) = w;
        }
    if (a.lse_out && hl == 0) a.lse_out[item] = row_lse2(mx, l_tot) * kLn2;
}

// Layers and KV heads share a grid dimension in tiles; a wave a row and head needs it for the layers alone.
constexpr int64_t kMaxGridZ = 65535;

// Tiles pay where they fill, and where there are enough workgroups to hide that each of
// them waits for one record after another (a wave a row and head / tiles, us a call, 32
// heads over 8 KV heads of 128; 16 sequences of 32 rows over 2000..9000 keys 109 / 115; 24
// of 24 over 200..500 36 / 33, over 2000..5000 103 / 103; 8 of 96 over 2000..5000 82 / 82; 48
// of 24 over 200..500 57 / 45; 48 of 96 over 50 148 / 97, over 2000 325 / 273; as chains,
// whose rows see many drafted rows, 8 of 96 over 1000 73 / 47, 48 of 96 over 50 262 / 89).
// Less will do where a row has one record (28 heads over 4 KV heads of 128: chains of
// 93 rows of 4 sequences over 21..37 keys 33.5 / 24.0, of 29 rows of 18 over 1 key 29.1 / 21.9,
// trees of 49 rows of 11 over 7..11 keys 19.9 / 22.0; 9 of 24 over 0..3, two layers, 21.8 / 18.0; 8
// heads of 8: 27 of 43 over 5..17, two layers, 26.8 / 31.0, 48 of 23 over 4..13 25.5 / 22.7; with
// more records, 47 rows of 9 over 76..247 keys 19.4 / 29.6), down to 8192 rows (46 of 4, 32
// heads over 8, 5888 rows 18.0 / 21.9).
bool tile_route(const AttnArgs& a) {
    if (a.variant == 1 || a.dtype == 1 || a.n_splits > 16) return false;
    if ((int64_t)a.n_layers * a.n_kv_heads > kMaxGridZ) return false;
    const int64_t rows = (int64_t)a.max_q * (a.n_heads / a.n_kv_heads), total = rows * a.n_kv_heads * a.n_layers * a.n_seqs;
    return a.n_splits > 1 ? rows >= 64 && total >= 24576 : rows >= 16 && total >= 8192;
}

template <int D>
hipError_t launch_tiles(const AttnArgs& a, const DraftArgs& d, hipStream_t stream) {
    const int64_t rows = (int64_t)a.max_q * (a.n_heads / a.n_kv_heads), z = (int64_t)a.n_layers * a.n_kv_heads;
    if (rows > 0x7fffffff || z > kMaxGridZ) return hipErrorInvalidValue;
    for (int seq0 = 0; seq0 < a.n_seqs; seq0 += 65535) {
        const int n = a.n_seqs - seq0 < 65535 ? a.n_seqs - seq0 : 65535;
        hipLaunchKernelGGL((tree_join_tiles<D>), dim3((unsigned)((rows + 127) / 128), (unsigned)n, (unsigned)z), dim3(256), 0, stream, a, d, seq0);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

template <typename T, int D>
hipError_t launch_d(const AttnArgs& a, const DraftArgs& d, hipStream_t stream) {
    const int64_t units = (int64_t)a.max_q * a.n_heads;
    if (units > 0x7fffffff || a.n_layers > kMaxGridZ) return hipErrorInvalidValue;
    for (int seq0 = 0; seq0 < a.n_seqs; seq0 += 65535) {
        const int n = a.n_seqs - seq0 < 65535 ? a.n_seqs - seq0 : 65535;
        hipLaunchKernelGGL((tree_join<T, D>), dim3((unsigned)((units + kJoinWaves - 1) / kJoinWaves), (unsigned)n, (unsigned)a.n_layers),
                           dim3(kJoinWaves * 64), 0, stream, a, d, seq0);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace

hipError_t launch_tree_join(const AttnArgs& a, const DraftArgs& d, hipStream_t stream) {
    if (a.max_q == 0) return hipSuccess;
    if (a.variant == 1) return launch_d<uint16_t, 576>(a, d, stream);
    if (tile_route(a)) return a.head_dim == 64 ? launch_tiles<64>(a, d, stream) : launch_tiles<128>(a, d, stream);
    if (a.dtype == 1) return a.head_dim == 64 ? launch_d<float, 64>(a, d, stream) : launch_d<float, 128>(a, d, stream);
    return a.head_dim == 64 ? launch_d<uint16_t, 64>(a, d, stream) : launch_d<uint16_t, 128>(a, d, stream);
}

hipError_t launch_tree_attention(const AttnArgs& a, const BlockScales* scales, const DraftArgs& d, hipStream_t stream) {
    if (a.n_splits > 0) {   // 0: no cache has a slot
        const hipError_t e = launch_attention(a, scales, stream);
        if (e != hipSuccess) return e;
    }
    return launch_tree_join(a, d, stream);
}

}  // namespace pkv
