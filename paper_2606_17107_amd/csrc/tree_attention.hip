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
// A tree's row sees few drafted rows (its depth, not the size of the tree), so a wave
// goes through the set bits of the row's mask and loads only those keys and values:
// scores, sums and outputs stay in fp32 registers.  Head sizes 64 and 128: CH = D/8
// lanes share a key, 64 / CH keys (or partials) are in work at once, merged at the end.
// Latent rows (576 channels): the whole wave shares a key, whose first 512 channels are
// its value.  A wave holds HB heads of one KV head, so a key is loaded once for them.
#include "attn_common.h"

namespace pkv {
namespace {

constexpr int kJoinWaves = 4;

template <typename T>
__device__ __forceinline__ void load8(const T* p, float (&x)[8]);
template <>
__device__ __forceinline__ void load8<float>(const float* p, float (&x)[8]) {
    const f32x4 a = *(const f32x4*)p, b = *(const f32x4*)(p + 4);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        x[e] = a[e];
        x[4 + e] = b[e];
    }
}
template <>
__device__ __forceinline__ void load8<uint16_t>(const uint16_t* p, float (&x)[8]) {
    const u32x4 a = *(const u32x4*)p;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        x[2 * e] = __uint_as_float(a[e] << 16);
        x[2 * e + 1] = __uint_as_float(a[e] & 0xffff0000u);
    }
}
__device__ __forceinline__ float load1(const float* p) { return *p; }
__device__ __forceinline__ float load1(const uint16_t* p) { return __uint_as_float((uint32_t)*p << 16); }

// One entry with weight 2^s (s > -inf, or NaN) and value x joins the sums.  A NaN or
// +inf score makes the sum NaN, which stays NaN.
__device__ __forceinline__ void join_entry(float s, const float (&x)[8], float& m, float& l, float (&acc)[8]) {
    const float m_new = fmaxf(m, s);
    const float keep = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - m_new);
    const float w = __builtin_amdgcn_exp2f(s - m_new);
    l = l * keep + w;
#pragma unroll
    for (int e = 0; e < 8; ++e) acc[e] = acc[e] * keep + w * x[e];
    m = m_new;
}

template <typename T, int D, int HB>
__global__ __launch_bounds__(kJoinWaves * 64) void tree_join(AttnArgs a, DraftArgs d, int seq0) {
    constexpr bool MLA = D == 576;
    constexpr int DV = MLA ? 512 : D;
    constexpr int CH = DV / 8;          // lanes per key
    constexpr int KG = 64 / CH;         // keys in work at once
    const int lane = threadIdx.x & 63;
    const int kg = lane / CH, c = lane % CH;
    const int G = a.n_heads / a.n_kv_heads;
    const int blocks = (G + HB - 1) / HB;              // waves per row and KV head
    const int64_t unit = (int64_t)blockIdx.x * kJoinWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int per_row = blocks * a.n_kv_heads;
    const int i = (int)(unit / per_row);
    const int rest = (int)(unit - (int64_t)i * per_row);
    const int kvh = rest / blocks;
    const int h0 = (rest - kvh * blocks) * HB;          // first head within the KV head
    const int seq = seq0 + (int)blockIdx.y;
    const int layer = (int)blockIdx.z;
    const SeqInfo si = seq_info(a, seq);
    if (i >= si.nq || i >= a.max_q) return;
    const int64_t row = si.q0 + i;
    const int64_t items = (int64_t)a.n_layers * a.total_q * a.n_heads;
    const int64_t item0 = ((int64_t)layer * a.total_q + row) * a.n_heads + kvh * G + h0;

    float m[HB], l[HB], acc[HB][8];
#pragma unroll
    for (int h = 0; h < HB; ++h) {
        m[h] = -INFINITY;
        l[h] = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) acc[h][e] = 0.f;
    }

    // The cache's partials.
    const int ns = a.n_splits;
#pragma unroll
    for (int h = 0; h < HB; ++h) {
        if (h0 + h >= G) continue;
        for (int s = kg; s < ns; s += KG) {
            const int64_t item = s * items + item0 + h;
            const float lse = a.ws_lse[item];
            if (lse == -INFINITY) continue;
            float x[8];
            load8<float>(a.ws_o + item * DV + c * 8, x);
            join_entry(lse, x, m[h], l[h], acc[h]);
        }
    }

    // The drafted rows it sees.
    float q[HB][8], q_rope[HB];
#pragma unroll
    for (int h = 0; h < HB; ++h) {
        const int head = kvh * G + min(h0 + h, G - 1);
        const T* src = (const T*)a.q + (int64_t)layer * a.q_stride[0] + row * a.q_stride[1] + (int64_t)head * a.q_stride[2];
        load8<T>(src + c * 8, q[h]);
        q_rope[h] = MLA ? load1(src + 512 + c) : 0.f;
    }
    const int64_t pos = a.q_pos[row];
    const T* const k0 = (const T*)d.k + (int64_t)layer * d.k_stride[0] + (int64_t)kvh * d.k_stride[1] + si.q0 * d.k_stride[2];
    const T* const v0 = (const T*)d.v + (int64_t)layer * d.v_stride[0] + (int64_t)kvh * d.v_stride[1] + si.q0 * d.v_stride[2];
    const float sc2 = a.scale * kLog2e;
    const int words = (si.nq + 31) / 32;
    for (int w = 0; w < words; ++w) {
        uint32_t bits;
        if (d.mask) bits = w < d.mask_words ? d.mask[row * d.mask_words + w] : 0u;
        else bits = i >= w * 32 + 31 ? ~0u : i >= w * 32 ? (2u << (i - w * 32)) - 1 : 0u;
        if (si.nq - w * 32 < 32) bits &= (1u << (si.nq - w * 32)) - 1;   // no rows behind the sequence
        bits = (uint32_t)__builtin_amdgcn_readfirstlane((int)bits);
        while (bits) {
            // The next KG set bits, one for each group of lanes.
            int at = -1;
#pragma unroll
            for (int g = 0; g < KG; ++g) {
                const int b = bits ? __builtin_ctz(bits) : -1;
                bits &= bits - 1;
                if (g == kg) at = b;
            }
            if (at < 0) continue;
            const int64_t r = w * 32 + at;
            if (a.window > 0 && a.q_pos[si.q0 + r] <= pos - a.window) continue;
            float k[8], v[8];
            load8<T>(k0 + r * d.k_stride[2] + c * 8, k);
            const float k_rope = MLA ? load1(k0 + r * d.k_stride[2] + 512 + c) : 0.f;
            if constexpr (!MLA) load8<T>(v0 + r * d.v_stride[2] + c * 8, v);
#pragma unroll
            for (int h = 0; h < HB; ++h) {
                float s = q_rope[h] * k_rope;
#pragma unroll
                for (int e = 0; e < 8; ++e) s = fmaf(q[h][e], k[e], s);
#pragma unroll
                for (int o = CH / 2; o >= 1; o >>= 1) s += __shfl_xor(s, o);
                s *= sc2;
                if (s == -INFINITY) continue;   // weighs nothing
                join_entry(s, MLA ? k : v, m[h], l[h], acc[h]);
            }
        }
    }

    // The groups of lanes hold disjoint entries.
#pragma unroll
    for (int h = 0; h < HB; ++h) {
#pragma unroll
        for (int o = CH; o < 64; o <<= 1) {
            const float m2 = __shfl_xor(m[h], o), l2 = __shfl_xor(l[h], o);
            const float m_new = fmaxf(m[h], m2);
            const float r1 = m[h] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m[h] - m_new);
            const float r2 = m2 == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m2 - m_new);
            l[h] = l[h] * r1 + l2 * r2;
#pragma unroll
            for (int e = 0; e < 8; ++e) acc[h][e] = acc[h][e] * r1 + __shfl_xor(acc[h][e], o) * r2;
            m[h] = m_new;
        }
        if (h0 + h >= G || kg != 0) continue;
        const float inv = row_inverse(l[h]);
        T* dst = (T*)a.out + (int64_t)layer * a.o_stride[0] + row * a.o_stride[1] +
                 (int64_t)(kvh * G + h0 + h) * a.o_stride[2] + c * 8;
        if constexpr (sizeof(T) == 4) {
            *(f32x4*)dst = f32x4{acc[h][0] * inv, acc[h][1] * inv, acc[h][2] * inv, acc[h][3] * inv};
            *(f32x4*)(dst + 4) = f32x4{acc[h][4] * inv, acc[h][5] * inv, acc[h][6] * inv, acc[h][7] * inv};
        } else {
            u32x4 o;
#pragma unroll
            for (int e = 0; e < 4; ++e) o[e] = bf_rne(acc[h][2 * e] * inv) | (bf_rne(acc[h][2 * e + 1] * inv) << 16);
            *(u32x4*)dst = o;
        }
        if (a.lse_out && c == 0) a.lse_out[item0 + h] = row_lse2(m[h], l[h]) * kLn2;
    }
}

template <typename T, int D, int HB>
hipError_t launch_hb(const AttnArgs& a, const DraftArgs& d, hipStream_t stream) {
    const int G = a.n_heads / a.n_kv_heads;
    const int64_t units = (int64_t)a.max_q * a.n_kv_heads * ((G + HB - 1) / HB);
    const int64_t blocks = (units + kJoinWaves - 1) / kJoinWaves;
    if (blocks > 0x7fffffff || a.n_layers > 65535) return hipErrorInvalidValue;
    for (int seq0 = 0; seq0 < a.n_seqs; seq0 += 65535) {
        const int n = a.n_seqs - seq0 < 65535 ? a.n_seqs - seq0 : 65535;
        hipLaunchKernelGGL((tree_join<T, D, HB>), dim3((unsigned)blocks, (unsigned)n, (unsigned)a.n_layers),
                           dim3(kJoinWaves * 64), 0, stream, a, d, seq0);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

template <typename T, int D>
hipError_t launch_d(const AttnArgs& a, const DraftArgs& d, hipStream_t stream) {
    return a.n_heads / a.n_kv_heads >= 4 ? launch_hb<T, D, 4>(a, d, stream) : launch_hb<T, D, 1>(a, d, stream);
}

}  // namespace

hipError_t launch_tree_join(const AttnArgs& a, const DraftArgs& d, hipStream_t stream) {
    if (a.max_q == 0) return hipSuccess;
    if (a.variant == 1) return launch_d<uint16_t, 576>(a, d, stream);
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
