// Trees of drafted tokens beside a cache: which rows descend from which (masks), the
// path that the target model's probabilities accept (verify), and the accepted rows'
// way into the cache (commit).
#include "attn_columns.h"

namespace pkv {
namespace {

// Rows [q0, q0 + n) of a sequence (none where the bounds do not fit the call).
__device__ inline void tree_rows(const int32_t* cu_q, int total_q, int seq, int& q0, int& n) {
    q0 = 0;
    n = total_q;
    if (cu_q) {
        q0 = cu_q[seq];
        n = cu_q[seq + 1] - q0;
    }
    if (q0 < 0 || n < 0 || (int64_t)q0 + n > total_q) n = 0;
}

// ---- masks -----------------------------------------------------------------------

// Row i sees itself and every row on the way to the tree's root.  Parents come before
// their children, so a row's ancestors are met in falling order and each word of its
// mask is finished before the next lower one begins: a thread per row follows the
// parents in LDS and stores every word once.  A call is a launch and one such chain (as
// many LDS reads as the tree is deep).
__global__ __launch_bounds__(256) void tree_masks(TreeMaskArgs a) {
    __shared__ int parent[kTreeMaxRows];
    int q0, n;
    tree_rows(a.cu_q, a.total_q, (int)blockIdx.x, q0, n);
    n = min(n, a.max_q);
    const int kv = a.q_pos ? a.kv_len[blockIdx.x] : 0;
    bool bad = false;
    for (int i = threadIdx.x; i < n; i += 256) {
        int p = a.parent[q0 + i];
        if (p < -1 || p >= i) {
            bad = true;
            p = -1;
        }
        parent[i] = p;
    }
    __syncthreads();
    if (bad && a.err_flag) *a.err_flag = 1;
    for (int i = threadIdx.x; i < n; i += 256) {
        uint32_t* const out = a.mask + (int64_t)(q0 + i) * a.mask_words;
        int w = a.mask_words - 1, depth = -1;
        uint32_t word = 0;
        for (int at = i; at >= 0; at = parent[at]) {
            for (; w > at >> 5; --w) {
                out[w] = word;
                word = 0;
            }
            word |= 1u << (at & 31);
            ++depth;
        }
        for (; w >= 0; --w) {
            out[w] = word;
            word = 0;
        }
        if (a.q_pos) a.q_pos[q0 + i] = kv + depth;
    }
}

// ---- verify ----------------------------------------------------------------------

// The weights that tests and the final draw go by: probabilities that are numbers above
// 0 and finite, anything else counts as 0.  Sums and comparisons are in 64 bits: the
// result is a choice, and rounding must not change it.
__device__ __forceinline__ double as_weight(float x) { return x > 0.f && x < INFINITY ? (double)x : 0.0; }
__device__ __forceinline__ double as_weight(uint16_t x) { return as_weight(__uint_as_float((uint32_t)x << 16)); }

// 16 bytes of a row of probabilities at the alignment of its type (rows of an odd
// vocabulary begin anywhere).
template <typename T>
struct __attribute__((packed, aligned(sizeof(T)))) Probs {
    T x[16 / sizeof(T)];
};

// A row's weights max(p - a q, 0), or without a draft p less the tokens that were tried.
template <typename T>
struct Weights {
    const T* p;
    const T* q;     // or null
    double a;
    int vocab;
};

constexpr int kPiece = 1024;   // elements of a row that a wave sums at once

// The weights of piece `piece`, element 64 VE e + VE lane + k of it in w[e][k].
// gone: null, or 32 words of LDS whose bits are elements that count as 0.
template <typename T, int VE = 16 / (int)sizeof(T), int E = kPiece / 64 / VE>
__device__ __forceinline__ void load_piece(const Weights<T>& r, int piece, const uint32_t* gone, double (&w)[E][VE]) {
    const int lane = (int)__lane_id();
    const int64_t base = (int64_t)piece * kPiece;
    Probs<T> p[E], q[E];
    if (base + kPiece <= r.vocab) {   // uniform
#pragma unroll
        for (int e = 0; e < E; ++e) {
            p[e] = *(const Probs<T>*)(r.p + base + (e * 64 + lane) * VE);
            if (r.q) q[e] = *(const Probs<T>*)(r.q + base + (e * 64 + lane) * VE);
        }
    } else {
#pragma unroll
        for (int e = 0; e < E; ++e)
#pragma unroll
            for (int k = 0; k < VE; ++k) {
                const int64_t v = base + (e * 64 + lane) * VE + k;
                p[e].x[k] = v < r.vocab ? r.p[v] : (T)0;
                if (r.q) q[e].x[k] = v < r.vocab ? r.q[v] : (T)0;
            }
    }
#pragma unroll
    for (int e = 0; e < E; ++e) {
        uint32_t out = 0;
        if (gone) out = gone[(e * 64 + lane) * VE >> 5] >> ((e * 64 + lane) * VE & 31);
#pragma unroll
        for (int k = 0; k < VE; ++k) {
            w[e][k] = as_weight(p[e].x[k]);
            if (r.q) w[e][k] = fmax(w[e][k] - r.a * as_weight(q[e].x[k]), 0.0);
            if ((out >> k) & 1) w[e][k] = 0.0;
        }
    }
}

// Sums over a wave by DPP, as attn_columns.h has them for integers: each half of a
// double is moved by itself.  Lanes without a source get 0.
template <int CTRL, int ROWS = 0xf>
__device__ __forceinline__ double dpp64(double v) {
    const uint64_t b = __builtin_bit_cast(uint64_t, v);
    const uint32_t lo = (uint32_t)dpp<CTRL, ROWS>(0, (int)(uint32_t)b), hi = (uint32_t)dpp<CTRL, ROWS>(0, (int)(uint32_t)(b >> 32));
    return __builtin_bit_cast(double, ((uint64_t)hi << 32) | lo);
}
__device__ __forceinline__ double lane_value(double v, int lane) {
    const uint64_t b = __builtin_bit_cast(uint64_t, v);
    const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)b, lane);
    const uint32_t hi = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(b >> 32), lane);
    return __builtin_bit_cast(double, ((uint64_t)hi << 32) | lo);
}
__device__ __forceinline__ double wave_sum(double v) {
    v += dpp64<kDppRor + 8>(v);
    v += dpp64<kDppRor + 4>(v);
    v += dpp64<kDppRor + 2>(v);
    v += dpp64<kDppRor + 1>(v);
    return (lane_value(v, 0) + lane_value(v, 16)) + (lane_value(v, 32) + lane_value(v, 48));
}
// Inclusive running sum over the lanes.
__device__ __forceinline__ double wave_scan(double v) {
    v += dpp64<kDppShr + 1>(v);
    v += dpp64<kDppShr + 2>(v);
    v += dpp64<kDppShr + 4>(v);
    v += dpp64<kDppShr + 8>(v);
    v += dpp64<kDppBcast15, 0xa>(v);
    v += dpp64<kDppBcast31, 0xc>(v);
    return v;
}

// Sum of a piece, in every lane.
template <typename T, int VE = 16 / (int)sizeof(T), int E = kPiece / 64 / VE>
__device__ __forceinline__ double lane_sum(const double (&w)[E][VE]) {
    double s = 0.0;
#pragma unroll
    for (int e = 0; e < E; ++e)
#pragma unroll
        for (int k = 0; k < VE; ++k) s += w[e][k];
    return s;
}
template <typename T>
__device__ __forceinline__ double piece_sum(const Weights<T>& r, int piece, const uint32_t* gone) {
    constexpr int VE = 16 / (int)sizeof(T), E = kPiece / 64 / VE;
    double w[E][VE];
    load_piece(r, piece, gone, w);
    return wave_sum(lane_sum<T>(w));
}

// The tokens of cur's children that lie in a piece, as bits of 32 words of LDS that
// the wave has to itself; null if there are none.  at(i): token of row i if it is a child of cur, else -1.
template <typename F>
__device__ __forceinline__ const uint32_t* tried_tokens(int piece, int cur, int n, uint32_t* words, F at) {
    const int lane = (int)__lane_id();
    bool any = false;
    for (int i0 = cur + 1; i0 < n; i0 += 64) {
        const int t = i0 + lane < n ? at(i0 + lane) : -1;
        const bool in = t >= 0 && t / kPiece == piece;
        if (__builtin_amdgcn_ballot_w64(in) == 0) continue;
        if (!any && lane < kPiece / 32) words[lane] = 0;
        any = true;
        __builtin_amdgcn_wave_barrier();   // (a wave's LDS accesses are in order)
        asm volatile("" ::: "memory");
        if (in) atomicOr(&words[(t & (kPiece - 1)) >> 5], 1u << (t & 31));
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    return any ? words : nullptr;
}

// One wave finds the token: the smallest v whose running sum passes u times the sum of
// all pieces, by the pieces' sums and then in the piece; the last v with a weight if
// rounding leaves none.  -1: no weight at all.  sums(k): sum of piece k; gone(k): its tried tokens.
template <typename T, typename S, typename GN>
__device__ int find_token(const Weights<T>& r, int pieces, double u, S sums, GN gone) {
    constexpr int VE = 16 / (int)sizeof(T), E = kPiece / 64 / VE;
    const int lane = (int)__lane_id();
    double total = 0.0;
    for (int b = 0; b < pieces; b += 64) total += lane_value(wave_scan(b + lane < pieces ? sums(b + lane) : 0.0), 63);
    if (!(total > 0.0)) return -1;
    const double aim = u * total;
    double run = 0.0, before = 0.0;
    int piece = 0;
    for (int b = 0; b < pieces; b += 64) {
        const double one = b + lane < pieces ? sums(b + lane) : 0.0;
        const double s = run + wave_scan(one);
        const uint64_t full = __builtin_amdgcn_ballot_w64(one > 0.0), over = __builtin_amdgcn_ballot_w64(one > 0.0 && s > aim);
        if (full) {
            const int k = over ? __builtin_ctzll(over) : 63 - __builtin_clzll(full);
            piece = b + k;
            before = k > 0 ? lane_value(s, k - 1) : run;
            if (over) break;
        }
        run = lane_value(s, 63);
    }
    double w[E][VE], part[E], upto[E];
    load_piece(r, piece, gone(piece), w);
#pragma unroll
    for (int e = 0; e < E; ++e) {
        part[e] = 0.0;
#pragma unroll
        for (int k = 0; k < VE; ++k) part[e] += w[e][k];
        upto[e] = wave_scan(part[e]);
    }
    int first = 0x7fffffff, last = -1;
#pragma unroll
    for (int e = 0; e < E; ++e) {
        const double left = __shfl_up(upto[e], 1);
        double at = before + (lane > 0 ? left : 0.0);
#pragma unroll
        for (int k = 0; k < VE; ++k) {
            const int v = (e * 64 + lane) * VE + k;
            at += w[e][k];
            if (w[e][k] > 0.0) {
                last = v;
                if (at > aim) first = min(first, v);
            }
        }
        before += lane_value(upto[e], 63);
    }
    first = wave_min_u(first);
    last = wave_max_u(last);
    return piece * kPiece + (first < 0x7fffffff ? first : max(last, 0));
}

// What the walk leaves for the draw, one per sequence.
struct VerifyState {
    double a;          // weights max(p - a q, 0)
    int32_t cur;       // row of the tree where the walk ended, -1: no rows
    int32_t tried;     // its children were tried (and refused)
};

constexpr int kWalkThreads = 1024;
constexpr int64_t kWalkBytes = 256 << 10;
constexpr int kWalkPieces = 256;   // pieces of the largest row that the walk's workgroup draws from itself

// The walk down one tree, one workgroup per sequence.  Every wave walks, from the same
// values in LDS, so the workgroup meets again only for sums over a row of
// probabilities: those are formed where a child drawn from the draft's probabilities
// is refused and a sibling is to be tried.  DRAW: it draws the next token, too.
template <typename T, bool DRAW>
__global__ __launch_bounds__(kWalkThreads) void tree_walk(TreeVerifyArgs a) {
    constexpr int NT = kWalkThreads, NW = NT / 64;
    __shared__ int parent[kTreeMaxRows], token[kTreeMaxRows];
    __shared__ float u[kTreeMaxRows], pr[kTreeMaxRows], qr[kTreeMaxRows];
    __shared__ double part[NW], sums[DRAW ? kWalkPieces : 1];
    __shared__ uint32_t bits[DRAW ? NW : 1][kPiece / 32];
    const int seq = (int)blockIdx.x, tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const double u_draw = DRAW ? (double)a.u_sample[seq] : 0.0;
    int q0, n;
    tree_rows(a.cu_q, a.total_q, seq, q0, n);
    n = min(n, a.max_q);
    const T* const target = (const T*)a.target;
    const T* const draft = (const T*)a.draft;
    bool bad = false;
    for (int i = tid; i < n; i += NT) {
        int p = a.parent[q0 + i];
        const int t = a.tokens[q0 + i];
        float pw = 0.f, qw = 0.f;
        if (i == 0) {
            p = -1;
        } else if (p < -1 || p >= i || t < 0 || t >= a.vocab) {
            bad = true;
            p = -1;   // no candidate
        }
        if (p >= 0) {
            pw = (float)as_weight(target[(int64_t)(q0 + p) * a.target_stride + t]);
            if (draft) qw = (float)as_weight(draft[(int64_t)(q0 + p) * a.draft_stride + t]);
        }
        parent[i] = p;
        token[i] = t;
        u[i] = a.u_accept[q0 + i];
        pr[i] = pw;
        qr[i] = qw;
    }
    __syncthreads();
    if (bad && a.err_flag) *a.err_flag = 1;

    const int pieces = (a.vocab + kPiece - 1) / kPiece;
    auto row_of = [&](int cur, double wa) {
        return Weights<T>{target + (int64_t)(q0 + cur) * a.target_stride,
                          draft ? draft + (int64_t)(q0 + cur) * a.draft_stride : nullptr, wa, a.vocab};
    };
    // Up to 64 rows are held by the lanes of every wave, more are read from LDS.
    const bool held = n <= 64;
    const int hi = min(lane, max(n - 1, 0));
    const int my_parent = parent[hi], my_token = token[hi];
    const float my_u = u[hi], my_p = pr[hi], my_q = qr[hi];
    auto value = [&](float mine, const float* all, int i) {
        return held ? __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(mine), i)) : all[i];
    };
    // First child of cur in rows [from, to), -1: none; x >= 0: with this token.
    auto child = [&](int cur, int from, int to, int x) __attribute__((always_inline)) {
        for (int b = held ? 0 : from & ~63; b < to; b += 64) {
            const int r = b + lane, at = min(r, n - 1);
            const bool is = (held ? my_parent : parent[at]) == cur && (x < 0 || (held ? my_token : token[at]) == x);
            const uint64_t hit = __builtin_amdgcn_ballot_w64(r >= from && r < to && is);
            if (hit) return b + (int)__builtin_ctzll(hit);
        }
        return -1;
    };
    int32_t* const path = a.path + (int64_t)seq * a.max_path;
    int cur = 0, length = n > 0 ? 1 : 0;
    bool tried = true;
    double wa = 0.0, wb = 1.0;   // the weights left at cur are max(p - wa q, 0), their sum is wb
    if (n > 0 && tid == 0) path[0] = q0;
    int i0 = 1;                  // rows before i0 are no more candidates
    while (n > 0) {
        if (length >= a.max_path) {
            tried = false;
            break;
        }
        const int i = child(cur, i0, n, -1);   // the next child
        if (i < 0) break;
        i0 = i + 1;
        double r;
        bool accept;
        if (draft) {
            const double q = (double)value(my_q, qr, i);
            r = fmax((double)value(my_p, pr, i) - wa * q, 0.0);
            accept = r > 0.0 && (double)value(my_u, u, i) * q * wb < r;
        } else {
            // A token that a refused sibling had is gone.
            const int x = held ? __builtin_amdgcn_readlane(my_token, i) : token[i];
            r = child(cur, cur + 1, i, x) >= 0 ? 0.0 : (double)value(my_p, pr, i);
            accept = r > 0.0 && (double)value(my_u, u, i) * wb < r;
        }
        if (accept) {
            if (tid == 0) path[length] = q0 + i;
            ++length;
            cur = i;
            wa = 0.0;
            wb = 1.0;
            continue;
        }
        if (!draft) {
            wb -= r;
            continue;
        }
        wa += wb;
        // The sum is needed only if another child follows.
        if (child(cur, i0, n, -1) < 0) break;
        const Weights<T> row = row_of(cur, wa);
        double sum = 0.0;
#pragma unroll 2
        for (int k = wave; k < pieces; k += NW) sum += piece_sum(row, k, nullptr);
        if (lane == 0) part[wave] = sum;
        __syncthreads();
        wb = 0.0;
        for (int w = 0; w < NW; ++w) wb += part[w];
        __syncthreads();
    }
    for (int k = length + tid; k < a.max_path; k += NT) path[k] = -1;
    if (tid == 0) {
        a.n_accepted[seq] = length;
        if (n == 0) a.next_token[seq] = -1;
    }
    if constexpr (!DRAW) {
        if (tid == 0) ((VerifyState*)a.workspace)[seq] = VerifyState{wa, n > 0 ? cur : -1, tried};
    } else {
        if (n == 0) return;
        int next = -1;
        // (the second time, where nothing was left: the row's own probabilities)
        for (int again = 0; again < 2; ++again) {
            const Weights<T> row = row_of(cur, wa);
            auto gone = [&](int k) -> const uint32_t* {
                if (draft || !tried) return nullptr;
                return tried_tokens(k, cur, n, bits[wave], [&](int i) { return parent[i] == cur ? token[i] : -1; });
            };
#pragma unroll 2
            for (int k = wave; k < pieces; k += NW) {
                const double s = piece_sum(row, k, gone(k));
                if (lane == 0) sums[k] = s;
            }
            __syncthreads();
            if (wave == 0) {
                next = find_token(row, pieces, u_draw, [&](int k) { return sums[k]; }, gone);
                if (lane == 0) part[0] = next;
            }
            __syncthreads();
            if (part[0] >= 0.0) break;
            wa = 0.0;
            tried = false;
            __syncthreads();
        }
        if (tid == 0) {
            a.next_token[seq] = next;
            if (next < 0 && a.err_flag) *a.err_flag = 1;
        }
    }
}

// The draw where rows are long, in two launches: waves sum the pieces of the row where
// each walk ended, then one wave a sequence finds the token.
struct DrawRow {
    int q0, n, cur;
    bool tried;
};
template <typename T>
__device__ __forceinline__ bool draw_row(const TreeVerifyArgs& a, int seq, DrawRow& d, Weights<T>& r) {
    const VerifyState s = ((const VerifyState*)a.workspace)[seq];
    if (s.cur < 0) return false;
    tree_rows(a.cu_q, a.total_q, seq, d.q0, d.n);
    d.n = min(d.n, a.max_q);
    d.cur = s.cur;
    d.tried = s.tried != 0 && !a.draft;
    r.p = (const T*)a.target + (int64_t)(d.q0 + s.cur) * a.target_stride;
    r.q = a.draft ? (const T*)a.draft + (int64_t)(d.q0 + s.cur) * a.draft_stride : nullptr;
    r.a = s.a;
    r.vocab = a.vocab;
    return true;
}
__device__ __forceinline__ const uint32_t* draw_gone(const TreeVerifyArgs& a, const DrawRow& d, int piece, uint32_t* words) {
    if (!d.tried) return nullptr;
    return tried_tokens(piece, d.cur, d.n, words, [&](int i) {
        const int p = a.parent[d.q0 + i], t = a.tokens[d.q0 + i];
        return p == d.cur ? t : -1;
    });
}
__device__ __forceinline__ double* draw_sums(const TreeVerifyArgs& a, int seq, int pieces) {
    return (double*)((VerifyState*)a.workspace + a.n_seqs) + (int64_t)seq * pieces;
}

template <typename T>
__global__ __launch_bounds__(256) void tree_sums(TreeVerifyArgs a, int pieces) {
    __shared__ uint32_t bits[4][kPiece / 32];
    const int seq = (int)blockIdx.y, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int k = (int)blockIdx.x * 4 + wave;
    DrawRow d;
    Weights<T> r;
    if (k >= pieces || !draw_row(a, seq, d, r)) return;
    const double s = piece_sum(r, k, draw_gone(a, d, k, bits[wave]));
    if (__lane_id() == 0) draw_sums(a, seq, pieces)[k] = s;
}

template <typename T>
__global__ __launch_bounds__(64) void tree_pick(TreeVerifyArgs a, int pieces) {
    __shared__ uint32_t bits[kPiece / 32];
    const int seq = (int)blockIdx.x;
    const double u_draw = (double)a.u_sample[seq];
    DrawRow d;
    Weights<T> r;
    if (!draw_row(a, seq, d, r)) return;
    double* const sums = draw_sums(a, seq, pieces);
    auto gone = [&](int k) { return draw_gone(a, d, k, bits); };
    int next = find_token(r, pieces, u_draw, [&](int k) { return sums[k]; }, gone);
    if (next < 0) {   // nothing is left: the row's own probabilities
        r.a = 0.0;
        r.q = nullptr;
        d.tried = false;
        for (int k = 0; k < pieces; ++k) {
            const double s = piece_sum(r, k, nullptr);
            if (__lane_id() == 0) sums[k] = s;
        }
        __syncthreads();
        next = find_token(r, pieces, u_draw, [&](int k) { return sums[k]; }, gone);
    }
    if (__lane_id() == 0) {
        a.next_token[seq] = next;
        if (next < 0 && a.err_flag) *a.err_flag = 1;
    }
}

// ---- commit ----------------------------------------------------------------------

// Slot and source row of step `step` of a sequence's path; false if nothing is to be
// written there (behind the accepted rows) or nothing can be (flagged).
__device__ inline bool commit_step(const TreeCommitArgs& a, int seq, int step, int64_t& row, int64_t& slot) {
    const int n = a.n_accepted[seq];
    row = a.path[(int64_t)seq * a.max_path + step];
    slot = (int64_t)a.kv_len[seq] + step;
    if (step >= n) return false;
    bool good = row >= 0 && row < a.n_rows && a.kv_len[seq] >= 0;
    if (!a.table[0] && a.kv_base) {
        const int64_t base = a.kv_base[seq];
        good = good && base >= 0;
        slot += base;
    }
    good = good && slot < a.capacity;
    if (!good && a.err_flag) *a.err_flag = 1;
    return good;
}

// A thread moves one 16-byte piece of one accepted row: pieces of a row's keys, then of
// its values, layer by layer.
__global__ __launch_bounds__(256) void tree_commit(TreeCommitArgs a, int seq0) {
    const int seq = seq0 + (int)blockIdx.z, step = (int)blockIdx.y;
    int64_t row, slot;
    if (!commit_step(a, seq, step, row, slot)) return;
    const int kc = a.row_bytes[0] / 16, vc = a.row_bytes[1] / 16;   // pieces of a row of one head
    const int per_layer = a.n_kv_heads * (kc + vc);
    const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int layer = (int)(id / per_layer);
    if (layer >= a.n_layers) return;
    int piece = (int)(id - (int64_t)layer * per_layer);
    const int t = piece >= a.n_kv_heads * kc;
    if (t) piece -= a.n_kv_heads * kc;
    const int per_head = t ? vc : kc;
    const int head = piece / per_head, c = piece - head * per_head;
    int64_t dst = layer * a.dst_stride[t][0] + head * a.dst_stride[t][1];
    if (a.table[t]) {
        const int entry = (int)(slot >> a.page_shift);
        const int page = entry < a.max_pages ? a.table[t][(int64_t)seq * a.max_pages + entry] : -1;
        if (page < 0 || page >= a.n_pages) {
            if (a.err_flag) *a.err_flag = 1;
            return;
        }
        dst += page * a.page_stride[t] + (slot & ((1 << a.page_shift) - 1)) * a.dst_stride[t][2];
    } else {
        dst += slot * a.dst_stride[t][2];
    }
    const u32x4 x = *(const u32x4*)(a.src[t] + layer * a.src_stride[t][0] + head * a.src_stride[t][1] +
                                    row * a.src_stride[t][2] + c * 16);
    *(u32x4*)(a.dst[t] + dst + c * 16) = x;
}

__global__ __launch_bounds__(256) void tree_segments(TreeCommitArgs a, StoreSegment* segs) {
    const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (id >= (int64_t)a.n_seqs * a.max_path) return;
    const int seq = (int)(id / a.max_path), step = (int)(id - (int64_t)seq * a.max_path);
    int64_t row, slot;
    const bool good = commit_step(a, seq, step, row, slot);
    // A row that is already at its position: no rotation.
    segs[id] = good ? StoreSegment{row, seq, 1, (int32_t)slot, (int32_t)slot} : StoreSegment{0, seq, 0, 0, 0};
}

}  // namespace

hipError_t launch_tree_masks(const TreeMaskArgs& a, hipStream_t stream) {
    hipLaunchKernelGGL(tree_masks, dim3((unsigned)a.n_seqs), dim3(256), 0, stream, a);
    return hipGetLastError();
}

namespace {
int verify_pieces(int vocab) { return (int)(((int64_t)vocab + kPiece - 1) / kPiece); }

template <typename T>
hipError_t launch_verify_t(const TreeVerifyArgs& a, hipStream_t stream) {
    const int pieces = verify_pieces(a.vocab);
    const bool draw = pieces <= kWalkPieces && (int64_t)a.vocab * (int)sizeof(T) * (a.draft ? 2 : 1) <= kWalkBytes;
    if (draw)
        hipLaunchKernelGGL((tree_walk<T, true>), dim3((unsigned)a.n_seqs), dim3(kWalkThreads), 0, stream, a);
    else
        hipLaunchKernelGGL((tree_walk<T, false>), dim3((unsigned)a.n_seqs), dim3(kWalkThreads), 0, stream, a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || draw) return e;
    hipLaunchKernelGGL((tree_sums<T>), dim3((unsigned)((pieces + 3) / 4), (unsigned)a.n_seqs), dim3(256), 0, stream, a, pieces);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((tree_pick<T>), dim3((unsigned)a.n_seqs), dim3(64), 0, stream, a, pieces);
    return hipGetLastError();
}
}  // namespace

size_t tree_verify_workspace_bytes(int n_seqs, int vocab) {
    return (size_t)n_seqs * (sizeof(VerifyState) + (size_t)verify_pieces(vocab) * sizeof(double));
}

hipError_t launch_tree_verify(const TreeVerifyArgs& a, hipStream_t stream) {
    return a.dtype == 1 ? launch_verify_t<float>(a, stream) : launch_verify_t<uint16_t>(a, stream);
}

hipError_t launch_tree_commit(const TreeCommitArgs& a, hipStream_t stream) {
    const int64_t pieces = (int64_t)a.n_layers * a.n_kv_heads * (a.row_bytes[0] + a.row_bytes[1]) / 16;
    const int64_t blocks = (pieces + 255) / 256;
    if (blocks > 0x7fffffff || a.max_path > 65535) return hipErrorInvalidValue;
    for (int seq0 = 0; seq0 < a.n_seqs; seq0 += 65535) {
        const int n = a.n_seqs - seq0 < 65535 ? a.n_seqs - seq0 : 65535;
        hipLaunchKernelGGL(tree_commit, dim3((unsigned)blocks, (unsigned)a.max_path, (unsigned)n), dim3(256), 0, stream, a, seq0);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

hipError_t launch_tree_segments(const TreeCommitArgs& a, StoreSegment* segs, hipStream_t stream) {
    const int64_t n = (int64_t)a.n_seqs * a.max_path;
    hipLaunchKernelGGL(tree_segments, dim3((unsigned)((n + 255) / 256)), dim3(256), 0, stream, a, segs);
    return hipGetLastError();
}

}  // namespace pkv
