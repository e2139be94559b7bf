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
// many LDS reads as the tree is deep): 4.8 us back to back for 1 tree of 16 rows and for 256
// trees of up to 64, of which the kernel takes 1.7 and 2.7.
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
__device__ __forceinline__ double as_weight(float x) {
    constexpr int kPositive = 0x180;   // the classes of positive subnormal and normal numbers
    return (double)(__builtin_amdgcn_classf(x, kPositive) ? x : 0.f);
}
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

// A piece of a row (and of the draft's) as it lies in memory: element 64 VE e + VE lane + k
// of the piece is x[k] of p[e].  Elements behind the row are 0.
template <typename T>
struct Piece {
    static constexpr int VE = 16 / (int)sizeof(T), E = kPiece / 64 / VE;
    Probs<T> p[E], q[E];

    // A piece that lies in the row whole.
    template <bool DRAFT>
    __device__ __forceinline__ void load_whole(const Weights<T>& r, int piece) {
        const int64_t at = (int64_t)piece * kPiece + (int)__lane_id() * VE;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            p[e] = *(const Probs<T>*)(r.p + at + e * 64 * VE);
            if (DRAFT) q[e] = *(const Probs<T>*)(r.q + at + e * 64 * VE);
        }
    }
    __device__ __forceinline__ void load(const Weights<T>& r, int piece) {
        const int lane = (int)__lane_id();
        const int64_t base = (int64_t)piece * kPiece;
        if (base + kPiece <= r.vocab) {   // uniform
            if (r.q) load_whole<true>(r, piece);
            else load_whole<false>(r, piece);
        } else {
#pragma unroll
            for (int e = 0; e < E; ++e)
#pragma unroll
                for (int k = 0; k < VE; ++k) {
                    const int v = (int)base + (e * 64 + lane) * VE + k, at = min(v, r.vocab - 1);   // (no branches)
                    const T x = r.p[at], y = r.q ? r.q[at] : (T)0;
                    p[e].x[k] = v < r.vocab ? x : (T)0;
                    q[e].x[k] = v < r.vocab ? y : (T)0;
                }
        }
    }
    // The weights.  gone: null, or 32 words of LDS whose bits are elements that count as 0.
    __device__ __forceinline__ void weights(const Weights<T>& r, const uint32_t* gone, double (&w)[E][VE]) const {
        const int lane = (int)__lane_id();
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
    __device__ __forceinline__ double lane_sum(const Weights<T>& r, const uint32_t* gone) const {
        double w[E][VE], s = 0.0;
        weights(r, gone, w);
#pragma unroll
        for (int e = 0; e < E; ++e)
#pragma unroll
            for (int k = 0; k < VE; ++k) s += w[e][k];
        return s;
    }
};

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
__device__ __forceinline__ float lane_float(float v, int lane) {
    return __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(v), lane));
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
template <typename T>
__device__ __forceinline__ double piece_sum(const Weights<T>& r, int piece, const uint32_t* gone) {
    Piece<T> x;
    x.load(r, piece);
    return wave_sum(x.lane_sum(r, gone));
}

// Sums of all pieces of a row, by NW waves of which this is number `wave`.  A wave has
// the loads of four whole pieces in flight (4 trees of 32 drawn tokens, 3 children a
// row, over 100000: 81 us a call; with one piece and the next one's loads 96 us).  A
// pass of one workgroup is then held up about alike by its conversions to 64 bits, 9 instructions
// for each pair of probabilities, and by its loads: VALU instructions issue in 52% of the
// cycles of the SIMDs that hold its waves, which wait for 41% of theirs.
template <int NW, bool DRAFT, typename T>
__device__ __forceinline__ void sum_pieces(const Weights<T>& r, int pieces, int wave, double* sums) {
    constexpr int N = 4;
    const int whole = r.vocab / kPiece;
    for (int k0 = wave; k0 < whole; k0 += N * NW) {
        Piece<T> x[N];
#pragma unroll
        for (int j = 0; j < N; ++j) x[j].template load_whole<DRAFT>(r, min(k0 + j * NW, whole - 1));
#pragma unroll
        for (int j = 0; j < N; ++j) {
            if (k0 + j * NW < whole) {   // uniform
                const double v = wave_sum(x[j].lane_sum(r, nullptr));
                if (__lane_id() == 0) sums[k0 + j * NW] = v;
            }
        }
    }
    if (whole < pieces && wave == whole % NW) {
        const double v = piece_sum(r, whole, nullptr);
        if (__lane_id() == 0) sums[whole] = v;
    }
}

// Tokens that were tried and lie in a piece, as bits of 32 words of LDS that the wave has
// to itself; null if there are none.  at(i): the token of row i if it was tried, else -1.
template <typename F>
__device__ __forceinline__ const uint32_t* tried_tokens(int piece, int n, uint32_t* words, F at) {
    const int lane = (int)__lane_id();
    bool any = false;
    for (int b = 0; b < n; b += 64) {
        const int t = b + lane < n ? at(b + lane) : -1;
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
    constexpr int VE = Piece<T>::VE, E = Piece<T>::E;
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
    Piece<T> x;
    x.load(r, piece);
    x.weights(r, gone(piece), w);
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

// Where a walk is.
struct Walk {
    double a, b;       // the weights left at cur are max(p - a q, 0), their sum is taken to be b
    int cur;           // row where the walk is
    int next;          // first row that may be cur's next child
    int length;        // rows on the path
    bool tried;        // cur's children before `next` were tried, and refused
    bool pending;      // b is to be summed before the next child is tried
};

// Steps down the tree until it ends or a sum is needed (w.b, where w.pending).  child(cur, from, to, x): first
// child of cur in rows [from, to), with token x if x >= 0; -1: none.  token, pr, qr, u:
// values of a row; accept(i, length): row i is on the path.
template <typename C, typename X, typename P, typename Q, typename U, typename A>
__device__ __forceinline__ void walk(Walk& w, bool drawn, int n, int max_path, C child, X token, P pr, Q qr, U u, A accept) {
    w.pending = false;
    for (;;) {
        if (w.length >= max_path) {
            w.tried = false;
            return;
        }
        const int i = child(w.cur, w.next, n, -1);
        if (i < 0) return;
        w.next = i + 1;
        double r, bar;
        if (drawn) {
            const double q = (double)qr(i);
            r = fmax((double)pr(i) - w.a * q, 0.0);
            bar = (double)u(i) * q * w.b;
        } else {
            // A token that a refused sibling had is gone.
            r = child(w.cur, w.cur + 1, i, token(i)) >= 0 ? 0.0 : (double)pr(i);
            bar = (double)u(i) * w.b;
        }
        if (r > 0.0 && bar < r) {
            accept(i, w.length);
            ++w.length;
            w.cur = i;
            w.a = 0.0;
            w.b = 1.0;
        } else if (!drawn) {
            w.b -= r;
        } else {
            w.a += w.b;
            w.pending = child(w.cur, w.next, n, -1) >= 0;   // the sum is needed only if another child follows
            return;
        }
    }
}

// What a launch leaves for the next, one per sequence.
struct VerifyState {
    double a;
    int32_t cur;       // -1: no rows
    int32_t next;
    int32_t length;
    int32_t flags;     // 1: tried, 2: pending
    int32_t pad[2];
};

// Rows of the tree: a row's parent (-1: no candidate) and token, and its token's weights
// at the parent.
struct TreeRow {
    int parent, token;
    float p, q, u;
};
template <typename T>
__device__ __forceinline__ TreeRow load_row(const TreeVerifyArgs& a, int q0, int i, bool& bad) {
    TreeRow r;
    r.parent = a.parent[q0 + i];
    r.token = a.tokens[q0 + i];
    r.u = a.u_accept[q0 + i];
    r.p = r.q = 0.f;
    if (i == 0) {
        r.parent = -1;
    } else if (r.parent < -1 || r.parent >= i || r.token < 0 || r.token >= a.vocab) {
        bad = true;
        r.parent = -1;
    }
    if (r.parent >= 0) {
        r.p = (float)as_weight(((const T*)a.target)[(int64_t)(q0 + r.parent) * a.target_stride + r.token]);
        if (a.draft) r.q = (float)as_weight(((const T*)a.draft)[(int64_t)(q0 + r.parent) * a.draft_stride + r.token]);
    }
    return r;
}

template <typename T>
__device__ __forceinline__ Weights<T> row_weights(const TreeVerifyArgs& a, int row, double wa) {
    return Weights<T>{(const T*)a.target + (int64_t)row * a.target_stride,
                      a.draft ? (const T*)a.draft + (int64_t)row * a.draft_stride : nullptr, wa, a.vocab};
}

__device__ __forceinline__ double* piece_sums(const TreeVerifyArgs& a, int seq, int pieces) {
    return (double*)((VerifyState*)a.workspace + a.n_seqs) + (int64_t)seq * pieces;
}

// A tree as a wave walks it: values of up to 64 rows are held by its lanes, of more rows
// read from LDS.
struct TreeLds {
    int parent[kTreeMaxRows], token[kTreeMaxRows];
    float u[kTreeMaxRows], p[kTreeMaxRows], q[kTreeMaxRows];
};
// By all threads of a workgroup of NT, which meet at the end.
template <typename T, int NT>
__device__ __forceinline__ bool load_tree(const TreeVerifyArgs& a, int q0, int n, TreeLds& t) {
    bool bad = false;
    for (int i = threadIdx.x; i < n; i += NT) {
        const TreeRow r = load_row<T>(a, q0, i, bad);
        t.parent[i] = r.parent;
        t.token[i] = r.token;
        t.u[i] = r.u;
        t.p[i] = r.p;
        t.q[i] = r.q;
    }
    __syncthreads();
    return bad;
}
template <typename A>
__device__ __forceinline__ void walk_tree(Walk& w, const TreeVerifyArgs& a, int n, const TreeLds& t, A accept) {
    const int lane = (int)__lane_id(), mine = min(lane, n - 1);
    const bool held = n <= 64;
    const int my_parent = t.parent[mine], my_token = t.token[mine];
    const float my_u = t.u[mine], my_p = t.p[mine], my_q = t.q[mine];
    auto child = [&](int cur, int from, int to, int x) __attribute__((always_inline)) {
        for (int b = held ? 0 : from & ~63; b < to; b += 64) {
            const int r = b + lane, at = min(r, n - 1);
            const bool is = (held ? my_parent : t.parent[at]) == cur && (x < 0 || (held ? my_token : t.token[at]) == x);
            const uint64_t hit = __builtin_amdgcn_ballot_w64(r >= from && r < to && is);
            if (hit) return b + (int)__builtin_ctzll(hit);
        }
        return -1;
    };
    walk(w, a.draft != nullptr, n, a.max_path, child,
         [&](int i) { return held ? __builtin_amdgcn_readlane(my_token, i) : t.token[i]; },
         [&](int i) { return held ? lane_float(my_p, i) : t.p[i]; }, [&](int i) { return held ? lane_float(my_q, i) : t.q[i]; },
         [&](int i) { return held ? lane_float(my_u, i) : t.u[i]; }, accept);
}

__device__ __forceinline__ VerifyState verify_state(const Walk& w) {
    return VerifyState{w.a, w.cur, w.next, w.length, (w.tried ? 1 : 0) | (w.pending ? 2 : 0), {0, 0}};
}
// (n_accepted and path of a sequence without rows)
__device__ __forceinline__ void no_rows(const TreeVerifyArgs& a, int seq, int from, int step) {
    for (int k = from; k < a.max_path; k += step) a.path[(int64_t)seq * a.max_path + k] = -1;
    if (from != 0) return;
    a.n_accepted[seq] = 0;
    a.next_token[seq] = -1;
    ((VerifyState*)a.workspace)[seq].cur = -1;
}

// The walk from the root on of trees of more than 64 rows, one workgroup each; as far as
// it goes without a sum.  (The trees of up to 64 rows: tree_sums.)
template <typename T>
__global__ __launch_bounds__(256) void tree_walk(TreeVerifyArgs a) {
    __shared__ TreeLds t;
    const int seq = (int)blockIdx.x;
    int q0, n;
    tree_rows(a.cu_q, a.total_q, seq, q0, n);
    n = min(n, a.max_q);
    if (n == 0) return no_rows(a, seq, threadIdx.x, 256);
    if (load_tree<T, 256>(a, q0, n, t) && a.err_flag) *a.err_flag = 1;
    if (threadIdx.x >= 64) return;
    int32_t* const path = a.path + (int64_t)seq * a.max_path;
    const int lane = (int)__lane_id();
    if (lane == 0) path[0] = q0;
    Walk w{0.0, 1.0, 0, 1, 1, true, false};
    walk_tree(w, a, n, t, [&](int i, int at) {
        if (lane == 0) path[at] = q0 + i;
    });
    for (int k = w.length + lane; k < a.max_path; k += 64) path[k] = -1;
    if (lane == 0) {
        a.n_accepted[seq] = w.length;
        ((VerifyState*)a.workspace)[seq] = verify_state(w);
    }
}

// Behind tree_sums, one workgroup per sequence: what is left of a walk that needs sums
// (a drawn token was refused where a sibling follows: the first such sum is that of
// tree_sums' pieces, the workgroup forms the others), and the draw.  Where nothing is left
// to walk it is a chain of state, sums and one piece: 4 to 5.6 us.  (512 threads: more
// would leave a wave fewer registers than the sums of a piece and the search need.)
constexpr int kFinishThreads = 512;
template <typename T>
__global__ __launch_bounds__(kFinishThreads) void tree_finish(TreeVerifyArgs a, int pieces) {
    constexpr int NW = kFinishThreads / 64;
    __shared__ TreeLds t;
    __shared__ uint32_t bits[kPiece / 32];
    __shared__ int found;
    const int seq = (int)blockIdx.x, lane = (int)__lane_id();
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    double* const sums = piece_sums(a, seq, pieces);
    const VerifyState s = ((const VerifyState*)a.workspace)[seq];
    const float u_draw = a.u_sample[seq];
    int q0, n;
    tree_rows(a.cu_q, a.total_q, seq, q0, n);
    n = min(n, a.max_q);
    if (s.cur < 0) return;
    int32_t* const path = a.path + (int64_t)seq * a.max_path;
    Walk w{s.a, 0.0, s.cur, s.next, s.length, (s.flags & 1) != 0, (s.flags & 2) != 0};
    bool by_tokens = w.tried && !a.draft;
    if (w.pending) load_tree<T, kFinishThreads>(a, q0, n, t);
    // `sums` are those of the weights where the walk is.
    for (bool again = false;;) {
        if (w.pending) {
            double b = 0.0;
            for (int k = lane; k < pieces; k += 64) b += sums[k];
            w.b = wave_sum(b);   // (alike in every wave)
            walk_tree(w, a, n, t, [&](int i, int at) {
                if (threadIdx.x == 0) path[at] = q0 + i;
            });
            if (threadIdx.x == 0) a.n_accepted[seq] = w.length;
        } else {
            if (wave == 0) {
                const int next = find_token(row_weights<T>(a, q0 + w.cur, w.a), pieces, (double)u_draw, [&](int k) { return sums[k]; },
                                            [&](int k) -> const uint32_t* {
                    if (!by_tokens) return nullptr;
                    return tried_tokens(k, n, bits, [&](int i) { return i > w.cur && a.parent[q0 + i] == w.cur ? a.tokens[q0 + i] : -1; });
                });
                if (lane == 0) found = next;
            }
            __syncthreads();
            if (found >= 0 || again) break;
            again = true;   // nothing is left: the row's own probabilities
            w.a = 0.0;
            by_tokens = false;
        }
        __syncthreads();
        // The sums of the weights where the walk is now.
        const Weights<T> r = row_weights<T>(a, q0 + w.cur, w.a);
        if (r.q) sum_pieces<NW, true>(r, pieces, wave, sums);
        else sum_pieces<NW, false>(r, pieces, wave, sums);
        __syncthreads();
    }
    if (threadIdx.x == 0) {
        a.next_token[seq] = found;
        if (found < 0 && a.err_flag) *a.err_flag = 1;
    }
}

// Sums of the weights at the row where a walk ends, one wave for each piece of the row.
// WALK: trees of at most 64 rows; each wave walks by itself, one row a lane, and piece
// 0's wave reports the path.  A walk that needs a sum itself stops there (the sum is
// that of the pieces), and the workgroup that draws the token goes on.  The walk is a
// chain of loads (bounds; parents and tokens; their probabilities) of 4 us that every wave
// spends at the same time, then each wave has its piece in flight whole: 64 chains of 8
// drawn tokens of 131072, fp32, 67 MB in 14.4 us; in a launch of its own before the sums the walk costs
// 6 us more (26.3 against 19.8 us a call), and the whole verification in one launch, whose last
// arrival draws the token, 16 trees of up to 48 rows of 100003 tokens 25 us against 11.8.
template <typename T, bool WALK>
__global__ __launch_bounds__(256) void tree_sums(TreeVerifyArgs a, int pieces) {
    __shared__ uint32_t bits[4][kPiece / 32];
    const int seq = (int)blockIdx.y, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = (int)__lane_id();
    const int k = (int)blockIdx.x * 4 + wave;
    if (k >= pieces) return;
    VerifyState* const state = (VerifyState*)a.workspace + seq;
    int q0, n;
    tree_rows(a.cu_q, a.total_q, seq, q0, n);
    n = min(n, a.max_q);
    const uint32_t* gone = nullptr;
    int cur;
    double wa;
    if constexpr (WALK) {
        int32_t* const path = a.path + (int64_t)seq * a.max_path;
        if (n == 0) {
            if (k == 0) no_rows(a, seq, lane, 64);
            return;
        }
        bool bad = false;
        TreeRow r{-1, -1, 0.f, 0.f, 0.f};
        if (lane < n) r = load_row<T>(a, q0, lane, bad);
        auto child = [&](int c, int from, int to, int x) __attribute__((always_inline)) {
            const uint64_t hit = __builtin_amdgcn_ballot_w64(lane >= from && lane < to && r.parent == c && (x < 0 || r.token == x));
            return hit ? (int)__builtin_ctzll(hit) : -1;
        };
        int on_path = q0;   // lane j: row j of the path
        Walk w{0.0, 1.0, 0, 1, 1, true, false};
        walk(w, a.draft != nullptr, n, a.max_path, child, [&](int i) { return __builtin_amdgcn_readlane(r.token, i); },
             [&](int i) { return lane_float(r.p, i); }, [&](int i) { return lane_float(r.q, i); },
             [&](int i) { return lane_float(r.u, i); }, [&](int i, int at) { on_path = lane == at ? q0 + i : on_path; });
        cur = w.cur;
        wa = w.a;
        if (!a.draft && w.tried)
            gone = tried_tokens(k, n, bits[wave], [&](int) { return r.parent == cur ? r.token : -1; });
        if (k == 0) {
            if (bad && a.err_flag) *a.err_flag = 1;
            for (int i = lane; i < a.max_path; i += 64) path[i] = i < w.length ? on_path : -1;
            if (lane == 0) {
                a.n_accepted[seq] = w.length;
                *state = verify_state(w);
            }
        }
    } else {
        const VerifyState s = *state;
        cur = s.cur;
        wa = s.a;
        if (cur < 0) return;
        if (!a.draft && (s.flags & 1))
            gone = tried_tokens(k, n, bits[wave], [&](int i) { return i > cur && a.parent[q0 + i] == cur ? a.tokens[q0 + i] : -1; });
    }
    const double s = piece_sum(row_weights<T>(a, q0 + cur, wa), k, gone);
    if (lane == 0) piece_sums(a, seq, pieces)[k] = s;
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

constexpr int kCommitThreads = 128;

// A thread moves one 16-byte piece of one accepted row: pieces of a row's keys, then of
// its values, layer by layer; a workgroup has one step of one sequence.  Small calls are
// a chain (counts, path and lengths; page entry; row), large ones a stream, whose
// stores go past the caches: 64 sequences of 1..8 rows, 8 layers of 8 heads of 128 in
// bf16 pages 6.6 us a call replayed from a graph over four caches (6.0 issued one by
// one; with 256 threads 7.1, with cached stores 7.3, with eight steps a thread, all
// their loads in flight, 11.3), 32 layers of 4 heads of 128 in fp32 15.9 us (cached
// stores 19.8), 72 MB read and written.
__global__ __launch_bounds__(kCommitThreads) void tree_commit(TreeCommitArgs a, int seq0) {
    const int seq = seq0 + (int)blockIdx.z, step = (int)blockIdx.y;
    int64_t row, slot;
    if (!commit_step(a, seq, step, row, slot)) return;
    const int kc = a.row_bytes[0] / 16, vc = a.row_bytes[1] / 16;   // pieces of a row of one head
    const int per_layer = a.n_kv_heads * (kc + vc);
    const int64_t id = (int64_t)blockIdx.x * kCommitThreads + threadIdx.x;
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
    __builtin_nontemporal_store(x, (u32x4*)(a.dst[t] + dst + c * 16));
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
    const dim3 seqs((unsigned)a.n_seqs);
    const dim3 grid((unsigned)((pieces + 3) / 4), (unsigned)a.n_seqs);
    if (a.max_q <= 64) {
        hipLaunchKernelGGL((tree_sums<T, true>), grid, dim3(256), 0, stream, a, pieces);
    } else {
        hipLaunchKernelGGL((tree_walk<T>), seqs, dim3(256), 0, stream, a);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        hipLaunchKernelGGL((tree_sums<T, false>), grid, dim3(256), 0, stream, a, pieces);
    }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((tree_finish<T>), seqs, dim3(kFinishThreads), 0, stream, a, pieces);
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
    const int64_t blocks = (pieces + kCommitThreads - 1) / kCommitThreads;
    if (blocks > 0x7fffffff || a.max_path > 65535) return hipErrorInvalidValue;
    for (int seq0 = 0; seq0 < a.n_seqs; seq0 += 65535) {
        const int n = a.n_seqs - seq0 < 65535 ? a.n_seqs - seq0 : 65535;
        hipLaunchKernelGGL(tree_commit, dim3((unsigned)blocks, (unsigned)a.max_path, (unsigned)n), dim3(kCommitThreads), 0, stream, a, seq0);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace pkv
