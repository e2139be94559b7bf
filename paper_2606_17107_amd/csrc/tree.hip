// Trees of drafted tokens beside a cache: which rows descend from which (masks), the
// path that the target model's probabilities accept (verify), and the accepted rows'
// way into the cache (commit).
#include "attn_common.h"

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
template <typename T>
__device__ __forceinline__ double weight(const T* p, int64_t i);
template <>
__device__ __forceinline__ double weight<float>(const float* p, int64_t i) {
    const float x = p[i];
    return x > 0.f && x < INFINITY ? (double)x : 0.0;
}
template <>
__device__ __forceinline__ double weight<uint16_t>(const uint16_t* p, int64_t i) {
    const float x = __uint_as_float((uint32_t)p[i] << 16);
    return x > 0.f && x < INFINITY ? (double)x : 0.0;
}

constexpr int kVerifyChunk = 4096;   // probabilities per workgroup of the final draw

// What the walk leaves for the draw, one per sequence.
struct VerifyState {
    double a;          // weights max(p - a q, 0)
    int32_t cur;       // row of the tree where the walk ended, -1: no rows
    int32_t tried;     // its children were tried (and refused)
    uint32_t arrived;  // chunks whose sum is there
    uint32_t pad;
};

__device__ inline double wave_sum(double v) {
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) v += __shfl_xor(v, o);
    return v;
}

// Sum over a block of NW waves, in every thread.  `part`: NW doubles of LDS, free on entry.
template <int NW>
__device__ inline double block_sum(double v, double* part) {
    v = wave_sum(v);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
    __syncthreads();
    double s = 0.0;
#pragma unroll
    for (int w = 0; w < NW; ++w) s += part[w];
    __syncthreads();
    return s;
}

// The walk down one tree, one workgroup per sequence.  Every wave walks, from the same
// values in LDS, so the workgroup meets again only for sums over a row of
// probabilities: those are formed where a child drawn from the draft's probabilities
// is refused and a sibling is to be tried.
template <typename T>
__global__ __launch_bounds__(1024) void tree_walk(TreeVerifyArgs a) {
    constexpr int NT = 1024;
    __shared__ int parent[kTreeMaxRows], token[kTreeMaxRows];
    __shared__ float u[kTreeMaxRows], pr[kTreeMaxRows], qr[kTreeMaxRows];
    __shared__ double part[NT / 64];
    const int seq = (int)blockIdx.x, tid = threadIdx.x, lane = tid & 63;
    int q0, n;
    tree_rows(a.cu_q, a.total_q, seq, q0, n);
    n = min(n, a.max_q);
    VerifyState* const state = (VerifyState*)a.workspace + seq;
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
            pw = (float)weight(target + (int64_t)(q0 + p) * a.target_stride, t);
            if (draft) qw = (float)weight(draft + (int64_t)(q0 + p) * a.draft_stride, t);
        }
        parent[i] = p;
        token[i] = t;
        u[i] = a.u_accept[q0 + i];
        pr[i] = pw;
        qr[i] = qw;
    }
    __syncthreads();
    if (bad && a.err_flag) *a.err_flag = 1;

    int32_t* const path = a.path + (int64_t)seq * a.max_path;
    int cur = 0, length = n > 0 ? 1 : 0;
    bool tried = true;
    double wa = 0.0, wb = 1.0;   // the weights left at cur are max(p - wa q, 0), their sum is wb
    if (n > 0 && tid == 0) path[0] = q0;
    int i0 = 0;                  // rows before i0 are no more candidates
    while (n > 0) {
        if (length >= a.max_path) {
            tried = false;
            break;
        }
        // The next child of cur.
        int i = -1;
        for (int b = i0 & ~63; b < n && i < 0; b += 64) {
            const int r = b + lane;
            const uint64_t hit = __builtin_amdgcn_ballot_w64(r < n && r >= i0 && parent[min(r, n - 1)] == cur);
            if (hit) i = b + __builtin_ctzll(hit);
        }
        if (i < 0) break;
        i0 = i + 1;
        bool accept;
        double r;
        if (draft) {
            const double q = (double)qr[i];
            r = fmax((double)pr[i] - wa * q, 0.0);
            accept = r > 0.0 && (double)u[i] * q * wb < r;
        } else {
            // A token that a refused sibling had is gone.
            bool twin = false;
            for (int b = 0; b < i && !twin; b += 64) {
                const int j = b + lane;
                twin = __builtin_amdgcn_ballot_w64(j < i && parent[min(j, n - 1)] == cur && token[min(j, n - 1)] == token[i]) != 0;
            }
            r = twin ? 0.0 : (double)pr[i];
            accept = r > 0.0 && (double)u[i] * wb < r;
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
        bool more = false;
        for (int b = i0 & ~63; b < n && !more; b += 64) {
            const int j = b + lane;
            more = __builtin_amdgcn_ballot_w64(j < n && j >= i0 && parent[min(j, n - 1)] == cur) != 0;
        }
        if (!more) break;
        const T* const prow = target + (int64_t)(q0 + cur) * a.target_stride;
        const T* const qrow = draft + (int64_t)(q0 + cur) * a.draft_stride;
        double sum = 0.0;
#pragma unroll 8
        for (int v = tid; v < a.vocab; v += NT) sum += fmax(weight(prow, v) - wa * weight(qrow, v), 0.0);
        wb = block_sum<NT / 64>(sum, part);
    }
    for (int k = length + tid; k < a.max_path; k += NT) path[k] = -1;
    if (tid == 0) {
        a.n_accepted[seq] = length;
        if (n == 0) a.next_token[seq] = -1;
        *state = VerifyState{wa, n > 0 ? cur : -1, tried, 0, 0};
    }
}

// The draw from the weights that are left at the row where the walk ended.  One
// workgroup per chunk of the vocabulary and sequence sums its chunk; the last of a
// sequence to arrive finds the chunk, and in it the token, where the running sum
// passes u times the whole.  Running sums are formed in one order whatever the order
// of arrival.
template <typename T>
__global__ __launch_bounds__(256) void tree_draw(TreeVerifyArgs a, int chunks) {
    constexpr int NT = 256, PER = kVerifyChunk / NT;
    __shared__ uint32_t gone[kVerifyChunk / 32];   // tokens of refused children in the chunk
    __shared__ double part[NT / 64], sub[PER];
    __shared__ int last_arrival, first_over, last_full;
    const int seq = (int)blockIdx.y, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    VerifyState* const state = (VerifyState*)a.workspace + seq;
    double* const sums = (double*)((VerifyState*)a.workspace + a.n_seqs) + (int64_t)seq * chunks;
    const int cur = state->cur;
    if (cur < 0) return;
    double wa = state->a;
    bool tried = state->tried != 0;
    int q0, n;
    tree_rows(a.cu_q, a.total_q, seq, q0, n);
    n = min(n, a.max_q);
    const T* const prow = (const T*)a.target + (int64_t)(q0 + cur) * a.target_stride;
    const T* const qrow = a.draft ? (const T*)a.draft + (int64_t)(q0 + cur) * a.draft_stride : nullptr;

    auto load_gone = [&](int chunk) {
        if (qrow || !tried) return;   // uniform
        __syncthreads();
        for (int k = tid; k < kVerifyChunk / 32; k += NT) gone[k] = 0;
        __syncthreads();
        for (int i = cur + 1 + tid; i < n; i += NT) {
            const int t = a.tokens[q0 + i] - chunk * kVerifyChunk;
            if (a.parent[q0 + i] == cur && t >= 0 && t < kVerifyChunk) atomicOr(&gone[t >> 5], 1u << (t & 31));
        }
        __syncthreads();
    };
    // Weight of element k of a chunk.
    auto left = [&](int chunk, int k) -> double {
        const int64_t v = (int64_t)chunk * kVerifyChunk + k;
        if (v >= a.vocab) return 0.0;
        const double p = weight(prow, v);
        if (qrow) return fmax(p - wa * weight(qrow, v), 0.0);
        return tried && ((gone[k >> 5] >> (k & 31)) & 1) ? 0.0 : p;
    };
    auto chunk_sum = [&](int chunk) -> double {
        double s = 0.0;
#pragma unroll
        for (int e = 0; e < PER; ++e) s += left(chunk, e * NT + tid);
        return block_sum<NT / 64>(s, part);
    };

    const int mine = (int)blockIdx.x;
    load_gone(mine);
    const double my_sum = chunk_sum(mine);
    if (tid == 0) {
        __hip_atomic_store(&sums[mine], my_sum, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        last_arrival = __hip_atomic_fetch_add(&state->arrived, 1u, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT) == (uint32_t)chunks - 1;
    }
    __syncthreads();
    if (!last_arrival) return;

    auto sum_of = [&](int k) { return __hip_atomic_load(&sums[k], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); };
    // Inclusive running sum over the lanes of a wave.
    auto wave_scan = [&](double v) {
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const double up = __shfl_up(v, o);
            if (lane >= o) v += up;
        }
        return v;
    };
    // Every wave does this alike.  `total` is the running sum's own end, so that it is passed somewhere.
    auto find_chunk = [&](double u_at, double& before, bool& any) -> int {
        double total = 0.0;
        for (int b = 0; b < chunks; b += 64) {
            const double s = wave_scan(b + lane < chunks ? sum_of(b + lane) : 0.0);
            total += __shfl(s, 63);
        }
        any = total > 0.0;
        const double aim = u_at * total;
        double run = 0.0;
        int last = -1;
        double last_before = 0.0;
        for (int b = 0; b < chunks; b += 64) {
            const double one = b + lane < chunks ? sum_of(b + lane) : 0.0;
            const double s = run + wave_scan(one);
            const uint64_t full = __builtin_amdgcn_ballot_w64(one > 0.0), over = __builtin_amdgcn_ballot_w64(one > 0.0 && s > aim);
            const uint64_t pick = over ? over & (0 - over) : full;
            if (pick) {
                const int k = 63 - __builtin_clzll(pick);
                last = b + k;
                last_before = k > 0 ? __shfl(s, k - 1) : run;
                if (over) break;
            }
            run = __shfl(s, 63);
        }
        before = last_before;
        return last;
    };
    const double u_at = (double)a.u_sample[seq];
    double before;
    bool any;
    int chunk = find_chunk(u_at, before, any);
    if (!any) {
        // Nothing is left (target and draft agree, or every token was tried): the row's own probabilities.
        wa = 0.0;
        tried = false;
        __syncthreads();
        for (int k = 0; k < chunks; ++k) {
            const double s = chunk_sum(k);
            if (tid == 0) __hip_atomic_store(&sums[k], s, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        }
        __threadfence();
        __syncthreads();
        chunk = find_chunk(u_at, before, any);
        if (!any) {   // nor are there any
            if (tid == 0) {
                a.next_token[seq] = -1;
                if (a.err_flag) *a.err_flag = 1;
            }
            return;
        }
    }
    // The whole's sum once more (find_chunk's), for the aim.
    double total = 0.0;
    for (int b = 0; b < chunks; b += 64) total += __shfl(wave_scan(b + lane < chunks ? sum_of(b + lane) : 0.0), 63);
    const double aim = u_at * total;
    // In the chunk: sums of its runs of NT elements, then the running sum of one run.
    load_gone(chunk);
    for (int e = 0; e < PER; ++e) {
        const double s = block_sum<NT / 64>(left(chunk, e * NT + tid), part);
        if (tid == 0) sub[e] = s;
    }
    __syncthreads();
    int e_at = -1;
    double run = before, run_at = before;
    for (int e = 0; e < PER; ++e) {
        if (sub[e] > 0.0) {
            e_at = e;
            run_at = run;
            if (run + sub[e] > aim) break;
        }
        run += sub[e];
    }
    if (e_at < 0) e_at = 0;   // (a chunk with a sum above 0 has such a run)
    const double w = left(chunk, e_at * NT + tid);
    double s = wave_scan(w);
    if (lane == 63) part[wave] = s;
    __syncthreads();
    double base = run_at;
    for (int k = 0; k < wave; ++k) base += part[k];
    s += base;
    // The first element that passes the aim; where rounding leaves none, the last with a weight.
    if (tid == 0) {
        first_over = NT;
        last_full = -1;
    }
    __syncthreads();
    if (w > 0.0) {
        atomicMax(&last_full, tid);
        if (s > aim) atomicMin(&first_over, tid);
    }
    __syncthreads();
    if (tid == 0) {
        const int k = first_over < NT ? first_over : last_full;
        a.next_token[seq] = (int)((int64_t)chunk * kVerifyChunk + e_at * NT + max(k, 0));
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
int verify_chunks(int vocab) { return (int)(((int64_t)vocab + kVerifyChunk - 1) / kVerifyChunk); }

template <typename T>
hipError_t launch_verify_t(const TreeVerifyArgs& a, hipStream_t stream) {
    hipLaunchKernelGGL((tree_walk<T>), dim3((unsigned)a.n_seqs), dim3(1024), 0, stream, a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    const int chunks = verify_chunks(a.vocab);
    hipLaunchKernelGGL((tree_draw<T>), dim3((unsigned)chunks, (unsigned)a.n_seqs), dim3(256), 0, stream, a, chunks);
    return hipGetLastError();
}
}  // namespace

size_t tree_verify_workspace_bytes(int n_seqs, int vocab) {
    return (size_t)n_seqs * (sizeof(VerifyState) + (size_t)verify_chunks(vocab) * sizeof(double));
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
