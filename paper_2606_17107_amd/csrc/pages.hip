// Upkeep of a paged cache on the device: freeing, forking and compacting the pages
// of sequences, with counts of the block-table entries that refer to each page.  The
// cache's tensors are opaque bytes here (any dtype, scales as well as codes).
//
// A fork and a compaction are a plan, made by one workgroup in a single pass over
// the counts (who gets which page follows page and record numbers alone, so results
// do not depend on timing), and a launch that applies it: block-table rows and the
// copies of pages.  Nothing is read back by the host, so a captured graph replays
// them with whatever the tables hold then.  The copies are the cost, a stream read
// once and written once: 16-byte units, four loads in flight a thread, tiles of 16 KB.
// Measured: 220 pages of 1 MB moved, 88 us with the plan's 5 (copies at 5.5 TB/s, what a
// copy of this size reaches here; 103 with 2048 blocks that take several tiles each); 128
// forks with a last page of up to 64 x 8 x 128 codes in 8 layers copied, 39 us with 10 for
// the branches freed before and the plan (46 with the tiles of a layer neighbours: a short
// tail then leaves the same XCDs without work in every layer).
#include "attn_columns.h"

namespace pkv {
namespace {

constexpr int kPlan = 1024;        // threads of the planning workgroup
constexpr int kPer = 8;            // pages per thread and round of a scan
constexpr int kThreads = 256;
constexpr int kAhead = 4;          // units per thread whose loads are issued before the first store
constexpr int kTile = kThreads * kAhead;
constexpr int kBlocks = 16384;     // blocks of the applying launch at most: how many moves there are the host cannot know

// Exclusive prefix sum over the workgroup's threads, in thread order; *total is the
// sum.  Every thread takes part.
__device__ inline int block_scan(int v, int* total) {
    __shared__ int sums[kPlan / 64];
    const int wave = (int)threadIdx.x >> 6, lane = (int)threadIdx.x & 63;
    const int incl = wave_prefix_sum_i(v);
    __syncthreads();   // sums of an earlier call are read
    if (lane == 63) sums[wave] = incl;
    __syncthreads();
    int before = 0, all = 0;
#pragma unroll
    for (int w = 0; w < kPlan / 64; ++w) {
        const int s = sums[w];
        before += w < wave ? s : 0;
        all += s;
    }
    *total = all;
    return before + incl - v;
}

__device__ inline void flag(const PagesArgs& a) {
    if (a.err_flag) *a.err_flag = 1;
}
__device__ inline bool in_pool(const PagesArgs& a, int page) { return page >= 0 && page < a.n_pages; }

__global__ __launch_bounds__(kThreads) void pages_free_kernel(PagesArgs a) {
    const int seq = a.seqs[blockIdx.x];
    if (seq < 0 || seq >= a.n_seqs) {
        if (threadIdx.x == 0 && blockIdx.y == 0) flag(a);
        return;
    }
    int64_t keep = a.keep ? max(a.keep[blockIdx.x], 0) : 0;
    keep = (keep + a.page_size - 1) >> a.page_shift;
    for (int64_t e = keep + blockIdx.y * kThreads + threadIdx.x; e < a.max_pages; e += (int64_t)gridDim.y * kThreads) {
        int32_t* const at = a.table + (int64_t)seq * a.max_pages + e;
        if (*at == -1) continue;
        const int page = atomicExch(at, -1);   // once, also when a sequence is listed twice
        if (!in_pool(a, page)) {
            if (page != -1) flag(a);
            continue;
        }
        if (atomicSub(a.ref + page, 1) <= 0) {   // a page that nobody counted
            atomicAdd(a.ref + page, 1);
            flag(a);
        }
    }
}

constexpr int kNone = -1, kSkipped = -2;   // PagesArgs::pages of a fork

// Which records are valid, which page each new last page becomes, and the copies.
__global__ __launch_bounds__(kPlan) void pages_fork_plan(PagesArgs a) {
    const int t = threadIdx.x;
    const bool in_place = a.table_in == a.table;
    for (uint32_t s = t; s < (uint32_t)a.n_seqs; s += kPlan) a.claim[s] = 0x7fffffff;   // (an int would wrap on its last step)
    __syncthreads();
    auto in_range = [&](const PageFork& f) {
        return f.parent >= 0 && f.parent < a.n_seqs && f.child >= 0 && f.child < a.n_seqs && f.n_tokens >= 0 &&
               f.n_tokens <= (int64_t)a.max_pages * a.page_size;
    };
    for (int i = t; i < a.n; i += kPlan) {
        const PageFork f = a.forks[i];
        if (in_range(f)) atomicMin(a.claim + f.child, i);
    }
    auto claimed = [&](int s) { return __hip_atomic_load(a.claim + s, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); };
    __syncthreads();
    // Each record: skipped, without a new page, or its place among those that need one.
    int needed = 0;
    for (int i0 = 0; i0 < a.n; i0 += kPlan) {
        const int i = i0 + t;
        bool valid = false, wants = false;
        if (i < a.n) {
            const PageFork f = a.forks[i];
            valid = in_range(f) && claimed(f.child) == i && !(in_place && claimed(f.parent) != 0x7fffffff);
            const int tail = f.n_tokens & (a.page_size - 1);
            if (valid && tail) {
                const int page = a.table_in[(int64_t)f.parent * a.max_pages + (f.n_tokens >> a.page_shift)];
                wants = in_pool(a, page) && a.ref[page] > 0;
                if (!wants) flag(a);   // the parent has no such page, or one that nobody counts
            }
            if (!valid) flag(a);
        }
        int total;
        const int place = needed + block_scan(wants ? 1 : 0, &total);
        if (i < a.n) a.pages[i] = !valid ? kSkipped : wants ? place : kNone;
        needed += total;
    }
    // The lowest free pages, in order, until there are enough.
    int found = 0;
    for (int64_t p0 = 0; p0 < a.n_pages && found < needed; p0 += kPlan * kPer) {
        const int64_t p = p0 + t * kPer;
        uint32_t free = 0;
#pragma unroll
        for (int k = 0; k < kPer; ++k)
            if (p + k < a.n_pages && a.ref[p + k] == 0) free |= 1u << k;
        int total;
        int place = found + block_scan(__builtin_popcount(free), &total);
        while (free) {
            const int k = __builtin_ctz(free);
            free &= free - 1;
            if (place < needed) a.found[place] = (int)(p + k);
            ++place;
        }
        found += total;
    }
    found = min(found, needed);
    __syncthreads();
    for (int i = t; i < a.n; i += kPlan) {
        const int place = a.pages[i];
        if (place < 0) continue;
        if (place >= found) {   // the pool is full
            a.pages[i] = kNone;
            flag(a);
            continue;
        }
        const PageFork f = a.forks[i];
        const int page = a.found[place];
        a.pages[i] = page;
        a.ref[page] = 1;
        a.moves[place] = {a.table_in[(int64_t)f.parent * a.max_pages + (f.n_tokens >> a.page_shift)], page,
                          f.n_tokens & (a.page_size - 1), 0};
    }
    if (t == 0) a.head[0] = found;
}

// Pages in use, in page order: those from index n_used on move to the free ones below.
__global__ __launch_bounds__(kPlan) void pages_compact_plan(PagesArgs a) {
    const int t = threadIdx.x;
    int mine = 0, n;
    for (int64_t p = t; p < a.n_pages; p += kPlan) mine += a.ref_in[p] > 0 ? 1 : 0;
    block_scan(mine, &n);
    int holes = 0, movers = 0;
    for (int64_t p0 = 0; p0 < a.n_pages; p0 += kPlan * kPer) {
        const int64_t p = p0 + t * kPer;
        int ref[kPer], count = 0;
#pragma unroll
        for (int k = 0; k < kPer; ++k) {
            ref[k] = p + k < a.n_pages ? a.ref_in[p + k] : 0;
            const bool used = ref[k] > 0;
            if (p + k < a.n_pages && !used && p + k < n) count += 1;
            if (used && p + k >= n) count += 1 << 16;   // (at most 8192 of either)
        }
        int total;
        const int before = block_scan(count, &total);
        int hole = holes + (before & 0xffff), mover = movers + (before >> 16);
#pragma unroll
        for (int k = 0; k < kPer; ++k) {
            if (p + k >= a.n_pages) break;
            const bool used = ref[k] > 0, low = p + k < n;
            if (!used && low) a.moves[hole++].dst = (int)(p + k);
            if (used && !low) {
                a.moves[mover].src = (int)(p + k);
                a.moves[mover].tokens = a.page_size;
                a.moves[mover++].ref = ref[k];
            }
            a.pages[p + k] = used ? (int)(p + k) : kNone;
            a.ref[p + k] = used && low ? ref[k] : 0;
        }
        holes += total & 0xffff;
        movers += total >> 16;
    }
    __syncthreads();
    for (int i = t; i < movers; i += kPlan) {
        const PageMove m = a.moves[i];
        a.pages[m.src] = m.dst;
        a.ref[m.dst] = m.ref;
    }
    if (t == 0) {
        a.head[0] = movers;
        *a.n_used = n;
    }
}

// Units first .. first + kTile - 1 of a run of `units` in one piece from byte `at` of both pages.
template <typename T>
__device__ __forceinline__ void copy_run(const PageTensor& s, const PageMove& m, int64_t at, uint32_t first, uint32_t units) {
    const T* const from = (const T*)(s.data + (int64_t)m.src * s.page_stride + at) + first;
    T* const to = (T*)(s.data + (int64_t)m.dst * s.page_stride + at) + first;
    const uint32_t left = units - first;
    T v[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
        v[k] = __builtin_nontemporal_load(from + min(k * kThreads + threadIdx.x, left - 1));   // (no branches)
    }
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
        const uint32_t u = k * kThreads + threadIdx.x;
        if (u < left) __builtin_nontemporal_store(v[k], to + u);
    }
}

// The same of units counted over layers, slots and heads that lie apart.
template <typename T>
__device__ __forceinline__ void copy_units(const PageTensor& s, const PageMove& m, uint32_t first, uint32_t units_per_layer,
                                           uint32_t units) {
    T v[kAhead];
    char* to[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
        const uint32_t u = min(first + k * kThreads + threadIdx.x, units - 1);
        const uint32_t layer = u / units_per_layer;
        uint32_t rest = u - layer * units_per_layer;
        const uint32_t row = rest / (uint32_t)s.row_units;
        rest -= row * (uint32_t)s.row_units;
        const uint32_t slot = row / (uint32_t)s.heads;
        const int64_t at = (int64_t)layer * s.layer_stride + (int64_t)slot * s.slot_stride +
                           (int64_t)(row - slot * (uint32_t)s.heads) * s.head_stride + ((int64_t)rest << s.unit_shift);
        v[k] = __builtin_nontemporal_load((const T*)(s.data + (int64_t)m.src * s.page_stride + at));
        to[k] = s.data + (int64_t)m.dst * s.page_stride + at;
    }
#pragma unroll
    for (int k = 0; k < kAhead; ++k)
        if (first + k * kThreads + threadIdx.x < units) __builtin_nontemporal_store(v[k], (T*)to[k]);
}

// Block-table rows, and the copies: job j is a piece of the rows below row_jobs, then
// tile (move, tensor, tile of the tensor's share).  runs: tiles a layer of a tensor whose
// pages lie in one piece in each layer and fill half a tile or more there (no division a
// unit then), else 0.
template <bool FORK>
__global__ __launch_bounds__(kThreads) void pages_apply(PagesArgs a, int64_t row_jobs, int pieces, int4 tiles, int4 runs) {
    const int64_t per_move = (int64_t)tiles.x + tiles.y + tiles.z + tiles.w;
    const int64_t jobs = row_jobs + per_move * a.head[0];
    // Fork: the page had a count before the call.  One that the plan has handed out since has count 1 by
    // now (which nobody raises) and is among a.found, in ascending order.
    auto counted = [&](int page) {
        const int ref = a.ref[page];
        if (ref != 1) return ref > 0;
        int lo = 0, hi = a.head[0];
        while (lo < hi) {
            const int mid = (lo + hi) >> 1;
            if (a.found[mid] < page) lo = mid + 1;
            else hi = mid;
        }
        return lo == a.head[0] || a.found[lo] != page;
    };
    for (int64_t j = blockIdx.x; j < jobs; j += gridDim.x) {
        if (j < row_jobs) {
            if constexpr (FORK) {
                const int i = (int)(j / pieces);
                const int64_t e = (j - (int64_t)i * pieces) * kThreads + threadIdx.x;
                const int page = a.pages[i];
                if (page == kSkipped || e >= a.max_pages) continue;
                const PageFork f = a.forks[i];
                const int whole = f.n_tokens >> a.page_shift;
                int entry = kNone;
                if (e < whole) {
                    entry = a.table_in[(int64_t)f.parent * a.max_pages + e];
                    if (in_pool(a, entry) && counted(entry)) {
                        atomicAdd(a.ref + entry, 1);
                    } else {
                        entry = kNone;
                        flag(a);
                    }
                } else if (e == whole && (f.n_tokens & (a.page_size - 1))) {
                    entry = page;
                }
                a.table[(int64_t)f.child * a.max_pages + e] = entry;
            } else {
                const int64_t e = j * kThreads + threadIdx.x;
                if (e >= (int64_t)a.n_seqs * a.max_pages) continue;
                int entry = a.table_in[e];
                if (in_pool(a, entry)) {
                    entry = a.pages[entry];
                    if (entry < 0) flag(a);   // an entry of a page that nobody counts
                }
                a.table[e] = entry;
            }
            continue;
        }
        const int64_t c = j - row_jobs;
        const int64_t move = c / per_move;
        const PageMove m = a.moves[move];
        int tile = (int)(c - move * per_move), k = 0;
        const int n[4] = {tiles.x, tiles.y, tiles.z, tiles.w};
        const int r[4] = {runs.x, runs.y, runs.z, runs.w};
#pragma unroll
        for (int q = 0; q < 3; ++q) {
            if (k == q && tile >= n[q]) {
                tile -= n[q];
                k = q + 1;
            }
        }
        const PageTensor s = a.tensors[k];
        const uint32_t slots = (uint32_t)((m.tokens + s.slot_tokens - 1) / s.slot_tokens);
        const uint32_t per_layer = slots * (uint32_t)s.heads * (uint32_t)s.row_units;
        const int run = k == 0 ? r[0] : k == 1 ? r[1] : k == 2 ? r[2] : r[3];
        if (run) {
            // Layer after layer: what a short tail leaves without work is then shared by the XCDs, over
            // which blocks go round.
            const int piece = tile / s.layers, layer = tile - piece * s.layers;
            const uint32_t first = (uint32_t)piece * kTile;
            if (first >= per_layer) continue;
            const int64_t at = (int64_t)layer * s.layer_stride;
            switch (s.unit_shift) {
                case 4: copy_run<u32x4>(s, m, at, first, per_layer); break;
                case 3: copy_run<u32x2>(s, m, at, first, per_layer); break;
                case 2: copy_run<uint32_t>(s, m, at, first, per_layer); break;
                case 1: copy_run<uint16_t>(s, m, at, first, per_layer); break;
                default: copy_run<uint8_t>(s, m, at, first, per_layer); break;
            }
            continue;
        }
        const uint32_t units = per_layer * (uint32_t)s.layers;
        const uint32_t first = (uint32_t)tile * kTile;
        if (first >= units) continue;
        switch (s.unit_shift) {
            case 4: copy_units<u32x4>(s, m, first, per_layer, units); break;
            case 3: copy_units<u32x2>(s, m, first, per_layer, units); break;
            case 2: copy_units<uint32_t>(s, m, first, per_layer, units); break;
            case 1: copy_units<uint16_t>(s, m, first, per_layer, units); break;
            default: copy_units<uint8_t>(s, m, first, per_layer, units); break;
        }
    }
}

// Pieces of a block-table row, an entry a thread.
int row_pieces(const PagesArgs& a) { return (a.max_pages - 1) / kThreads + 1; }

template <bool FORK>
hipError_t launch_apply(const PagesArgs& a, hipStream_t stream) {
    const int pieces = row_pieces(a);
    const int64_t row_jobs = FORK ? (int64_t)a.n * pieces : ((int64_t)a.n_seqs * a.max_pages + kThreads - 1) / kThreads;
    int tiles[4] = {0, 0, 0, 0}, runs[4] = {0, 0, 0, 0};
    int64_t per_move = 0;
    for (int k = 0; k < a.n_tensors; ++k) {
        const PageTensor& s = a.tensors[k];
        const int64_t layer_units = (int64_t)s.slots * s.heads * s.row_units;
        const int64_t row = (int64_t)s.row_units << s.unit_shift;
        if ((s.heads == 1 || s.head_stride == row) && (s.slots == 1 || s.slot_stride == row * s.heads) &&
            layer_units >= kTile / 2)
            runs[k] = (int)((layer_units + kTile - 1) / kTile);
        tiles[k] = runs[k] ? runs[k] * s.layers : (int)((layer_units * s.layers + kTile - 1) / kTile);
        per_move += tiles[k];
    }
    // The number of moves is known on the device: at most one a fork, or half the pages.
    const int64_t jobs = row_jobs + per_move * (FORK ? a.n : a.n_pages / 2);
    if (jobs <= 0) return hipSuccess;
    const dim3 grid((unsigned)(jobs < kBlocks ? jobs : kBlocks));
    hipLaunchKernelGGL((pages_apply<FORK>), grid, dim3(kThreads), 0, stream, a, row_jobs, pieces,
                       make_int4(tiles[0], tiles[1], tiles[2], tiles[3]), make_int4(runs[0], runs[1], runs[2], runs[3]));
    return hipGetLastError();
}

size_t up16(size_t n) { return (n + 15) & ~(size_t)15; }

}  // namespace

// Workspace: [head][moves][pages][found][claim], each on a 16-byte boundary.
size_t pages_workspace_bytes(const PagesArgs& a, int n_forks) {
    const size_t moves = n_forks ? (size_t)n_forks : (size_t)(a.n_pages / 2);
    size_t n = 16 + moves * sizeof(PageMove);
    if (n_forks) n += 2 * up16((size_t)n_forks * 4) + up16((size_t)a.n_seqs * 4);
    else n += up16((size_t)a.n_pages * 4);
    return n;
}
void pages_set_workspace(PagesArgs& a, int n_forks, void* ws) {
    char* p = (char*)ws;
    a.head = (int32_t*)p;
    p += 16;
    a.moves = (PageMove*)p;
    p += (n_forks ? (size_t)n_forks : (size_t)(a.n_pages / 2)) * sizeof(PageMove);
    a.pages = (int32_t*)p;
    if (!n_forks) return;
    p += up16((size_t)n_forks * 4);
    a.found = (int32_t*)p;
    p += up16((size_t)n_forks * 4);
    a.claim = (int32_t*)p;
}

hipError_t launch_pages_free(const PagesArgs& a, hipStream_t stream) {
    const int y = row_pieces(a);
    hipLaunchKernelGGL(pages_free_kernel, dim3((unsigned)a.n, (unsigned)(y < 64 ? y : 64)), dim3(kThreads), 0, stream, a);
    return hipGetLastError();
}

hipError_t launch_pages_fork(const PagesArgs& a, hipStream_t stream) {
    hipLaunchKernelGGL(pages_fork_plan, dim3(1), dim3(kPlan), 0, stream, a);
    const hipError_t e = hipGetLastError();
    return e != hipSuccess ? e : launch_apply<true>(a, stream);
}

hipError_t launch_pages_compact(const PagesArgs& a, hipStream_t stream) {
    hipLaunchKernelGGL(pages_compact_plan, dim3(1), dim3(kPlan), 0, stream, a);
    const hipError_t e = hipGetLastError();
    return e != hipSuccess ? e : launch_apply<false>(a, stream);
}

}  // namespace pkv
