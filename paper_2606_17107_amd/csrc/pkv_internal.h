// Internal interface between the C ABI (api.hip) and the kernel launchers.
// Nothing here is exported from libpkv.so.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace pkv {

// ---- reposition + splice ---------------------------------------------------

struct SpliceSegment {   // same layout as pkv_segment in pkv.h
    int64_t src_slot0;
    int64_t dst_seq_base;
    int32_t n_tokens;
    int32_t src_pos0;
    int32_t dst_pos0;
    int32_t dst_seq_len;
};

struct SpliceArgs {
    const char* src_k;
    const char* src_v;
    char* dst_k;
    char* dst_v;
    // per-token mode
    const int32_t* src_pos;
    const int32_t* dst_pos;
    const int32_t* dst_slot;  // destination slots, or null (slot = dst_pos)
    // segment mode
    const SpliceSegment* segs;
    int32_t n_segs;
    int32_t max_seg_tokens;

    int32_t elem_bytes;      // 2 (bf16) or 4 (fp32)
    int32_t rope_style;
    int32_t n_layers;
    int32_t n_kv_heads;
    int32_t head_dim;
    int32_t v_dim;
    int32_t rope_offset;
    int32_t rope_dim;
    int64_t n_tokens;        // per-token mode: tokens; segment mode: source slots
    int64_t dst_capacity;
    double theta;
    const double* omega;      // host, rope_dim/2 per-pair frequencies, or null (theta schedule)
    int64_t src_k_stride[3];  // elements
    int64_t src_v_stride[3];
    int64_t dst_k_stride[3];
    int64_t dst_v_stride[3];
    int32_t* err_flag;
    // paged destination (per-token mode): logical slot p -> page
    // dst_pages[p >> page_shift], in-page slot p & (page_size - 1)
    const int32_t* dst_pages;  // null: contiguous destination
    const int32_t* dst_v_pages;  // V through its own table, or null (dst_pages)
    int32_t page_shift;
    int32_t max_pages;
    int64_t n_pages;
    int64_t dst_k_page_stride;  // elements
    int64_t dst_v_page_stride;
};

hipError_t launch_splice(const SpliceArgs& a, hipStream_t stream);

// ---- reposition + splice into a cache held in 8 bits ---------------------------

struct StoreSegment {   // same layout as pkv_segment_quant in pkv.h
    int64_t src_slot0;
    int32_t seq;
    int32_t n_tokens;
    int32_t src_pos0;
    int32_t dst_pos0;
};

struct StoreArgs {
    const char* src_k;
    const char* src_v;        // may be null
    uint8_t* dst_k;
    uint8_t* dst_v;
    const StoreSegment* segs;
    int32_t n_segs;
    int32_t max_seg_tokens;
    const int32_t* kv_len;    // slots in use before the call, per sequence
    int32_t n_seqs;
    int32_t elem_bytes;       // of the source: 2 (bf16) or 4 (fp32)
    int32_t rope_style;
    int32_t n_layers;
    int32_t n_kv_heads;
    int32_t head_dim;
    int32_t rope_offset;
    int32_t rope_dim;
    int64_t n_src;            // source slots
    int64_t dst_capacity;     // logical slots per sequence
    double theta;
    const double* omega;      // host, rope_dim/2 per-pair frequencies, or null (theta schedule)
    int64_t src_k_stride[3];  // elements
    int64_t src_v_stride[3];
    int64_t dst_k_stride[3];  // bytes
    int64_t dst_v_stride[3];
    int32_t* err_flag;
    const int32_t* block_table;
    const int32_t* v_block_table;  // may be null (block_table)
    int32_t page_shift;
    int32_t max_pages;
    int64_t n_pages;
    int64_t dst_k_page_stride;
    int64_t dst_v_page_stride;
    int32_t block_tokens;     // 32, 64 or 128
    uint8_t* k_scale;
    uint8_t* v_scale;
    int64_t k_scale_stride[4];   // {layer, head, page, block in page}
    int64_t v_scale_stride[4];
    // instead of segments (then n_segs is n_seqs): sequence s appends source rows
    // rows[s][0 .. n_rows[s]) of at most max_rows, unturned, behind its kv_len[s] slots
    const int32_t* rows;      // or null
    const int32_t* n_rows;
    int32_t max_rows;
};

bool store_fits(const StoreArgs& a);   // the launch is within the grid's limits
hipError_t launch_store(const StoreArgs& a, hipStream_t stream);

// ---- pages -----------------------------------------------------------------------

// One tensor of a page pool as the copies see it: a page of a layer is `slots` runs
// of `heads` rows; row bytes are moved in units of 2^unit_shift bytes.
struct PageTensor {
    char* data;
    int64_t layer_stride, page_stride, slot_stride, head_stride;   // bytes
    int32_t layers, slots, heads;
    int32_t row_units;        // units of one row
    int32_t unit_shift;       // 0 .. 4
    int32_t slot_tokens;      // cache slots of one of `slots`
};
struct PageMove {
    int32_t src, dst;
    int32_t tokens;           // live slots of the page
    int32_t ref;
};
struct PageFork {   // same layout as pkv_fork in pkv.h
    int32_t parent, child, n_tokens, reserved;
};
struct PagesArgs {
    PageTensor tensors[4];
    int32_t n_tensors;
    int32_t page_size, page_shift;
    int32_t n_seqs, max_pages;
    int64_t n_pages;
    int32_t* err_flag;
    const int32_t* ref_in;
    int32_t* ref;             // counts (fork, free), new counts (compact)
    const int32_t* table_in;
    int32_t* table;
    const PageFork* forks;
    int32_t n;                // forks, or sequences to free
    const int32_t* seqs;
    const int32_t* keep;
    int32_t* n_used;
    // workspace
    int32_t* head;            // [0]: number of moves
    PageMove* moves;
    int32_t* pages;           // fork: a new page per fork, -1 none, -2 skipped; compact: new index per page, -1 free
    int32_t* found;           // fork: free pages in ascending order
    int32_t* claim;           // fork: lowest record that names the row as its child
};

size_t pages_workspace_bytes(const PagesArgs& a, int n_forks);   // n_forks 0: of a compaction
void pages_set_workspace(PagesArgs& a, int n_forks, void* ws);
hipError_t launch_pages_free(const PagesArgs& a, hipStream_t stream);
hipError_t launch_pages_fork(const PagesArgs& a, hipStream_t stream);
hipError_t launch_pages_compact(const PagesArgs& a, hipStream_t stream);

// ---- suffix attention --------------------------------------------------------

// Addresses and strides of the block scales of a cache held in 8 bits: one byte e
// per block of slots, KV head, layer and tensor, for 2^(e - 127).
struct BlockScales {
    const uint8_t* k;
    const uint8_t* v;
    int64_t k_stride[4];   // {layer, head, page, block in page}
    int64_t v_stride[4];
    int32_t block_shift;   // log2 of the slots that share a scale
};

struct AttnArgs {
    const void* q;
    const void* k;
    const void* v;
    void* out;
    const int32_t* q_pos;
    const int32_t* kv_len;
    const int32_t* cu_q;      // may be null (one sequence)
    const int64_t* kv_base;   // may be null
    float* lse_out;           // may be null
    float* ws_o;              // split partial outputs (fp32) or null
    float* ws_lse;            // split partial log-sum-exp (fp32) or null
    int32_t dtype;            // 0 bf16, 1 fp32, 2 bf16 queries and outputs over a paged cache of E4M3 codes
    int32_t variant;          // 0 GQA, 1 MLA
    int32_t n_layers;
    int32_t n_seqs;
    int32_t n_heads;
    int32_t n_kv_heads;
    int32_t head_dim;
    int32_t head_dim_v;
    int32_t total_q;
    int32_t max_q;
    int32_t max_kv_len;
    int32_t n_splits;
    int32_t auto_splits;      // n_splits is the library's own choice (the few-row kernels are eligible)
    int32_t partials;         // every row goes to the workspace, for a pass that joins it with more keys
    int32_t window;           // 0: full causal; W > 0: slots j > q_pos - W only
    int64_t cache_slots;
    float scale;
    int64_t q_stride[3];
    int64_t k_stride[3];
    int64_t v_stride[3];
    int64_t o_stride[3];
    // paged cache: sequence s's slot p is in page block_table[s * max_pages +
    // (p >> page_shift)], in-page slot p & (page_size - 1)
    const int32_t* block_table;  // null: contiguous cache
    const int32_t* v_block_table;  // V through its own table, or null (block_table)
    int32_t page_shift;
    int32_t max_pages;
    int64_t n_pages;
    int64_t k_page_stride;       // elements
    int64_t v_page_stride;
};

// Split plan shared by the workspace query and the launcher.
int attention_splits(const AttnArgs& a);
size_t attention_workspace_bytes(const AttnArgs& a, int n_splits);
hipError_t launch_attention(const AttnArgs& a, const BlockScales* scales, hipStream_t stream);   // scales: dtype 2

// ---- trees of drafted tokens ----------------------------------------------------

// The drafted rows of a tree-attention call, which lie beside the cache, and which of
// them each row sees.
struct DraftArgs {
    const void* k;
    const void* v;
    int64_t k_stride[3];      // {layer, head, row}, elements
    int64_t v_stride[3];
    const uint32_t* mask;     // [total_q][mask_words], or null: a row sees the rows of its sequence up to itself
    int32_t mask_words;
};

// Attention over the cache (its partials, if it has slots at all, into a.ws_o and
// a.ws_lse: a.partials is set) joined with the drafted rows.
hipError_t launch_tree_attention(const AttnArgs& a, const BlockScales* scales, const DraftArgs& d, hipStream_t stream);
hipError_t launch_tree_join(const AttnArgs& a, const DraftArgs& d, hipStream_t stream);   // its second step

struct TreeMaskArgs {
    const int32_t* parent;
    const int32_t* cu_q;      // may be null (one sequence)
    const int32_t* kv_len;
    int32_t n_seqs, total_q, max_q, mask_words;
    uint32_t* mask;
    int32_t* q_pos;           // may be null
    int32_t* err_flag;        // may be null
};
constexpr int kTreeMaxRows = 1024;   // rows of one sequence whose tree is walked
hipError_t launch_tree_masks(const TreeMaskArgs& a, hipStream_t stream);

struct TreeVerifyArgs {
    const void* target;       // [total_q][vocab], row strides in elements
    const void* draft;        // or null
    int64_t target_stride, draft_stride;
    const int32_t* tokens;
    const int32_t* parent;
    const int32_t* cu_q;
    const float* u_accept;
    const float* u_sample;
    int32_t dtype;            // 0 bf16, 1 fp32
    int32_t n_seqs, total_q, max_q, vocab, max_path;
    int32_t* path;
    int32_t* n_accepted;
    int32_t* next_token;
    int32_t* err_flag;
    void* workspace;
};
size_t tree_verify_workspace_bytes(int n_seqs, int vocab);
hipError_t launch_tree_verify(const TreeVerifyArgs& a, hipStream_t stream);

struct TreeCommitArgs {
    const char* src[2];       // keys, values (or null)
    char* dst[2];
    int64_t src_stride[2][3]; // bytes, {layer, head, row}
    int64_t dst_stride[2][3];
    int32_t row_bytes[2];     // 0 without values
    int32_t n_layers, n_kv_heads, n_rows;
    int64_t capacity;         // slots of the tensor, or logical slots of a paged sequence
    const int32_t* path;
    const int32_t* n_accepted;
    const int32_t* kv_len;
    const int64_t* kv_base;   // may be null
    int32_t n_seqs, max_path;
    const int32_t* table[2];  // null: contiguous
    int32_t page_shift, max_pages;
    int64_t n_pages;
    int64_t page_stride[2];   // bytes
    int32_t* err_flag;
};
hipError_t launch_tree_commit(const TreeCommitArgs& a, hipStream_t stream);

}  // namespace pkv
