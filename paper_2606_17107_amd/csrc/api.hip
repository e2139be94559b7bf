// C ABI of libpkv: argument validation, aliasing checks and dispatch to the
// kernel launchers.  The contract of every entry point is documented in
// include/pkv.h.  Nothing here allocates device memory or synchronises.
#include <math.h>
#include <stdarg.h>
#include <stdio.h>
#include <string.h>

#include <mutex>

#include "pkv.h"
#include "pkv_internal.h"

#define PKV_EXPORT extern "C" __attribute__((visibility("default")))

// Split-KV scratch of pkv_suffix_attention_noalloc: a file-scope device array,
// so that entry point never allocates.  Each GPU the library runs on holds its
// own copy (PKV_NOALLOC_SCRATCH_BYTES) until the process ends.  In host code
// `scratch` names a host-side stand-in, not device memory: kernels only ever
// get the per-device address that hipGetSymbolAddress returns for it.
static __device__ __align__(256) unsigned char scratch[PKV_NOALLOC_SCRATCH_BYTES];

namespace {

thread_local char g_err[512] = "";

pkv_status fail(pkv_status st, const char* fmt, ...) {
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(g_err, sizeof g_err, fmt, ap);
    va_end(ap);
    return st;
}

pkv_status ok() {
    g_err[0] = '\0';
    return PKV_OK;
}

bool aligned16(const void* p) { return ((uintptr_t)p & 15u) == 0; }

// Byte range [lo, hi) touched by a tensor with non-negative strides.
struct Range {
    uintptr_t lo = 0, hi = 0;
};

Range extent(const void* p, const int64_t* stride, const int64_t* count, int ndim, int64_t row_elems,
             int elem_bytes) {
    Range r;
    if (!p) return r;
    int64_t last = 0;
    for (int i = 0; i < ndim; ++i) last += (count[i] - 1) * stride[i];
    r.lo = (uintptr_t)p;
    r.hi = r.lo + (uintptr_t)((last + row_elems) * elem_bytes);
    return r;
}

bool overlap(const Range& a, const Range& b) {
    if (a.lo == a.hi || b.lo == b.hi) return false;
    return a.lo < b.hi && b.lo < a.hi;
}

pkv_status device_status(hipError_t e, const char* what) {
    if (e == hipSuccess) return ok();
    return fail(PKV_ERR_DEVICE, "%s: %s", what, hipGetErrorString(e));
}

// Validation of a paged-cache descriptor serving `logical_slots` slots per
// sequence with elements of `eb` bytes; sets *shift to log2(page_size).
pkv_status check_paging(const pkv_paged_cache* pg, int64_t logical_slots, int eb, int* shift) {
    if (!pg) return fail(PKV_ERR_NULL, "paging is NULL");
    if (!pg->block_table) return fail(PKV_ERR_NULL, "paging.block_table is NULL");
    const int32_t b = pg->page_size;
    if (b < 32 || b > (1 << 20) || (b & (b - 1)))
        return fail(PKV_ERR_SHAPE, "page_size %d must be a power of two in [32, 2^20]", b);
    if (pg->max_pages <= 0 || pg->n_pages <= 0 || pg->n_pages > 0x7fffffff)
        return fail(PKV_ERR_SHAPE, "max_pages (%d) and n_pages (%lld) must be positive (n_pages < 2^31)",
                    pg->max_pages, (long long)pg->n_pages);
    if (pg->page_stride_k < 0 || pg->page_stride_v < 0)
        return fail(PKV_ERR_SHAPE, "page strides must be non-negative");
    if ((pg->page_stride_k * eb) % 16 || (pg->page_stride_v * eb) % 16)
        return fail(PKV_ERR_ALIGN, "page strides must be multiples of 16 bytes");
    if (logical_slots > (int64_t)pg->max_pages * b)
        return fail(PKV_ERR_SHAPE, "%lld logical slots exceed max_pages * page_size = %lld",
                    (long long)logical_slots, (long long)pg->max_pages * b);
    int sh = 0;
    while ((1 << sh) < b) ++sh;
    *shift = sh;
    return PKV_OK;
}

// Byte range of a paged pool: {layer, head, page, in-page slot} with strides
// {stride[0], stride[1], page_stride, stride[2]}.
Range paged_extent(const void* p, const int64_t* stride, int64_t page_stride, int64_t n_layers, int64_t n_heads,
                   const pkv_paged_cache* pg, int64_t row_elems, int eb) {
    const int64_t st[4] = {stride[0], stride[1], page_stride, stride[2]};
    const int64_t cnt[4] = {n_layers, n_heads, pg->n_pages, pg->page_size};
    return extent(p, st, cnt, 4, row_elems, eb);
}

// Validation of the block scales of a cache held in 8 bits (paging already checked).
pkv_status check_scales(const pkv_block_scales* s, const pkv_paged_cache* pg, bool has_v) {
    if (!s) return fail(PKV_ERR_NULL, "scales is NULL");
    if (!s->k_scale || (has_v && !s->v_scale)) return fail(PKV_ERR_NULL, "k_scale and v_scale are required");
    if (!has_v && s->v_scale) return fail(PKV_ERR_SHAPE, "v_scale is given without a V tensor");
    if (s->reserved != 0) return fail(PKV_ERR_SHAPE, "scales.reserved must be 0");
    const int32_t b = s->block_tokens;
    if ((b != 32 && b != 64 && b != 128) || b > pg->page_size)
        return fail(PKV_ERR_SHAPE, "block_tokens %d must be 32, 64 or 128 and at most page_size (%d)", b, pg->page_size);
    for (int i = 0; i < 4; ++i)
        if (s->k_stride[i] < 0 || (has_v && s->v_stride[i] < 0))
            return fail(PKV_ERR_SHAPE, "scale strides must be non-negative");
    return PKV_OK;
}

Range scale_extent(const uint8_t* p, const int64_t* stride, int64_t n_layers, int64_t n_heads, const pkv_block_scales* s,
                   const pkv_paged_cache* pg) {
    const int64_t cnt[4] = {n_layers, n_heads, pg->n_pages, pg->page_size / s->block_tokens};
    return extent(p, stride, cnt, 4, 1, 1);
}

// Shared validation of reposition+splice arguments.  Fills `a` on success.
pkv_status check_splice(const void* src_k, const void* src_v, void* dst_k, void* dst_v,
                        float rope_theta, int32_t rope_dim, const pkv_layout* L, bool allow_inplace,
                        pkv::SpliceArgs& a, const pkv_paged_cache* pg = nullptr) {
    if (!L) return fail(PKV_ERR_NULL, "layout is NULL");
    if (!src_k || !dst_k) return fail(PKV_ERR_NULL, "src_k and dst_k are required");
    if (L->dtype != PKV_BF16 && L->dtype != PKV_F32)
        return fail(PKV_ERR_UNSUPPORTED, "dtype %d (expected PKV_BF16 or PKV_F32)", L->dtype);
    if (L->rope_style != PKV_ROPE_HALF && L->rope_style != PKV_ROPE_INTERLEAVED)
        return fail(PKV_ERR_UNSUPPORTED, "rope_style %d", L->rope_style);
    if (L->v_dim > 0 && (!src_v || !dst_v))
        return fail(PKV_ERR_NULL, "v_dim = %d but src_v or dst_v is NULL", L->v_dim);
    if (L->v_dim == 0 && (src_v || dst_v))
        return fail(PKV_ERR_SHAPE, "v_dim = 0 (no V tensors) but src_v or dst_v is given");
    if (L->reserved != 0) return fail(PKV_ERR_SHAPE, "layout.reserved must be 0");
    if (L->n_layers <= 0 || L->n_kv_heads <= 0 || L->head_dim <= 0 || L->v_dim < 0 ||
        L->n_tokens < 0 || L->dst_capacity < 0)
        return fail(PKV_ERR_SHAPE,
                    "sizes must be positive (n_layers %d, n_kv_heads %d, head_dim %d) and "
                    "non-negative (v_dim %d, n_tokens %d, dst_capacity %d)",
                    L->n_layers, L->n_kv_heads, L->head_dim, L->v_dim, L->n_tokens, L->dst_capacity);
    if (rope_dim <= 0 || (rope_dim & 1))
        return fail(PKV_ERR_SHAPE, "rope_dim %d must be positive and even", rope_dim);
    if (rope_dim > 256)
        return fail(PKV_ERR_UNSUPPORTED, "rope_dim %d: rotary slices of at most 256 channels are supported",
                    rope_dim);
    if (L->rope_offset < 0 || (int64_t)L->rope_offset + rope_dim > L->head_dim)
        return fail(PKV_ERR_SHAPE, "rotary slice [%d, %d) lies outside the %d-channel row",
                    L->rope_offset, L->rope_offset + rope_dim, L->head_dim);
    if (!(rope_theta > 0.0f) || !isfinite(rope_theta))
        return fail(PKV_ERR_SHAPE, "rope_theta must be finite and positive");
    for (int i = 0; i < 3; ++i) {
        if (L->src_k_stride[i] < 0 || L->dst_k_stride[i] < 0 || L->src_v_stride[i] < 0 ||
            L->dst_v_stride[i] < 0)
            return fail(PKV_ERR_SHAPE, "strides must be non-negative");
    }
    const int eb = L->dtype == PKV_BF16 ? 2 : 4;
    const int ce = 16 / eb;
    if (L->head_dim % (2 * ce) || L->v_dim % (2 * ce) || L->rope_offset % ce || rope_dim % (2 * ce))
        return fail(PKV_ERR_UNSUPPORTED,
                    "row geometry: head_dim (%d) and v_dim (%d) must be multiples of %d, rope_offset "
                    "(%d) of %d and rope_dim (%d) of %d for this dtype",
                    L->head_dim, L->v_dim, 2 * ce, L->rope_offset, ce, rope_dim, 2 * ce);
    if ((L->head_dim + L->v_dim) / (2 * ce) > 256)
        return fail(PKV_ERR_UNSUPPORTED, "rows wider than %d bytes (K+V) are not supported", 256 * 32);
    if (!aligned16(src_k) || !aligned16(dst_k) || !aligned16(src_v) || !aligned16(dst_v))
        return fail(PKV_ERR_ALIGN, "tensor pointers must be 16-byte aligned");
    for (int i = 0; i < 3; ++i) {
        if ((L->src_k_stride[i] * eb) % 16 || (L->dst_k_stride[i] * eb) % 16 ||
            (L->src_v_stride[i] * eb) % 16 || (L->dst_v_stride[i] * eb) % 16)
            return fail(PKV_ERR_ALIGN, "strides must be multiples of 16 bytes");
    }
    // Aliasing: destination tensors must not overlap sources (except an exact in-place
    // tensor) nor each other.
    const int64_t src_cnt[3] = {L->n_layers, L->n_kv_heads, L->n_tokens > 0 ? L->n_tokens : 1};
    const int64_t dst_cnt[3] = {L->n_layers, L->n_kv_heads, L->dst_capacity > 0 ? L->dst_capacity : 1};
    Range sk = extent(src_k, L->src_k_stride, src_cnt, 3, L->head_dim, eb);
    Range sv = extent(src_v, L->src_v_stride, src_cnt, 3, L->v_dim, eb);
    Range dk = extent(dst_k, L->dst_k_stride, dst_cnt, 3, L->head_dim, eb);
    Range dv = extent(dst_v, L->dst_v_stride, dst_cnt, 3, L->v_dim, eb);
    int page_shift = 0;
    if (pg) {
        pkv_status st = check_paging(pg, L->dst_capacity, eb, &page_shift);
        if (st != PKV_OK) return st;
        dk = paged_extent(dst_k, L->dst_k_stride, pg->page_stride_k, L->n_layers, L->n_kv_heads, pg, L->head_dim, eb);
        dv = paged_extent(dst_v, L->dst_v_stride, pg->page_stride_v, L->n_layers, L->n_kv_heads, pg, L->v_dim, eb);
        allow_inplace = false;
    }
    const bool k_inplace = allow_inplace && src_k == dst_k &&
                           memcmp(L->src_k_stride, L->dst_k_stride, sizeof L->src_k_stride) == 0;
    const bool v_inplace = allow_inplace && src_v && src_v == dst_v &&
                           memcmp(L->src_v_stride, L->dst_v_stride, sizeof L->src_v_stride) == 0;
    if ((!k_inplace && overlap(sk, dk)) || (!v_inplace && overlap(sv, dv)) || overlap(sk, dv) ||
        overlap(sv, dk) || overlap(dk, dv))
        return fail(PKV_ERR_ALIAS, "source and destination tensors overlap (only an exact in-place "
                                   "tensor is allowed)");

    memset(&a, 0, sizeof a);
    a.src_k = (const char*)src_k;
    a.src_v = (const char*)src_v;
    a.dst_k = (char*)dst_k;
    a.dst_v = (char*)dst_v;
    a.elem_bytes = eb;
    a.rope_style = L->rope_style;
    a.n_layers = L->n_layers;
    a.n_kv_heads = L->n_kv_heads;
    a.head_dim = L->head_dim;
    a.v_dim = L->v_dim;
    a.rope_offset = L->rope_offset;
    a.rope_dim = rope_dim;
    a.n_tokens = L->n_tokens;
    a.dst_capacity = L->dst_capacity;
    a.theta = (double)rope_theta;
    for (int i = 0; i < 3; ++i) {
        a.src_k_stride[i] = L->src_k_stride[i];
        a.src_v_stride[i] = L->src_v_stride[i];
        a.dst_k_stride[i] = L->dst_k_stride[i];
        a.dst_v_stride[i] = L->dst_v_stride[i];
    }
    a.err_flag = L->err_flag;
    if (pg) {
        a.dst_pages = pg->block_table;
        a.dst_v_pages = pg->v_block_table;
        a.page_shift = page_shift;
        a.max_pages = pg->max_pages;
        a.n_pages = pg->n_pages;
        a.dst_k_page_stride = pg->page_stride_k;
        a.dst_v_page_stride = pg->page_stride_v;
    }
    return PKV_OK;
}

// Validation of attention arguments; fills `a` (without workspace pointers).
pkv_status check_attention(const void* q, const void* k, const void* v, void* out,
                           const int32_t* q_pos, const int32_t* kv_len, int32_t H, int32_t Hkv,
                           int32_t D, float scale, const pkv_attn_desc* d, bool check_alias,
                           pkv::AttnArgs& a, const pkv_paged_cache* pg = nullptr, bool q8 = false) {
    if (!d) return fail(PKV_ERR_NULL, "desc is NULL");
    if (!q || !k || !v || !out || !q_pos || !kv_len)
        return fail(PKV_ERR_NULL, "q, k_cache, v_cache, out, q_pos and kv_len are required");
    if (d->dtype != PKV_BF16 && d->dtype != PKV_F32) return fail(PKV_ERR_UNSUPPORTED, "dtype %d", d->dtype);
    if (d->variant != PKV_ATTN_GQA && d->variant != PKV_ATTN_MLA)
        return fail(PKV_ERR_UNSUPPORTED, "variant %d", d->variant);
    if (q8 && (d->dtype != PKV_BF16 || d->variant != PKV_ATTN_GQA))
        return fail(PKV_ERR_UNSUPPORTED, "attention over a cache held in 8 bits takes bf16 queries and GQA heads");
    if (d->window < 0) return fail(PKV_ERR_SHAPE, "desc.window (%d) must be >= 0", d->window);
    if (H <= 0 || Hkv <= 0 || D <= 0 || H % Hkv)
        return fail(PKV_ERR_SHAPE, "n_q_heads (%d) must be a positive multiple of n_kv_heads (%d)", H, Hkv);
    if (d->n_layers <= 0 || d->n_seqs <= 0 || d->total_q < 0 || d->max_q < 0 || d->max_kv_len < 0 ||
        d->n_splits < 0 || d->cache_slots < 0 || d->head_dim_v <= 0)
        return fail(PKV_ERR_SHAPE, "invalid sizes in desc");
    if (d->max_kv_len > (1 << 30))   // key indices and tile arithmetic stay inside int32
        return fail(PKV_ERR_SHAPE, "max_kv_len (%d) above 2^30", d->max_kv_len);
    if (d->n_seqs > 1 && !d->cu_q) return fail(PKV_ERR_NULL, "cu_q is required when n_seqs > 1");
    if (d->n_seqs == 1 && !d->cu_q && d->max_q < d->total_q)
        return fail(PKV_ERR_SHAPE, "max_q (%d) < total_q (%d)", d->max_q, d->total_q);
    if (!isfinite(scale)) return fail(PKV_ERR_SHAPE, "scale must be finite");
    if (d->variant == PKV_ATTN_GQA) {
        if (D != 64 && D != 128) return fail(PKV_ERR_UNSUPPORTED, "GQA head_dim %d (supported: 64, 128)", D);
        if (d->head_dim_v != D) return fail(PKV_ERR_SHAPE, "GQA needs head_dim_v == head_dim");
    } else {
        if (d->dtype != PKV_BF16) return fail(PKV_ERR_UNSUPPORTED, "MLA attention is bf16 only");
        if (Hkv != 1 || D != 576 || d->head_dim_v != 512)
            return fail(PKV_ERR_SHAPE, "MLA needs n_kv_heads 1, head_dim 576, head_dim_v 512");
        if (v != k || memcmp(d->v_stride, d->k_stride, sizeof d->k_stride) != 0)
            return fail(PKV_ERR_SHAPE, "MLA reads values from the latent channels of k_cache: v_cache must be "
                                       "k_cache with the same strides");
    }
    const int eb = d->dtype == PKV_BF16 ? 2 : 4;
    const int cb = q8 ? 1 : eb;   // bytes per element of the cache
    if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(out))
        return fail(PKV_ERR_ALIGN, "q, k_cache, v_cache and out must be 16-byte aligned");
    for (int i = 0; i < 3; ++i) {
        if (d->q_stride[i] < 0 || d->k_stride[i] < 0 || d->v_stride[i] < 0 || d->o_stride[i] < 0)
            return fail(PKV_ERR_SHAPE, "strides must be non-negative");
        if ((d->q_stride[i] * eb) % 16 || (d->k_stride[i] * cb) % 16 || (d->v_stride[i] * cb) % 16 ||
            (d->o_stride[i] * eb) % 16)
            return fail(PKV_ERR_ALIGN, "strides must be multiples of 16 bytes");
    }
    // The kernels address the keys of one tile (up to 32 slots) by 32-bit byte
    // offsets from its first key.
    constexpr int64_t kMaxSlotBytes = (int64_t)1 << 26;
    if (d->k_stride[2] > kMaxSlotBytes / cb || d->v_stride[2] > kMaxSlotBytes / cb)
        return fail(PKV_ERR_SHAPE, "slot strides k_stride[2] / v_stride[2] (%lld / %lld elements) exceed 64 MiB",
                    (long long)d->k_stride[2], (long long)d->v_stride[2]);
    int page_shift = 0;
    if (pg) {
        if (d->dtype != PKV_BF16) return fail(PKV_ERR_UNSUPPORTED, "paged attention is bf16 only");
        if (d->kv_base) return fail(PKV_ERR_SHAPE, "desc.kv_base must be NULL for a paged cache");
        pkv_status st = check_paging(pg, d->cache_slots, cb, &page_shift);
        if (st != PKV_OK) return st;
        if (d->variant == PKV_ATTN_MLA && (pg->page_stride_v != pg->page_stride_k || pg->v_block_table))
            return fail(PKV_ERR_SHAPE, "MLA reads values from the latent channels: page_stride_v must equal "
                                       "page_stride_k and there is no separate v_block_table");
    }
    // out must not overlap any input
    if (check_alias && d->total_q > 0) {
        const int64_t oc[3] = {d->n_layers, d->total_q, H};
        const int64_t qc[3] = {d->n_layers, d->total_q, H};
        const int64_t slots = d->cache_slots > 0 ? d->cache_slots : 1;
        const int64_t kc[3] = {d->n_layers, Hkv, slots};
        Range ro = extent(out, d->o_stride, oc, 3, d->head_dim_v, eb);
        Range rq = extent(q, d->q_stride, qc, 3, D, eb);
        Range rk = extent(k, d->k_stride, kc, 3, D, eb);
        Range rv = extent(v, d->v_stride, kc, 3, d->head_dim_v, eb);
        if (pg) {
            rk = paged_extent(k, d->k_stride, pg->page_stride_k, d->n_layers, Hkv, pg, D, cb);
            rv = paged_extent(v, d->v_stride, pg->page_stride_v, d->n_layers, Hkv, pg, d->head_dim_v, cb);
        }
        if (overlap(ro, rq) || overlap(ro, rk) || overlap(ro, rv))
            return fail(PKV_ERR_ALIAS, "out overlaps an input tensor");
    }
    memset(&a, 0, sizeof a);
    a.q = q;
    a.k = k;
    a.v = v;
    a.out = out;
    a.q_pos = q_pos;
    a.kv_len = kv_len;
    a.cu_q = d->cu_q;
    a.kv_base = d->kv_base;
    a.lse_out = d->lse_out;
    a.dtype = q8 ? 2 : d->dtype;
    a.variant = d->variant;
    a.n_layers = d->n_layers;
    a.n_seqs = d->n_seqs;
    a.n_heads = H;
    a.n_kv_heads = Hkv;
    a.head_dim = D;
    a.head_dim_v = d->head_dim_v;
    a.total_q = d->total_q;
    a.max_q = d->cu_q ? d->max_q : d->total_q;
    a.max_kv_len = d->max_kv_len;
    a.n_splits = d->n_splits;
    a.auto_splits = d->n_splits == 0;
    a.window = d->window;
    a.cache_slots = d->cache_slots;
    a.scale = scale;
    for (int i = 0; i < 3; ++i) {
        a.q_stride[i] = d->q_stride[i];
        a.k_stride[i] = d->k_stride[i];
        a.v_stride[i] = d->v_stride[i];
        a.o_stride[i] = d->o_stride[i];
    }
    if (pg) {
        a.block_table = pg->block_table;
        a.v_block_table = pg->v_block_table;
        a.page_shift = page_shift;
        a.max_pages = pg->max_pages;
        a.n_pages = pg->n_pages;
        a.k_page_stride = pg->page_stride_k;
        a.v_page_stride = pg->page_stride_v;
    }
    return PKV_OK;
}

}  // namespace

PKV_EXPORT pkv_status pkv_reposition_splice(const void* src_k, const void* src_v, void* dst_k,
                                            void* dst_v, const int32_t* src_pos, const int32_t* dst_pos,
                                            float rope_theta, int32_t rope_dim,
                                            const pkv_layout* layout, void* stream) {
    pkv::SpliceArgs a;
    pkv_status st = check_splice(src_k, src_v, dst_k, dst_v, rope_theta, rope_dim, layout, true, a);
    if (st != PKV_OK) return st;
    if (!src_pos || !dst_pos) return fail(PKV_ERR_NULL, "src_pos and dst_pos are required");
    a.src_pos = src_pos;
    a.dst_pos = dst_pos;
    if (a.n_tokens == 0) return ok();
    return device_status(pkv::launch_splice(a, (hipStream_t)stream), "reposition_splice launch");
}

PKV_EXPORT pkv_status pkv_reposition_splice_freqs(const void* src_k, const void* src_v, void* dst_k,
                                                  void* dst_v, const int32_t* src_pos, const int32_t* dst_pos,
                                                  const int32_t* dst_slot, const double* omega, int32_t rope_dim,
                                                  const pkv_layout* layout, void* stream) {
    pkv::SpliceArgs a;
    pkv_status st = check_splice(src_k, src_v, dst_k, dst_v, 1.0f, rope_dim, layout, true, a);
    if (st != PKV_OK) return st;
    if (!src_pos || !dst_pos) return fail(PKV_ERR_NULL, "src_pos and dst_pos are required");
    if (!omega) return fail(PKV_ERR_NULL, "omega is required");
    for (int i = 0; i < rope_dim / 2; ++i)
        if (!isfinite(omega[i])) return fail(PKV_ERR_SHAPE, "omega[%d] is not finite", i);
    a.src_pos = src_pos;
    a.dst_pos = dst_pos;
    a.dst_slot = dst_slot;
    a.omega = omega;
    if (a.n_tokens == 0) return ok();
    return device_status(pkv::launch_splice(a, (hipStream_t)stream), "reposition_splice_freqs launch");
}

PKV_EXPORT pkv_status pkv_reposition_splice_paged(const void* src_k, const void* src_v, void* dst_k,
                                                  void* dst_v, const int32_t* src_pos, const int32_t* dst_pos,
                                                  float rope_theta, int32_t rope_dim, const pkv_layout* layout,
                                                  const pkv_paged_cache* paging, void* stream) {
    pkv::SpliceArgs a;
    if (!paging) return fail(PKV_ERR_NULL, "paging is NULL");
    pkv_status st = check_splice(src_k, src_v, dst_k, dst_v, rope_theta, rope_dim, layout, false, a, paging);
    if (st != PKV_OK) return st;
    if (!src_pos || !dst_pos) return fail(PKV_ERR_NULL, "src_pos and dst_pos are required");
    a.src_pos = src_pos;
    a.dst_pos = dst_pos;
    if (a.n_tokens == 0) return ok();
    return device_status(pkv::launch_splice(a, (hipStream_t)stream), "reposition_splice_paged launch");
}

PKV_EXPORT pkv_status pkv_reposition_splice_batched(const void* src_k, const void* src_v, void* dst_k,
                                                    void* dst_v, const pkv_segment* segs, int32_t n_segs,
                                                    int32_t max_seg_tokens, float rope_theta,
                                                    int32_t rope_dim, const pkv_layout* layout,
                                                    void* stream) {
    static_assert(sizeof(pkv_segment) == sizeof(pkv::SpliceSegment), "segment layout");
    pkv::SpliceArgs a;
    pkv_status st = check_splice(src_k, src_v, dst_k, dst_v, rope_theta, rope_dim, layout, false, a);
    if (st != PKV_OK) return st;
    if (n_segs < 0 || max_seg_tokens < 0)
        return fail(PKV_ERR_SHAPE, "n_segs (%d) and max_seg_tokens (%d) must be non-negative", n_segs,
                    max_seg_tokens);
    if (n_segs > 65535) return fail(PKV_ERR_UNSUPPORTED, "at most 65535 segments per call");
    if (n_segs > 0 && !segs) return fail(PKV_ERR_NULL, "segs is NULL");
    if (!aligned16(segs)) return fail(PKV_ERR_ALIGN, "segs must be 16-byte aligned");
    if (n_segs == 0 || max_seg_tokens == 0) return ok();
    a.segs = (const pkv::SpliceSegment*)segs;
    a.n_segs = n_segs;
    a.max_seg_tokens = max_seg_tokens;
    return device_status(pkv::launch_splice(a, (hipStream_t)stream), "reposition_splice_batched launch");
}

namespace {

// Splits of a call; 0 for a tree without any cache, which has no first step.
int plan_splits(const pkv::AttnArgs& a) { return a.partials && a.max_kv_len == 0 ? 0 : pkv::attention_splits(a); }

size_t workspace_size(const pkv_attn_desc* desc, int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim, bool q8,
                      bool tree = false) {
    if (!desc) return 0;
    // Geometry checks only; pointers are not needed to size the workspace.
    static const char dummy[16] __attribute__((aligned(16))) = {0};
    static const int32_t idummy[4] __attribute__((aligned(16))) = {0};
    pkv::AttnArgs a;
    char saved[sizeof g_err];
    memcpy(saved, g_err, sizeof g_err);
    pkv_status st = check_attention(dummy, dummy, dummy, (void*)dummy, idummy, idummy, n_q_heads,
                                    n_kv_heads, head_dim, 1.0f, desc, false, a, nullptr, q8);
    memcpy(g_err, saved, sizeof g_err);
    if (st != PKV_OK) return 0;
    a.partials = tree;
    return pkv::attention_workspace_bytes(a, plan_splits(a));
}

}  // namespace

PKV_EXPORT size_t pkv_attention_workspace_size(const pkv_attn_desc* desc, int32_t n_q_heads,
                                               int32_t n_kv_heads, int32_t head_dim) {
    return workspace_size(desc, n_q_heads, n_kv_heads, head_dim, false);
}

PKV_EXPORT size_t pkv_attention_quant_workspace_size(const pkv_attn_desc* desc, int32_t n_q_heads, int32_t n_kv_heads,
                                                  int32_t head_dim) {
    return workspace_size(desc, n_q_heads, n_kv_heads, head_dim, true);
}

namespace {

constexpr int kMaxDevices = 64;
std::mutex g_scratch_mu;
void* g_scratch_dev[kMaxDevices] = {};   // device address of `scratch`, per device

// Device address of `scratch` on the current device, looked up once per device
// (with that device current: each GPU holds the array at its own address).
pkv_status scratch_on_current_device(void** out) {
    int dev = -1;
    hipError_t e = hipGetDevice(&dev);
    if (e != hipSuccess) return fail(PKV_ERR_DEVICE, "hipGetDevice: %s", hipGetErrorString(e));
    if (dev < 0 || dev >= kMaxDevices)
        return fail(PKV_ERR_UNSUPPORTED, "device %d: the allocation-free entry point serves devices 0..%d", dev,
                    kMaxDevices - 1);
    std::lock_guard<std::mutex> lock(g_scratch_mu);
    if (!g_scratch_dev[dev]) {
        void* p = nullptr;
        e = hipGetSymbolAddress(&p, HIP_SYMBOL(scratch));
        if (e != hipSuccess || !p)
            return fail(PKV_ERR_DEVICE, "hipGetSymbolAddress(scratch) on device %d: %s", dev, hipGetErrorString(e));
        g_scratch_dev[dev] = p;
    }
    *out = g_scratch_dev[dev];
    return PKV_OK;
}

// Workspace layout shared by both attention entry points:
// [split][layer][row][head][d_v] partial outputs, then [split][layer][row][head] LSEs.
void set_workspace(pkv::AttnArgs& a, void* workspace) {
    const size_t rows = (size_t)a.n_splits * a.n_layers * a.total_q * a.n_heads;
    a.ws_o = (float*)workspace;
    a.ws_lse = a.ws_o + rows * a.head_dim_v;
}

// The drafted rows of a tree-attention call (its other arguments are checked already).
pkv_status check_draft(const pkv_draft* t, const void* out, const pkv::AttnArgs& a, const pkv_attn_desc* d,
                       pkv::DraftArgs& da) {
    if (!t->k || !t->v) return fail(PKV_ERR_NULL, "draft.k and draft.v are required");
    if (t->reserved != 0) return fail(PKV_ERR_SHAPE, "draft.reserved must be 0");
    if (!aligned16(t->k) || !aligned16(t->v)) return fail(PKV_ERR_ALIGN, "draft.k and draft.v must be 16-byte aligned");
    if ((uintptr_t)t->mask & 3u) return fail(PKV_ERR_ALIGN, "draft.mask must be 4-byte aligned");
    const int eb = a.dtype == PKV_F32 ? 4 : 2;
    for (int i = 0; i < 3; ++i) {
        if (t->k_stride[i] < 0 || t->v_stride[i] < 0) return fail(PKV_ERR_SHAPE, "strides must be non-negative");
        if ((t->k_stride[i] * eb) % 16 || (t->v_stride[i] * eb) % 16)
            return fail(PKV_ERR_ALIGN, "strides must be multiples of 16 bytes");
    }
    constexpr int64_t kMaxRowBytes = (int64_t)1 << 26;   // as slot strides: rows by 32-bit strides
    if (t->k_stride[2] > kMaxRowBytes / eb || t->v_stride[2] > kMaxRowBytes / eb)
        return fail(PKV_ERR_SHAPE, "row strides of drafted rows exceed 64 MiB");
    if (a.variant == PKV_ATTN_MLA && (t->v != t->k || memcmp(t->v_stride, t->k_stride, sizeof t->k_stride) != 0))
        return fail(PKV_ERR_SHAPE, "MLA reads values from the latent channels: draft.v must be draft.k with the same strides");
    if (t->mask && (t->mask_words <= 0 || t->mask_words < (a.max_q + 31) / 32))
        return fail(PKV_ERR_SHAPE, "draft.mask_words (%d) must hold max_q (%d) bits", t->mask_words, a.max_q);
    if (a.total_q > 0) {
        const int64_t oc[3] = {a.n_layers, a.total_q, a.n_heads}, kc[3] = {a.n_layers, a.n_kv_heads, a.total_q};
        const Range ro = extent(out, d->o_stride, oc, 3, a.head_dim_v, eb);
        Range rm;
        if (t->mask) {
            rm.lo = (uintptr_t)t->mask;
            rm.hi = rm.lo + (uintptr_t)a.total_q * t->mask_words * 4;
        }
        if (overlap(ro, extent(t->k, t->k_stride, kc, 3, a.head_dim, eb)) ||
            overlap(ro, extent(t->v, t->v_stride, kc, 3, a.head_dim_v, eb)) || overlap(ro, rm))
            return fail(PKV_ERR_ALIAS, "out overlaps the drafted rows or their mask");
    }
    da.k = t->k;
    da.v = t->v;
    for (int i = 0; i < 3; ++i) {
        da.k_stride[i] = t->k_stride[i];
        da.v_stride[i] = t->v_stride[i];
    }
    da.mask = t->mask;
    da.mask_words = t->mask_words;
    return PKV_OK;
}

pkv_status run_attention(const void* q, const void* k_cache, const void* v_cache, void* out, const int32_t* q_pos,
                         const int32_t* kv_len, int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim, float scale,
                         const pkv_attn_desc* desc, const pkv_paged_cache* paging, const pkv_block_scales* scales,
                         void* workspace, size_t workspace_bytes, void* stream, const pkv_draft* draft = nullptr) {
    pkv::AttnArgs a;
    pkv::BlockScales bs;
    pkv::DraftArgs da;
    pkv_status st = check_attention(q, k_cache, v_cache, out, q_pos, kv_len, n_q_heads, n_kv_heads,
                                    head_dim, scale, desc, true, a, paging, scales != nullptr);
    if (st != PKV_OK) return st;
    if (scales) {
        st = check_scales(scales, paging, true);
        if (st != PKV_OK) return st;
        const int64_t oc[3] = {desc->n_layers, desc->total_q, n_q_heads};
        const Range ro = extent(out, desc->o_stride, oc, 3, desc->head_dim_v, 2);
        if (desc->total_q > 0 &&
            (overlap(ro, scale_extent(scales->k_scale, scales->k_stride, desc->n_layers, n_kv_heads, scales, paging)) ||
             overlap(ro, scale_extent(scales->v_scale, scales->v_stride, desc->n_layers, n_kv_heads, scales, paging))))
            return fail(PKV_ERR_ALIAS, "out overlaps the scales");
        bs.k = scales->k_scale;
        bs.v = scales->v_scale;
        for (int i = 0; i < 4; ++i) {
            bs.k_stride[i] = scales->k_stride[i];
            bs.v_stride[i] = scales->v_stride[i];
        }
        bs.block_shift = scales->block_tokens == 32 ? 5 : scales->block_tokens == 64 ? 6 : 7;
    }
    if (draft) {
        st = check_draft(draft, out, a, desc, da);
        if (st != PKV_OK) return st;
        a.partials = 1;
    }
    const int splits = plan_splits(a);
    const size_t need = pkv::attention_workspace_bytes(a, splits);
    if (need > 0) {
        if (!workspace) return fail(PKV_ERR_NULL, "workspace of %zu bytes is required", need);
        if (workspace_bytes < need)
            return fail(PKV_ERR_SHAPE, "workspace_bytes %zu < required %zu", workspace_bytes, need);
        if (!aligned16(workspace)) return fail(PKV_ERR_ALIGN, "workspace must be 16-byte aligned");
    }
    a.n_splits = splits;
    if (need > 0) set_workspace(a, workspace);
    if (a.total_q == 0) return ok();
    if (draft)
        return device_status(pkv::launch_tree_attention(a, scales ? &bs : nullptr, da, (hipStream_t)stream),
                             "tree_attention launch");
    return device_status(pkv::launch_attention(a, scales ? &bs : nullptr, (hipStream_t)stream),
                         "suffix_attention launch");
}

}  // namespace

PKV_EXPORT pkv_status pkv_suffix_attention(const void* q, const void* k_cache, const void* v_cache,
                                           void* out, const int32_t* q_pos, const int32_t* kv_len,
                                           int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim,
                                           float scale, const pkv_attn_desc* desc, void* workspace,
                                           size_t workspace_bytes, void* stream) {
    return run_attention(q, k_cache, v_cache, out, q_pos, kv_len, n_q_heads, n_kv_heads, head_dim, scale, desc,
                         nullptr, nullptr, workspace, workspace_bytes, stream);
}

PKV_EXPORT pkv_status pkv_suffix_attention_paged(const void* q, const void* k_pages, const void* v_pages,
                                                 void* out, const int32_t* q_pos, const int32_t* kv_len,
                                                 int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim,
                                                 float scale, const pkv_attn_desc* desc,
                                                 const pkv_paged_cache* paging, void* workspace,
                                                 size_t workspace_bytes, void* stream) {
    if (!paging) return fail(PKV_ERR_NULL, "paging is NULL");
    return run_attention(q, k_pages, v_pages, out, q_pos, kv_len, n_q_heads, n_kv_heads, head_dim, scale, desc,
                         paging, nullptr, workspace, workspace_bytes, stream);
}

PKV_EXPORT pkv_status pkv_suffix_attention_quant(const void* q, const void* k_pages, const void* v_pages, void* out,
                                              const int32_t* q_pos, const int32_t* kv_len, int32_t n_q_heads,
                                              int32_t n_kv_heads, int32_t head_dim, float scale,
                                              const pkv_attn_desc* desc, const pkv_paged_cache* paging,
                                              const pkv_block_scales* scales, void* workspace,
                                              size_t workspace_bytes, void* stream) {
    if (!paging) return fail(PKV_ERR_NULL, "paging is NULL");
    if (!scales) return fail(PKV_ERR_NULL, "scales is NULL");
    return run_attention(q, k_pages, v_pages, out, q_pos, kv_len, n_q_heads, n_kv_heads, head_dim, scale, desc,
                         paging, scales, workspace, workspace_bytes, stream);
}

PKV_EXPORT pkv_status pkv_suffix_attention_noalloc(const void* q, const void* k_cache, const void* v_cache,
                                                   void* out, const int32_t* q_pos, const int32_t* kv_len,
                                                   int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim,
                                                   float scale, const pkv_attn_desc* desc, void* stream) {
    pkv::AttnArgs a;
    pkv_status st = check_attention(q, k_cache, v_cache, out, q_pos, kv_len, n_q_heads, n_kv_heads, head_dim,
                                    scale, desc, true, a);
    if (st != PKV_OK) return st;
    int splits = pkv::attention_splits(a);
    size_t need = pkv::attention_workspace_bytes(a, splits);
    if (need > PKV_NOALLOC_SCRATCH_BYTES) {
        if (desc->n_splits > 0)
            return fail(PKV_ERR_SHAPE,
                        "%d splits need %zu bytes of partials, more than the %zu-byte scratch of the "
                        "allocation-free entry point (use fewer splits, n_splits = 0, or pkv_suffix_attention "
                        "with a workspace)",
                        splits, need, (size_t)PKV_NOALLOC_SCRATCH_BYTES);
        while (splits > 1 && pkv::attention_workspace_bytes(a, splits) > PKV_NOALLOC_SCRATCH_BYTES) --splits;
        need = pkv::attention_workspace_bytes(a, splits);
        // (auto_splits stays: with fewer records the few-row kernels cut the keys into longer runs)
    }
    a.n_splits = splits;
    if (need > 0) {
        void* sp = nullptr;
        st = scratch_on_current_device(&sp);
        if (st != PKV_OK) return st;
        set_workspace(a, sp);
    }
    if (a.total_q == 0) return ok();
    return device_status(pkv::launch_attention(a, nullptr, (hipStream_t)stream), "suffix_attention_noalloc launch");
}

namespace {

// The quantising splice.  accepted: instead of segments, the rows that are accepted.
pkv_status splice_quant(const void* src_k, const void* src_v, void* k_pages, void* v_pages, const pkv_segment_quant* segs,
                        int32_t n_segs, int32_t max_seg_tokens, const int32_t* kv_len, int32_t n_seqs, const double* omega,
                        float rope_theta, int32_t rope_dim, const pkv_layout* layout, const pkv_paged_cache* paging,
                        const pkv_block_scales* scales, const pkv::TreeCommitArgs* accepted, void* stream) {
    static_assert(sizeof(pkv_segment_quant) == sizeof(pkv::StoreSegment), "segment layout");
    const pkv_layout* L = layout;
    if (!L) return fail(PKV_ERR_NULL, "layout is NULL");
    if (!src_k || !k_pages) return fail(PKV_ERR_NULL, "src_k and k_pages are required");
    if (!kv_len) return fail(PKV_ERR_NULL, "kv_len is NULL");
    if (L->dtype != PKV_BF16 && L->dtype != PKV_F32)
        return fail(PKV_ERR_UNSUPPORTED, "dtype %d (expected PKV_BF16 or PKV_F32)", L->dtype);
    if (L->rope_style != PKV_ROPE_HALF && L->rope_style != PKV_ROPE_INTERLEAVED)
        return fail(PKV_ERR_UNSUPPORTED, "rope_style %d", L->rope_style);
    const bool has_v = L->v_dim != 0;
    if (has_v && (!src_v || !v_pages)) return fail(PKV_ERR_NULL, "v_dim = %d but src_v or v_pages is NULL", L->v_dim);
    if (!has_v && (src_v || v_pages))
        return fail(PKV_ERR_SHAPE, "v_dim = 0 (no V tensors) but src_v or v_pages is given");
    if (L->reserved != 0) return fail(PKV_ERR_SHAPE, "layout.reserved must be 0");
    if (L->n_layers <= 0 || L->n_kv_heads <= 0 || L->n_tokens < 0 || L->dst_capacity < 0 || L->dst_capacity > (1 << 30) ||
        n_seqs <= 0 || n_segs < 0 || max_seg_tokens < 0)
        return fail(PKV_ERR_SHAPE,
                    "sizes must be positive (n_layers %d, n_kv_heads %d, n_seqs %d) and non-negative (n_tokens %d, "
                    "dst_capacity %d, at most 2^30, n_segs %d, max_seg_tokens %d)",
                    L->n_layers, L->n_kv_heads, n_seqs, L->n_tokens, L->dst_capacity, n_segs, max_seg_tokens);
    if (L->head_dim != 64 && L->head_dim != 128)
        return fail(PKV_ERR_UNSUPPORTED, "head_dim %d (supported: 64, 128)", L->head_dim);
    if (has_v && L->v_dim != L->head_dim)
        return fail(PKV_ERR_UNSUPPORTED, "v_dim %d must be head_dim (%d) or 0", L->v_dim, L->head_dim);
    if (rope_dim <= 0 || (rope_dim & 1)) return fail(PKV_ERR_SHAPE, "rope_dim %d must be positive and even", rope_dim);
    if (L->rope_offset < 0 || (int64_t)L->rope_offset + rope_dim > L->head_dim)
        return fail(PKV_ERR_SHAPE, "rotary slice [%d, %lld) lies outside the %d-channel row", L->rope_offset,
                    (long long)L->rope_offset + rope_dim, L->head_dim);
    if (L->rope_offset % 8 || rope_dim % 16)
        return fail(PKV_ERR_UNSUPPORTED, "rope_offset (%d) must be a multiple of 8 and rope_dim (%d) of 16",
                    L->rope_offset, rope_dim);
    if (omega) {
        for (int i = 0; i < rope_dim / 2; ++i)
            if (!isfinite(omega[i])) return fail(PKV_ERR_SHAPE, "omega[%d] is not finite", i);
    } else if (!(rope_theta > 0.0f) || !isfinite(rope_theta)) {
        return fail(PKV_ERR_SHAPE, "rope_theta must be finite and positive");
    }
    if (n_segs > 65535) return fail(PKV_ERR_UNSUPPORTED, "at most 65535 %s per call", accepted ? "sequences" : "segments");
    if (n_segs > 0 && !segs && !accepted) return fail(PKV_ERR_NULL, "segs is NULL");
    if ((uintptr_t)segs & 7u) return fail(PKV_ERR_ALIGN, "segs must be 8-byte aligned");
    const int eb = L->dtype == PKV_BF16 ? 2 : 4;
    for (int i = 0; i < 3; ++i) {
        if (L->src_k_stride[i] < 0 || L->dst_k_stride[i] < 0 || L->src_v_stride[i] < 0 || L->dst_v_stride[i] < 0)
            return fail(PKV_ERR_SHAPE, "strides must be non-negative");
        if ((L->src_k_stride[i] * eb) % 16 || L->dst_k_stride[i] % 16 || (L->src_v_stride[i] * eb) % 16 ||
            L->dst_v_stride[i] % 16)
            return fail(PKV_ERR_ALIGN, "strides must be multiples of 16 bytes");
    }
    // The kernel addresses the rows of one block (up to 128 slots) by 32-bit byte offsets.
    constexpr int64_t kMaxRowBytes = (int64_t)1 << 24;
    if (L->src_k_stride[2] > kMaxRowBytes / eb || L->src_v_stride[2] > kMaxRowBytes / eb ||
        L->dst_k_stride[2] > kMaxRowBytes || L->dst_v_stride[2] > kMaxRowBytes)
        return fail(PKV_ERR_SHAPE, "slot strides exceed 16 MiB");
    if (!aligned16(src_k) || !aligned16(src_v) || !aligned16(k_pages) || !aligned16(v_pages))
        return fail(PKV_ERR_ALIGN, "tensor pointers must be 16-byte aligned");
    pkv::StoreArgs a;
    memset(&a, 0, sizeof a);
    int shift = 0;
    pkv_status st = check_paging(paging, L->dst_capacity, 1, &shift);
    if (st != PKV_OK) return st;
    st = check_scales(scales, paging, has_v);
    if (st != PKV_OK) return st;
    const int64_t sc[3] = {L->n_layers, L->n_kv_heads, L->n_tokens > 0 ? L->n_tokens : 1};
    Range r[6] = {extent(src_k, L->src_k_stride, sc, 3, L->head_dim, eb),
                  extent(src_v, L->src_v_stride, sc, 3, L->v_dim, eb),
                  paged_extent(k_pages, L->dst_k_stride, paging->page_stride_k, L->n_layers, L->n_kv_heads, paging,
                               L->head_dim, 1),
                  paged_extent(v_pages, L->dst_v_stride, paging->page_stride_v, L->n_layers, L->n_kv_heads, paging,
                               L->v_dim, 1),
                  scale_extent(scales->k_scale, scales->k_stride, L->n_layers, L->n_kv_heads, scales, paging),
                  scale_extent(scales->v_scale, scales->v_stride, L->n_layers, L->n_kv_heads, scales, paging)};
    for (int i = 0; i < 6; ++i)   // (the two sources may be one tensor)
        for (int j = i < 2 ? 2 : i + 1; j < 6; ++j)
            if (overlap(r[i], r[j])) return fail(PKV_ERR_ALIAS, "sources, pools and scales must not overlap");
    // (accepted rows for a cache without slots are flagged by the kernel)
    if (n_segs == 0 || max_seg_tokens == 0 || (L->dst_capacity == 0 && !accepted)) return ok();
    a.src_k = (const char*)src_k;
    a.src_v = (const char*)src_v;
    a.dst_k = (uint8_t*)k_pages;
    a.dst_v = (uint8_t*)v_pages;
    a.segs = (const pkv::StoreSegment*)segs;
    a.n_segs = n_segs;
    a.max_seg_tokens = max_seg_tokens;
    a.kv_len = kv_len;
    a.n_seqs = n_seqs;
    a.elem_bytes = eb;
    a.rope_style = L->rope_style;
    a.n_layers = L->n_layers;
    a.n_kv_heads = L->n_kv_heads;
    a.head_dim = L->head_dim;
    a.rope_offset = L->rope_offset;
    a.rope_dim = rope_dim;
    a.n_src = L->n_tokens;
    a.dst_capacity = L->dst_capacity;
    a.theta = (double)rope_theta;
    a.omega = omega;
    for (int i = 0; i < 3; ++i) {
        a.src_k_stride[i] = L->src_k_stride[i];
        a.src_v_stride[i] = L->src_v_stride[i];
        a.dst_k_stride[i] = L->dst_k_stride[i];
        a.dst_v_stride[i] = L->dst_v_stride[i];
    }
    a.err_flag = L->err_flag;
    a.block_table = paging->block_table;
    a.v_block_table = paging->v_block_table;
    a.page_shift = shift;
    a.max_pages = paging->max_pages;
    a.n_pages = paging->n_pages;
    a.dst_k_page_stride = paging->page_stride_k;
    a.dst_v_page_stride = paging->page_stride_v;
    a.block_tokens = scales->block_tokens;
    a.k_scale = scales->k_scale;
    a.v_scale = scales->v_scale;
    for (int i = 0; i < 4; ++i) {
        a.k_scale_stride[i] = scales->k_stride[i];
        a.v_scale_stride[i] = scales->v_stride[i];
    }
    if (!pkv::store_fits(a))
        return fail(PKV_ERR_UNSUPPORTED, "n_layers x n_kv_heads or max_seg_tokens beyond the grid's limits");
    if (accepted) {
        a.rows = accepted->path;
        a.n_rows = accepted->n_accepted;
        a.max_rows = accepted->max_path;
    }
    return device_status(pkv::launch_store(a, (hipStream_t)stream), accepted ? "tree_commit launch" : "reposition_splice_quant launch");
}

}  // namespace

PKV_EXPORT pkv_status pkv_reposition_splice_quant(const void* src_k, const void* src_v, void* k_pages, void* v_pages,
                                               const pkv_segment_quant* segs, int32_t n_segs, int32_t max_seg_tokens,
                                               const int32_t* kv_len, int32_t n_seqs, const double* omega,
                                               float rope_theta, int32_t rope_dim, const pkv_layout* layout,
                                               const pkv_paged_cache* paging, const pkv_block_scales* scales,
                                               void* stream) {
    return splice_quant(src_k, src_v, k_pages, v_pages, segs, n_segs, max_seg_tokens, kv_len, n_seqs, omega, rope_theta,
                        rope_dim, layout, paging, scales, nullptr, stream);
}

namespace {

// Validation of a page pool; fills `a` (without tables, counts and workspace).
pkv_status check_pool(const pkv_page_pool* P, pkv::PagesArgs& a) {
    if (!P) return fail(PKV_ERR_NULL, "pool is NULL");
    const int32_t b = P->page_size;
    if (b < 32 || b > (1 << 20) || (b & (b - 1)))
        return fail(PKV_ERR_SHAPE, "page_size %d must be a power of two in [32, 2^20]", b);
    if (P->n_seqs <= 0 || P->max_pages <= 0 || P->n_pages <= 0 || P->n_pages > 0x7fffffff)
        return fail(PKV_ERR_SHAPE, "n_seqs (%d), max_pages (%d) and n_pages (%lld) must be positive (n_pages < 2^31)",
                    P->n_seqs, P->max_pages, (long long)P->n_pages);
    if (P->n_tensors < 1 || P->n_tensors > 4) return fail(PKV_ERR_SHAPE, "n_tensors %d must be 1 .. 4", P->n_tensors);
    memset(&a, 0, sizeof a);
    Range r[4];
    for (int i = 0; i < P->n_tensors; ++i) {
        const pkv_page_tensor& t = P->tensors[i];
        if (!t.data) return fail(PKV_ERR_NULL, "tensor %d is NULL", i);
        if (t.n_layers <= 0 || t.n_slots <= 0 || t.n_heads <= 0 || t.row_bytes <= 0 || b % t.n_slots)
            return fail(PKV_ERR_SHAPE, "tensor %d: sizes must be positive and n_slots (%d) divide page_size", i, t.n_slots);
        const int64_t st[4] = {t.layer_stride, t.head_stride, t.page_stride, t.slot_stride};
        const int64_t cnt[4] = {t.n_layers, t.n_heads, P->n_pages, t.n_slots};
        for (int k = 0; k < 4; ++k)
            if (st[k] < 0 || (st[k] == 0 && cnt[k] > 1))
                return fail(PKV_ERR_SHAPE, "tensor %d: strides must be positive", i);
        r[i] = extent(t.data, st, cnt, 4, t.row_bytes, 1);
        for (int k = 0; k < i; ++k)
            if (overlap(r[i], r[k])) return fail(PKV_ERR_ALIAS, "tensors %d and %d overlap", k, i);
        // Rows move in the widest units that every address allows.
        uint64_t bits = (uint64_t)(uintptr_t)t.data | (uint64_t)t.row_bytes | 16u;
        for (int k = 0; k < 4; ++k)
            if (cnt[k] > 1) bits |= (uint64_t)st[k];
        pkv::PageTensor& p = a.tensors[i];
        while (!((bits >> p.unit_shift) & 1)) ++p.unit_shift;
        p.data = (char*)t.data;
        p.layer_stride = t.layer_stride;
        p.page_stride = t.page_stride;
        p.slot_stride = t.slot_stride;
        p.head_stride = t.head_stride;
        p.layers = t.n_layers;
        p.slots = t.n_slots;
        p.heads = t.n_heads;
        p.row_units = t.row_bytes >> p.unit_shift;
        p.slot_tokens = b / t.n_slots;
        const double units = (double)p.layers * p.slots * p.heads * p.row_units;
        if (units >= 2147483648.0 - 65536.0)
            return fail(PKV_ERR_UNSUPPORTED, "tensor %d: a page of all layers has 2^31 units or more", i);
    }
    a.n_tensors = P->n_tensors;
    a.page_size = b;
    while ((1 << a.page_shift) < b) ++a.page_shift;
    a.n_seqs = P->n_seqs;
    a.max_pages = P->max_pages;
    a.n_pages = P->n_pages;
    a.err_flag = P->err_flag;
    return PKV_OK;
}

// x and y (n int32 each) are one array or apart.
bool same_or_apart(const int32_t* x, const int32_t* y, int64_t n) {
    return x == y || (uintptr_t)x + (uintptr_t)n * 4 <= (uintptr_t)y || (uintptr_t)y + (uintptr_t)n * 4 <= (uintptr_t)x;
}

pkv_status use_workspace(pkv::PagesArgs& a, int n_forks, void* workspace, size_t bytes) {
    const size_t need = pkv::pages_workspace_bytes(a, n_forks);
    if (!workspace) return fail(PKV_ERR_NULL, "workspace of %zu bytes is required", need);
    if (bytes < need) return fail(PKV_ERR_SHAPE, "workspace_bytes %zu < required %zu", bytes, need);
    if (!aligned16(workspace)) return fail(PKV_ERR_ALIGN, "workspace must be 16-byte aligned");
    pkv::pages_set_workspace(a, n_forks, workspace);
    return PKV_OK;
}

}  // namespace

PKV_EXPORT size_t pkv_pages_workspace_size(const pkv_page_pool* pool, int32_t n_forks) {
    pkv::PagesArgs a;
    char saved[sizeof g_err];
    memcpy(saved, g_err, sizeof g_err);
    const pkv_status st = check_pool(pool, a);
    memcpy(g_err, saved, sizeof g_err);
    if (st != PKV_OK || n_forks < 0 || n_forks > 65535) return 0;
    return pkv::pages_workspace_bytes(a, n_forks);
}

PKV_EXPORT pkv_status pkv_pages_free(const pkv_page_pool* pool, int32_t* ref, int32_t* block_table, const int32_t* seqs,
                                     const int32_t* keep, int32_t n, void* stream) {
    pkv::PagesArgs a;
    const pkv_status st = check_pool(pool, a);
    if (st != PKV_OK) return st;
    if (!ref || !block_table) return fail(PKV_ERR_NULL, "ref and block_table are required");
    if (n < 0) return fail(PKV_ERR_SHAPE, "n (%d) must be non-negative", n);
    if (n > 65535) return fail(PKV_ERR_UNSUPPORTED, "at most 65535 sequences per call");
    if (n > 0 && !seqs) return fail(PKV_ERR_NULL, "seqs is NULL");
    if (n == 0) return ok();
    a.ref = ref;
    a.table = block_table;
    a.seqs = seqs;
    a.keep = keep;
    a.n = n;
    return device_status(pkv::launch_pages_free(a, (hipStream_t)stream), "pages_free launch");
}

PKV_EXPORT pkv_status pkv_pages_fork(const pkv_page_pool* pool, int32_t* ref, const int32_t* table_in,
                                     int32_t* table_out, const pkv_fork* forks, int32_t n_forks, void* workspace,
                                     size_t workspace_bytes, void* stream) {
    static_assert(sizeof(pkv_fork) == sizeof(pkv::PageFork), "fork layout");
    pkv::PagesArgs a;
    pkv_status st = check_pool(pool, a);
    if (st != PKV_OK) return st;
    if (!ref || !table_in || !table_out) return fail(PKV_ERR_NULL, "ref, table_in and table_out are required");
    if (n_forks < 0) return fail(PKV_ERR_SHAPE, "n_forks (%d) must be non-negative", n_forks);
    if (n_forks > 65535) return fail(PKV_ERR_UNSUPPORTED, "at most 65535 forks per call");
    if (n_forks > 0 && !forks) return fail(PKV_ERR_NULL, "forks is NULL");
    if (!aligned16(forks)) return fail(PKV_ERR_ALIGN, "forks must be 16-byte aligned");
    if (!same_or_apart(table_in, table_out, (int64_t)a.n_seqs * a.max_pages))
        return fail(PKV_ERR_ALIAS, "table_in and table_out overlap in part");
    if (n_forks == 0) return ok();
    st = use_workspace(a, n_forks, workspace, workspace_bytes);
    if (st != PKV_OK) return st;
    a.ref_in = ref;
    a.ref = ref;
    a.table_in = table_in;
    a.table = table_out;
    a.forks = (const pkv::PageFork*)forks;
    a.n = n_forks;
    return device_status(pkv::launch_pages_fork(a, (hipStream_t)stream), "pages_fork launch");
}

PKV_EXPORT pkv_status pkv_pages_compact(const pkv_page_pool* pool, const int32_t* ref_in, int32_t* ref_out,
                                        const int32_t* table_in, int32_t* table_out, int32_t* n_used, void* workspace,
                                        size_t workspace_bytes, void* stream) {
    pkv::PagesArgs a;
    pkv_status st = check_pool(pool, a);
    if (st != PKV_OK) return st;
    if (!ref_in || !ref_out || !table_in || !table_out || !n_used)
        return fail(PKV_ERR_NULL, "ref_in, ref_out, table_in, table_out and n_used are required");
    if (!same_or_apart(table_in, table_out, (int64_t)a.n_seqs * a.max_pages))
        return fail(PKV_ERR_ALIAS, "table_in and table_out overlap in part");
    if (!same_or_apart(ref_in, ref_out, a.n_pages)) return fail(PKV_ERR_ALIAS, "ref_in and ref_out overlap in part");
    st = use_workspace(a, 0, workspace, workspace_bytes);
    if (st != PKV_OK) return st;
    a.ref_in = ref_in;
    a.ref = ref_out;
    a.table_in = table_in;
    a.table = table_out;
    a.n_used = n_used;
    return device_status(pkv::launch_pages_compact(a, (hipStream_t)stream), "pages_compact launch");
}

// ---- trees of drafted tokens ------------------------------------------------------

PKV_EXPORT pkv_status pkv_tree_masks(const int32_t* parent, const int32_t* cu_q, const int32_t* kv_len, int32_t n_seqs,
                                     int32_t total_q, int32_t max_q, uint32_t* mask, int32_t mask_words, int32_t* q_pos,
                                     int32_t* err_flag, void* stream) {
    if (!parent || !mask) return fail(PKV_ERR_NULL, "parent and mask are required");
    if (q_pos && !kv_len) return fail(PKV_ERR_NULL, "q_pos needs kv_len");
    if (n_seqs <= 0 || total_q < 0 || max_q < 0 || mask_words <= 0)
        return fail(PKV_ERR_SHAPE, "n_seqs (%d) and mask_words (%d) must be positive, total_q (%d) and max_q (%d) non-negative",
                    n_seqs, mask_words, total_q, max_q);
    if (n_seqs > 1 && !cu_q) return fail(PKV_ERR_NULL, "cu_q is required when n_seqs > 1");
    if (!cu_q) {
        if (max_q < total_q) return fail(PKV_ERR_SHAPE, "max_q (%d) < total_q (%d)", max_q, total_q);
        max_q = total_q;
    }
    if (max_q > pkv::kTreeMaxRows)
        return fail(PKV_ERR_UNSUPPORTED, "trees of %d rows (at most %d)", max_q, pkv::kTreeMaxRows);
    if (mask_words < (max_q + 31) / 32) return fail(PKV_ERR_SHAPE, "mask_words (%d) must hold max_q (%d) bits", mask_words, max_q);
    if (total_q == 0 || max_q == 0) return ok();
    const pkv::TreeMaskArgs a = {parent, cu_q, kv_len, n_seqs, total_q, max_q, mask_words, mask, q_pos, err_flag};
    return device_status(pkv::launch_tree_masks(a, (hipStream_t)stream), "tree_masks launch");
}

PKV_EXPORT size_t pkv_tree_attention_workspace_size(const pkv_attn_desc* desc, int32_t n_q_heads, int32_t n_kv_heads,
                                                    int32_t head_dim, int32_t quant) {
    return workspace_size(desc, n_q_heads, n_kv_heads, head_dim, quant != 0, true);
}

PKV_EXPORT pkv_status pkv_tree_attention(const void* q, const void* k_cache, const void* v_cache, void* out,
                                         const int32_t* q_pos, const int32_t* kv_len, int32_t n_q_heads,
                                         int32_t n_kv_heads, int32_t head_dim, float scale, const pkv_attn_desc* desc,
                                         const pkv_draft* draft, const pkv_paged_cache* paging,
                                         const pkv_block_scales* scales, void* workspace, size_t workspace_bytes,
                                         void* stream) {
    if (!draft) return fail(PKV_ERR_NULL, "draft is NULL");
    if (scales && !paging) return fail(PKV_ERR_NULL, "a cache held in 8 bits is paged: paging is NULL");
    return run_attention(q, k_cache, v_cache, out, q_pos, kv_len, n_q_heads, n_kv_heads, head_dim, scale, desc, paging,
                         scales, workspace, workspace_bytes, stream, draft);
}

namespace {

pkv_status check_verify(const pkv_verify_desc* d) {
    if (!d) return fail(PKV_ERR_NULL, "desc is NULL");
    if (d->dtype != PKV_BF16 && d->dtype != PKV_F32)
        return fail(PKV_ERR_UNSUPPORTED, "dtype %d (expected PKV_BF16 or PKV_F32)", d->dtype);
    if (d->n_seqs <= 0 || d->total_q < 0 || d->max_q < 0 || d->vocab <= 0 || d->max_path <= 0)
        return fail(PKV_ERR_SHAPE,
                    "n_seqs (%d), vocab (%d) and max_path (%d) must be positive, total_q (%d) and max_q (%d) non-negative",
                    d->n_seqs, d->vocab, d->max_path, d->total_q, d->max_q);
    if (d->reserved != 0) return fail(PKV_ERR_SHAPE, "desc.reserved must be 0");
    if (d->n_seqs > 1 && !d->cu_q) return fail(PKV_ERR_NULL, "cu_q is required when n_seqs > 1");
    if (!d->cu_q && d->max_q < d->total_q) return fail(PKV_ERR_SHAPE, "max_q (%d) < total_q (%d)", d->max_q, d->total_q);
    if (d->target_stride < 0 || d->draft_stride < 0) return fail(PKV_ERR_SHAPE, "strides must be non-negative");
    if ((d->cu_q ? d->max_q : d->total_q) > pkv::kTreeMaxRows)
        return fail(PKV_ERR_UNSUPPORTED, "trees of %d rows (at most %d)", d->max_q, pkv::kTreeMaxRows);
    if (d->n_seqs > 65535) return fail(PKV_ERR_UNSUPPORTED, "at most 65535 sequences per call");
    return PKV_OK;
}

}  // namespace

PKV_EXPORT size_t pkv_tree_verify_workspace_size(const pkv_verify_desc* desc) {
    char saved[sizeof g_err];
    memcpy(saved, g_err, sizeof g_err);
    const pkv_status st = check_verify(desc);
    memcpy(g_err, saved, sizeof g_err);
    return st == PKV_OK ? pkv::tree_verify_workspace_bytes(desc->n_seqs, desc->vocab) : 0;
}

PKV_EXPORT pkv_status pkv_tree_verify(const void* target_probs, const void* draft_probs, const int32_t* tokens,
                                      const int32_t* parent, const float* u_accept, const float* u_sample, int32_t* path,
                                      int32_t* n_accepted, int32_t* next_token, const pkv_verify_desc* desc,
                                      void* workspace, size_t workspace_bytes, void* stream) {
    const pkv_status st = check_verify(desc);
    if (st != PKV_OK) return st;
    const bool rows = desc->total_q > 0;   // (a call without rows has no tensors of rows)
    if ((rows && (!target_probs || !tokens || !parent || !u_accept)) || !u_sample || !path || !n_accepted || !next_token)
        return fail(PKV_ERR_NULL, "target_probs, tokens, parent, u_accept, u_sample, path, n_accepted and next_token are required");
    const uintptr_t eb = desc->dtype == PKV_BF16 ? 2 : 4;
    if ((uintptr_t)target_probs % eb || (uintptr_t)draft_probs % eb)
        return fail(PKV_ERR_ALIGN, "probabilities must be aligned to their type");
    const size_t need = pkv::tree_verify_workspace_bytes(desc->n_seqs, desc->vocab);
    if (!workspace) return fail(PKV_ERR_NULL, "workspace of %zu bytes is required", need);
    if (workspace_bytes < need) return fail(PKV_ERR_SHAPE, "workspace_bytes %zu < required %zu", workspace_bytes, need);
    if (!aligned16(workspace)) return fail(PKV_ERR_ALIGN, "workspace must be 16-byte aligned");
    pkv::TreeVerifyArgs a;
    memset(&a, 0, sizeof a);
    a.target = target_probs;
    a.draft = draft_probs;
    a.target_stride = desc->target_stride;
    a.draft_stride = desc->draft_stride;
    a.tokens = tokens;
    a.parent = parent;
    a.cu_q = desc->cu_q;
    a.u_accept = u_accept;
    a.u_sample = u_sample;
    a.dtype = desc->dtype;
    a.n_seqs = desc->n_seqs;
    a.total_q = desc->total_q;
    a.max_q = desc->cu_q ? desc->max_q : desc->total_q;
    a.vocab = desc->vocab;
    a.max_path = desc->max_path;
    a.path = path;
    a.n_accepted = n_accepted;
    a.next_token = next_token;
    a.err_flag = desc->err_flag;
    a.workspace = workspace;
    return device_status(pkv::launch_tree_verify(a, (hipStream_t)stream), "tree_verify launch");
}

PKV_EXPORT size_t pkv_tree_commit_workspace_size(int32_t n_seqs, int32_t max_path, int32_t quant) {
    (void)n_seqs, (void)max_path, (void)quant;
    return 0;
}

PKV_EXPORT pkv_status pkv_tree_commit(const void* draft_k, const void* draft_v, void* cache_k, void* cache_v,
                                      const int32_t* path, const int32_t* n_accepted, const int32_t* kv_len,
                                      const int64_t* kv_base, int32_t n_seqs, int32_t max_path, const pkv_layout* layout,
                                      const pkv_paged_cache* paging, const pkv_block_scales* scales, void* workspace,
                                      size_t workspace_bytes, void* stream) {
    (void)workspace, (void)workspace_bytes;
    const pkv_layout* L = layout;
    if (!L) return fail(PKV_ERR_NULL, "layout is NULL");
    if (!path || !n_accepted || !kv_len) return fail(PKV_ERR_NULL, "path, n_accepted and kv_len are required");
    if (n_seqs <= 0 || max_path <= 0)
        return fail(PKV_ERR_SHAPE, "n_seqs (%d) and max_path (%d) must be positive", n_seqs, max_path);
    if (paging && kv_base) return fail(PKV_ERR_SHAPE, "kv_base must be NULL for a paged cache");
    if (scales && !paging) return fail(PKV_ERR_NULL, "a cache held in 8 bits is paged: paging is NULL");
    if (max_path > 65535) return fail(PKV_ERR_UNSUPPORTED, "max_path (%d) above 65535", max_path);
    pkv::TreeCommitArgs t;
    memset(&t, 0, sizeof t);
    t.n_rows = L->n_tokens;
    t.capacity = L->dst_capacity;
    t.path = path;
    t.n_accepted = n_accepted;
    t.kv_len = kv_len;
    t.kv_base = kv_base;
    t.n_seqs = n_seqs;
    t.max_path = max_path;
    t.err_flag = L->err_flag;
    // Rows that are at their positions: any rotary slice will do, the smallest one.
    pkv_layout at = *L;
    at.rope_offset = 0;
    at.rope_style = PKV_ROPE_HALF;
    if (L->n_tokens == 0) {   // no drafted rows, and so no tensors of them: whatever is accepted is flagged
        static const char none[16] __attribute__((aligned(16))) = {0};   // (never read)
        if (!draft_k) draft_k = none;
        if (!draft_v && L->v_dim > 0) draft_v = none;
        for (int i = 0; i < 3; ++i) at.src_k_stride[i] = at.src_v_stride[i] = 0;
    }
    if (scales)
        return splice_quant(draft_k, draft_v, cache_k, cache_v, nullptr, n_seqs, max_path, kv_len, n_seqs, nullptr, 1.0f, 16, &at,
                            paging, scales, &t, stream);
    pkv::SpliceArgs a;
    const pkv_status st = check_splice(draft_k, draft_v, cache_k, cache_v, 1.0f, 2 * (at.dtype == PKV_F32 ? 4 : 8), &at, false, a,
                                       paging);
    if (st != PKV_OK) return st;
    t.src[0] = a.src_k;
    t.src[1] = a.src_v;
    t.dst[0] = a.dst_k;
    t.dst[1] = a.dst_v;
    for (int i = 0; i < 3; ++i) {
        t.src_stride[0][i] = a.src_k_stride[i] * a.elem_bytes;
        t.src_stride[1][i] = a.src_v_stride[i] * a.elem_bytes;
        t.dst_stride[0][i] = a.dst_k_stride[i] * a.elem_bytes;
        t.dst_stride[1][i] = a.dst_v_stride[i] * a.elem_bytes;
    }
    t.row_bytes[0] = a.head_dim * a.elem_bytes;
    t.row_bytes[1] = a.v_dim * a.elem_bytes;
    t.n_layers = a.n_layers;
    t.n_kv_heads = a.n_kv_heads;
    if (paging) {
        t.table[0] = a.dst_pages;
        t.table[1] = a.dst_v_pages ? a.dst_v_pages : a.dst_pages;
        t.page_shift = a.page_shift;
        t.max_pages = a.max_pages;
        t.n_pages = a.n_pages;
        t.page_stride[0] = a.dst_k_page_stride * a.elem_bytes;
        t.page_stride[1] = a.dst_v_page_stride * a.elem_bytes;
    }
    return device_status(pkv::launch_tree_commit(t, (hipStream_t)stream), "tree_commit launch");
}

PKV_EXPORT const char* pkv_last_error(void) { return g_err; }

PKV_EXPORT int32_t pkv_version(void) { return PKV_VERSION; }
