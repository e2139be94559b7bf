"""Host-side refusals of the 8-bit cache's and the pages' entry points (fake device addresses, so only without a
GPU), their structs, and the binding's checks of its arguments."""
import ctypes

import pytest
import torch

from paper_2606_17107_amd import pkv

needs_no_gpu = pytest.mark.skipif(torch.cuda.is_available(), reason="fake-pointer validation tests run only without a GPU")

BASE = 1 << 40
GB = 1 << 30


def test_struct_sizes():
    assert ctypes.sizeof(pkv.pkv_segment_quant) == 24
    assert ctypes.sizeof(pkv.pkv_block_scales) == 8 + 16 + 64
    assert ctypes.sizeof(pkv.pkv_page_tensor) == 8 + 32 + 16
    assert ctypes.sizeof(pkv.pkv_page_pool) == 16 + 8 + 4 * 56 + 8
    assert ctypes.sizeof(pkv.pkv_fork) == 16


# ---- splice -------------------------------------------------------------------

def splice_args(**kw):
    L = pkv.pkv_layout()
    L.dtype, L.n_layers, L.n_kv_heads, L.head_dim, L.v_dim = 0, 2, 4, 128, 128
    L.n_tokens, L.rope_offset, L.rope_style, L.dst_capacity, L.reserved = 100, 0, 0, 256, 0
    L.src_k_stride = L.src_v_stride = pkv._i64x3(4 * 100 * 128, 100 * 128, 128)
    L.dst_k_stride = L.dst_v_stride = pkv._i64x3(20 * 64 * 512, 128, 512)
    pg = pkv.pkv_paged_cache()
    pg.page_size, pg.max_pages, pg.block_table, pg.n_pages = 64, 4, BASE, 20
    pg.page_stride_k = pg.page_stride_v = 64 * 512
    s = pkv.pkv_block_scales(64, 0, BASE + 10 * GB, BASE + 11 * GB, pkv._i64x4(80, 1, 4, 4), pkv._i64x4(80, 1, 4, 4))
    a = dict(src_k=BASE + GB, src_v=BASE + 2 * GB, k_pages=BASE + 3 * GB, v_pages=BASE + 4 * GB, segs=BASE + 5 * GB, n_segs=2,
             max_seg_tokens=50, kv_len=BASE + 6 * GB, n_seqs=3, omega=None, rope_theta=1e4, rope_dim=128, layout=L,
             paging=pg, scales=s)
    for k, v in kw.items():
        if k in a:
            a[k] = v
        else:
            obj, field = k.split("__")
            setattr({"L": L, "pg": pg, "s": s}[obj], field, v)
    return a


SPLICE_REFUSALS = [
    (dict(layout=None), 1), (dict(paging=None), 1), (dict(scales=None), 1), (dict(src_k=None), 1), (dict(k_pages=None), 1),
    (dict(src_v=None), 1), (dict(v_pages=None), 1), (dict(kv_len=None), 1), (dict(segs=None), 1),
    (dict(pg__block_table=None), 1), (dict(s__k_scale=None), 1), (dict(s__v_scale=None), 1),
    (dict(L__dtype=2), 5), (dict(L__rope_style=2), 5), (dict(L__head_dim=96), 5), (dict(L__head_dim=256), 5),
    (dict(L__v_dim=64), 5), (dict(L__v_dim=0), 2), (dict(L__reserved=1), 2), (dict(s__reserved=1), 2),
    (dict(L__n_layers=0), 2), (dict(L__n_kv_heads=0), 2), (dict(L__n_tokens=-1), 2), (dict(L__dst_capacity=-1), 2),
    (dict(L__dst_capacity=257), 2), (dict(n_segs=-1), 2), (dict(max_seg_tokens=-1), 2), (dict(n_seqs=0), 2),
    (dict(n_segs=65536), 5), (dict(rope_dim=0), 2), (dict(rope_dim=127), 2), (dict(rope_dim=256), 2), (dict(rope_dim=24), 5),
    (dict(L__rope_offset=4, rope_dim=64), 5), (dict(L__rope_offset=-8, rope_dim=64), 2), (dict(rope_theta=0.0), 2),
    (dict(rope_theta=float("nan")), 2), (dict(omega=[1.0] * 63 + [float("inf")]), 2),
    (dict(s__block_tokens=16), 2), (dict(s__block_tokens=96), 2), (dict(s__block_tokens=128), 2), (dict(s__block_tokens=0), 2),
    (dict(pg__page_size=48), 2), (dict(pg__page_size=16), 2), (dict(pg__n_pages=0), 2), (dict(pg__max_pages=0), 2),
    (dict(src_k=BASE + GB + 8), 3), (dict(v_pages=BASE + 4 * GB + 8), 3), (dict(segs=BASE + 5 * GB + 4), 3),
    (dict(L__src_k_stride=pkv._i64x3(51200, 12800, 132)), 3), (dict(L__dst_k_stride=pkv._i64x3(655360, 128, 520)), 3),
    (dict(L__src_v_stride=pkv._i64x3(51200, -12800, 128)), 2), (dict(pg__page_stride_v=-64), 2), (dict(pg__page_stride_k=72), 3),
    (dict(s__k_stride=pkv._i64x4(80, 1, -4, 4)), 2),
    (dict(k_pages=BASE + GB), 4), (dict(v_pages=BASE + 3 * GB + 1024), 4), (dict(s__v_scale=BASE + 10 * GB + 3), 4),
    (dict(s__k_scale=BASE + 3 * GB + 100), 4), (dict(L__n_layers=1 << 20, L__n_kv_heads=64), 4),
]


@needs_no_gpu
@pytest.mark.parametrize("change,status", SPLICE_REFUSALS)
def test_splice_refusals(change, status):
    assert pkv.pkv_reposition_splice_quant(**splice_args(**change)) == status, pkv.pkv_last_error()
    assert pkv.pkv_last_error()


@needs_no_gpu
def test_splice_nothing_to_do():
    for change in (dict(n_segs=0), dict(n_segs=0, segs=None), dict(max_seg_tokens=0), dict(L__dst_capacity=0)):
        assert pkv.pkv_reposition_splice_quant(**splice_args(**change)) == 0
    one = splice_args(n_segs=0)   # keys and values from one tensor are fine
    one["src_v"] = one["src_k"]
    assert pkv.pkv_reposition_splice_quant(**one) == 0
    keys = splice_args(n_segs=0, src_v=None, v_pages=None, L__v_dim=0, s__v_scale=None)
    assert pkv.pkv_reposition_splice_quant(**keys) == 0


@needs_no_gpu
def test_splice_slots_too_far_apart():
    """The rows of a block are addressed by 32-bit offsets: slots lie at most 16 MiB apart."""
    far, eb = 1 << 24, 2
    for name, most in (("src_k", far // eb), ("src_v", far // eb), ("dst_k", far), ("dst_v", far)):
        args = lambda step: splice_args(n_segs=0, **{"L__%s_stride" % name: pkv._i64x3(0, 0, step)})   # noqa: E731
        assert pkv.pkv_reposition_splice_quant(**args(most + 16)) == 2 and b"16 MiB" in pkv.pkv_last_error().encode()
        assert b"16 MiB" not in (pkv.pkv_reposition_splice_quant(**args(most)), pkv.pkv_last_error().encode())[1]


# ---- attention ------------------------------------------------------------------

def attention_args(**kw):
    d = pkv.pkv_attn_desc()
    d.dtype, d.variant, d.n_layers, d.n_seqs, d.head_dim_v = 0, 0, 2, 1, 128
    d.total_q, d.max_q, d.max_kv_len, d.cache_slots = 3, 3, 200, 256
    d.q_stride = d.o_stride = pkv._i64x3(3 * 8 * 128, 8 * 128, 128)
    d.k_stride = d.v_stride = pkv._i64x3(20 * 64 * 512, 128, 512)
    pg = pkv.pkv_paged_cache()
    pg.page_size, pg.max_pages, pg.block_table, pg.n_pages = 64, 4, BASE, 20
    pg.page_stride_k = pg.page_stride_v = 64 * 512
    s = pkv.pkv_block_scales(64, 0, BASE + 10 * GB, BASE + 11 * GB, pkv._i64x4(80, 1, 4, 4), pkv._i64x4(80, 1, 4, 4))
    a = dict(q=BASE + GB, k_pages=BASE + 2 * GB, v_pages=BASE + 3 * GB, out=BASE + 4 * GB, q_pos=BASE + 5 * GB,
             kv_len=BASE + 6 * GB, n_q_heads=8, n_kv_heads=4, head_dim=128, scale=0.1, desc=d, paging=pg, scales=s,
             workspace=None, workspace_bytes=0)
    for k, v in kw.items():
        if k in a:
            a[k] = v
        else:
            obj, field = k.split("__")
            setattr({"d": d, "pg": pg, "s": s}[obj], field, v)
    return a


ATTENTION_REFUSALS = [
    (dict(desc=None), 1), (dict(paging=None), 1), (dict(scales=None), 1), (dict(q=None), 1), (dict(out=None), 1),
    (dict(k_pages=None), 1), (dict(v_pages=None), 1), (dict(q_pos=None), 1), (dict(kv_len=None), 1),
    (dict(pg__block_table=None), 1), (dict(s__k_scale=None), 1), (dict(s__v_scale=None), 1), (dict(d__n_seqs=2), 1),
    (dict(d__dtype=1), 5), (dict(d__dtype=2), 5), (dict(d__variant=1), 5), (dict(head_dim=256), 5), (dict(head_dim=576), 5),
    (dict(d__head_dim_v=64), 2), (dict(n_q_heads=6), 2), (dict(scale=float("inf")), 2), (dict(d__window=-1), 2),
    (dict(d__kv_base=BASE), 2), (dict(d__cache_slots=257), 2), (dict(d__max_kv_len=(1 << 30) + 1), 2),
    (dict(s__block_tokens=48), 2), (dict(s__block_tokens=128), 2), (dict(s__reserved=7), 2), (dict(pg__page_size=100), 2),
    (dict(s__v_stride=pkv._i64x4(-1, 1, 4, 4)), 2), (dict(d__k_stride=pkv._i64x3(655360, 128, (1 << 26) + 16)), 2),
    (dict(d__k_stride=pkv._i64x3(655360, 128, 520)), 3), (dict(d__q_stride=pkv._i64x3(4096, 1024, 132)), 3),
    (dict(q=BASE + GB + 2), 3), (dict(k_pages=BASE + 2 * GB + 8), 3), (dict(pg__page_stride_k=100), 3),
    (dict(out=BASE + GB), 4), (dict(out=BASE + 3 * GB + 4096), 4), (dict(out=BASE + 11 * GB), 4), (dict(out=BASE + 10 * GB - 64), 4),
    (dict(d__n_splits=2), 1), (dict(d__n_splits=2, workspace=BASE + 12 * GB, workspace_bytes=16), 2),
    (dict(d__n_splits=2, workspace=BASE + 12 * GB + 4, workspace_bytes=1 << 28), 3),
]


@needs_no_gpu
@pytest.mark.parametrize("change,status", ATTENTION_REFUSALS)
def test_attention_refusals(change, status):
    assert pkv.pkv_suffix_attention_quant(**attention_args(**change)) == status, pkv.pkv_last_error()
    assert pkv.pkv_last_error()


@needs_no_gpu
def test_attention_nothing_to_do_and_workspace():
    assert pkv.pkv_suffix_attention_quant(**attention_args(d__total_q=0, d__max_q=0)) == 0
    d = attention_args(d__n_splits=2)["desc"]
    assert pkv.pkv_attention_quant_workspace_size(d, 8, 4, 128) == 2 * 2 * 3 * 8 * 129 * 4
    d.dtype = 1
    assert pkv.pkv_attention_quant_workspace_size(d, 8, 4, 128) == 0
    assert pkv.pkv_attention_quant_workspace_size(None, 8, 4, 128) == 0


# ---- pages ------------------------------------------------------------------------

def pool(**kw):
    p = pkv.pkv_page_pool()
    p.page_size, p.n_tensors, p.n_seqs, p.max_pages, p.n_pages = 64, 2, 6, 10, 100
    for i in range(2):
        p.tensors[i] = pkv.pkv_page_tensor(BASE + (1 + i) * GB, 100 * 64 * 512, 64 * 512, 512, 128, 2, 64, 4, 128)
    for k, v in kw.items():
        if k.startswith("t"):
            setattr(p.tensors[1], k[1:], v)
        else:
            setattr(p, k, v)
    return p


POOL_REFUSALS = [
    (dict(page_size=48), 2), (dict(page_size=16), 2), (dict(page_size=1 << 21), 2), (dict(n_tensors=0), 2), (dict(n_tensors=5), 2),
    (dict(n_seqs=0), 2), (dict(max_pages=0), 2), (dict(n_pages=0), 2), (dict(n_pages=1 << 31), 2), (dict(tdata=None), 1),
    (dict(tn_layers=0), 2), (dict(tn_slots=0), 2), (dict(tn_slots=48), 2), (dict(tn_slots=128), 2), (dict(tn_heads=0), 2),
    (dict(trow_bytes=0), 2), (dict(tpage_stride=0), 2), (dict(thead_stride=-128), 2), (dict(tdata=BASE + GB + 512), 4),
    (dict(trow_bytes=127, tn_layers=1 << 19), 5),
]


@needs_no_gpu
@pytest.mark.parametrize("change,status", POOL_REFUSALS)
def test_pool_refusals(change, status):
    p = pool(**change)
    ws = BASE + 20 * GB
    assert pkv.pkv_pages_free(p, BASE, BASE, BASE, None, 1) == status, pkv.pkv_last_error()
    assert pkv.pkv_pages_fork(p, BASE, BASE, BASE, BASE, 1, ws, 1 << 30) == status
    assert pkv.pkv_pages_compact(p, BASE, BASE, BASE, BASE, BASE, ws, 1 << 30) == status
    assert pkv.pkv_pages_workspace_size(p, 1) == 0 and pkv.pkv_pages_workspace_size(p, 0) == 0


@needs_no_gpu
def test_pages_refusals():
    p, ws, n = pool(), BASE + 20 * GB, 1 << 20
    R, T, F = BASE, BASE + 4096, BASE + 8192
    free, fork, compact = pkv.pkv_pages_free, pkv.pkv_pages_fork, pkv.pkv_pages_compact
    assert free(None, R, T, F, None, 1) == 1 and free(p, None, T, F, None, 1) == 1 and free(p, R, None, F, None, 1) == 1
    assert free(p, R, T, None, None, 1) == 1 and free(p, R, T, F, None, -1) == 2 and free(p, R, T, F, None, 65536) == 5
    assert free(p, R, T, None, None, 0) == 0
    assert fork(None, R, T, T, F, 1, ws, n) == 1 and fork(p, None, T, T, F, 1, ws, n) == 1
    assert fork(p, R, None, T, F, 1, ws, n) == 1 and fork(p, R, T, None, F, 1, ws, n) == 1
    assert fork(p, R, T, T, None, 1, ws, n) == 1 and fork(p, R, T, T, F, 1, None, n) == 1
    assert fork(p, R, T, T, F, -1, ws, n) == 2 and fork(p, R, T, T, F, 65536, ws, n) == 5 and fork(p, R, T, T, None, 0, None, 0) == 0
    assert fork(p, R, T, T, F + 8, 1, ws, n) == 3 and fork(p, R, T, T, F, 1, ws + 8, n) == 3
    assert fork(p, R, T, T + 16, F, 1, ws, n) == 4
    need = pkv.pkv_pages_workspace_size(p, 5)
    assert need >= 5 * (16 + 4 + 4) + 6 * 4 and fork(p, R, T, T, F, 5, ws, need - 1) == 2
    assert compact(p, None, R, T, T, F, ws, n) == 1 and compact(p, R, None, T, T, F, ws, n) == 1
    assert compact(p, R, R, None, T, F, ws, n) == 1 and compact(p, R, R, T, None, F, ws, n) == 1
    assert compact(p, R, R, T, T, None, ws, n) == 1 and compact(p, R, R, T, T, F, None, n) == 1
    assert compact(p, R, R + 16, T, T, F, ws, n) == 4 and compact(p, R, R, T, T + 4, F, ws, n) == 4
    assert compact(p, R, R, T, T, F, ws + 4, n) == 3
    need = pkv.pkv_pages_workspace_size(p, 0)
    assert need >= 50 * 16 + 100 * 4 and compact(p, R, R, T, T, F, ws, need - 1) == 2
    assert pkv.pkv_pages_workspace_size(p, -1) == 0 and pkv.pkv_pages_workspace_size(p, 65536) == 0


# ---- the binding -------------------------------------------------------------------

def test_binding_refuses_host_tensors_and_shapes():
    """Every tensor-level call refuses host tensors before an address goes down; make_* check shapes."""
    k = torch.zeros(1, 8, 64, 2, 64, dtype=torch.uint8)
    s = torch.zeros(1, 8, 2, 2, dtype=torch.uint8)
    table = torch.zeros(1, 4, dtype=torch.int32)
    ref = torch.zeros(8, dtype=torch.int32)
    src = torch.zeros(1, 2, 10, 64, dtype=torch.bfloat16)
    q = torch.zeros(1, 3, 4, 64, dtype=torch.bfloat16)
    segs = pkv.make_segments_quant([dict(src_slot0=0, seq=0, n_tokens=1, src_pos0=0, dst_pos0=0)], "cpu")
    assert segs.numel() == 24 and pkv.make_forks([dict(parent=0, child=1, n_tokens=2)] * 3, "cpu").numel() == 48
    with pytest.raises(ValueError, match="GPU"):
        pkv.reposition_splice_quant(src, src, k, k, s, s, segs, 1, 1, table[0], table, 1e4, 64)
    with pytest.raises(ValueError, match="GPU"):
        pkv.suffix_attention_quant(q, k, k, s, s, torch.zeros_like(q), table[0], table[0], table, 1.0, 10)
    for call in (lambda: pkv.pages_free([k], ref, table, 64, table[0]),
                 lambda: pkv.pages_fork([k], ref, table, 64, segs, 1), lambda: pkv.pages_compact([k], ref, table, 64)):
        with pytest.raises(ValueError, match="GPU"):
            call()
    p = pkv.make_page_pool([k, s], table, 64)
    assert (p.n_pages, p.n_seqs, p.max_pages, p.n_tensors) == (8, 1, 4, 2)
    assert (p.tensors[0].n_slots, p.tensors[0].row_bytes, p.tensors[1].n_slots, p.tensors[1].row_bytes) == (64, 64, 2, 1)
    assert (p.tensors[0].slot_stride, p.tensors[0].head_stride, p.tensors[1].head_stride) == (128, 64, 1)
    for bad in ([], [k] * 5, [k, s[:, :7]], [k[0, 0]], [k.transpose(3, 4)]):
        with pytest.raises(ValueError):
            pkv.make_page_pool(bad, table, 64)
    b = pkv.make_block_scales(s, None, 64)
    assert b.block_tokens == 32 and list(b.k_stride) == [32, 1, 4, 2] and not b.v_scale


@pytest.mark.parametrize("what", ["codes", "scales", "pages", "heads", "blocks", "values", "table", "lengths", "v table"])
def test_binding_checks_the_cache(what):
    """The checks of an 8-bit cache's tensors, run on host tensors (they compare devices with the one asked for)."""
    cpu = torch.device("cpu")
    k = torch.zeros(1, 8, 64, 2, 64, dtype=torch.uint8)
    s = torch.zeros(1, 8, 2, 2, dtype=torch.uint8)
    table, kv = torch.zeros(3, 4, dtype=torch.int32), torch.zeros(3, dtype=torch.int32)
    good = dict(k_pool=k, v_pool=k.clone(), k_scale=s, v_scale=s.clone(), block_table=table, v_block_table=None, kv_len=kv)
    pkv._check_q8_cache(cpu, **good)
    pkv._check_q8_cache(cpu, **dict(good, v_pool=None, v_scale=None))
    pkv._check_q8_cache(cpu, **dict(good, k_pool=k.view(torch.float8_e4m3fn), v_pool=k.view(torch.float8_e4m3fn)))
    bad = {"codes": dict(k_pool=k.short()), "scales": dict(k_scale=s.float()), "pages": dict(k_scale=s[:, :7], v_scale=s[:, :7]),
           "heads": dict(k_scale=s[..., :1], v_scale=s[..., :1]),
           "blocks": dict(k_scale=s.repeat(1, 1, 2, 1)[:, :, :3], v_scale=s.repeat(1, 1, 2, 1)[:, :, :3]),
           "values": dict(v_scale=None), "table": dict(block_table=table.long()), "lengths": dict(kv_len=kv[:2]),
           "v table": dict(v_block_table=table[:2])}[what]
    with pytest.raises((TypeError, ValueError)):
        pkv._check_q8_cache(cpu, **dict(good, **bad))
