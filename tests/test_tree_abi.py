"""Host-side refusals of the entry points for trees of drafted tokens (fake device addresses, so only without a GPU), their
structs, the binding's checks of its arguments, and the references against small cases worked out by hand."""
import ctypes

import numpy as np
import pytest
import torch

import tree_ref as T
from paper_2606_17107_amd import pkv

needs_no_gpu = pytest.mark.skipif(torch.cuda.is_available(), reason="fake-pointer validation tests run only without a GPU")

BASE = 1 << 40
GB = 1 << 30


def test_struct_sizes():
    assert ctypes.sizeof(pkv.pkv_draft) == 16 + 48 + 16
    assert ctypes.sizeof(pkv.pkv_verify_desc) == 24 + 8 + 16 + 8 + 8


def apply(a, objs, kw):
    for k, v in kw.items():
        if k in a:
            a[k] = v
        else:
            obj, field = k.split("__")
            setattr(objs[obj], field, v)
    return a


# ---- masks ----------------------------------------------------------------------

def masks_args(**kw):
    return apply(dict(parent=BASE, cu_q=BASE + GB, kv_len=BASE + 2 * GB, n_seqs=3, total_q=40, max_q=20, mask=BASE + 3 * GB,
                      mask_words=1, q_pos=BASE + 4 * GB, err_flag=None), {}, kw)


@needs_no_gpu
@pytest.mark.parametrize("kw,status", [
    (dict(parent=None), 1), (dict(mask=None), 1), (dict(kv_len=None), 1), (dict(cu_q=None), 1), (dict(n_seqs=0), 2),
    (dict(total_q=-1), 2), (dict(max_q=-1), 2), (dict(mask_words=0), 2), (dict(max_q=33), 2), (dict(max_q=1025, mask_words=33), 5),
    (dict(cu_q=None, n_seqs=1), 2), (dict(cu_q=None, n_seqs=1, max_q=1025, total_q=1025, mask_words=40), 5)])
def test_masks_refusals(kw, status):
    assert pkv.pkv_tree_masks(**masks_args(**kw)) == status
    assert pkv.pkv_last_error()


@needs_no_gpu
def test_masks_nothing_to_do():
    assert pkv.pkv_tree_masks(**masks_args(total_q=0)) == 0
    assert pkv.pkv_tree_masks(**masks_args(max_q=0)) == 0


# ---- attention ------------------------------------------------------------------

def attention_args(paged=False, quant=False, mla=False, **kw):
    H, Hkv, D, Dv = (16, 1, 576, 512) if mla else (8, 2, 128, 128)
    d = pkv.pkv_attn_desc()
    d.dtype, d.variant, d.n_layers, d.n_seqs, d.head_dim_v, d.total_q, d.max_q, d.max_kv_len = 0, int(mla), 2, 3, Dv, 30, 12, 256
    d.cu_q, d.cache_slots = BASE, 256
    d.q_stride = pkv._i64x3(30 * H * D, H * D, D)
    d.o_stride = pkv._i64x3(30 * H * Dv, H * Dv, Dv)
    d.k_stride = d.v_stride = pkv._i64x3(Hkv * 2000 * D, 2000 * D, D)
    pg = pkv.pkv_paged_cache()
    pg.page_size, pg.max_pages, pg.block_table, pg.n_pages = 64, 4, BASE + GB, 20
    pg.page_stride_k = pg.page_stride_v = 64 * Hkv * D
    s = pkv.pkv_block_scales(64, 0, BASE + 10 * GB, BASE + 11 * GB, pkv._i64x4(80, 1, 4, 4), pkv._i64x4(80, 1, 4, 4))
    t = pkv.pkv_draft(BASE + 2 * GB, BASE + (2 if mla else 3) * GB, pkv._i64x3(30 * Hkv * D, D, Hkv * D),
                      pkv._i64x3(30 * Hkv * D, D, Hkv * D), BASE + 4 * GB, 1, 0)
    a = dict(q=BASE + 5 * GB, k_cache=BASE + 6 * GB, v_cache=BASE + (6 if mla else 7) * GB, out=BASE + 8 * GB, q_pos=BASE,
             kv_len=BASE, n_q_heads=H, n_kv_heads=Hkv, head_dim=D, scale=0.1, desc=d, draft=t, paging=pg if paged or quant else None,
             scales=s if quant else None, workspace=BASE + 9 * GB, workspace_bytes=1 << 30)
    return apply(a, dict(d=d, pg=pg, s=s, t=t), kw)


ATTENTION_REFUSALS = [
    (dict(draft=None), 1), (dict(t__k=None), 1), (dict(t__v=None), 1), (dict(q=None), 1), (dict(workspace=None), 1),
    (dict(workspace_bytes=64), 2), (dict(workspace=BASE + 8), 3), (dict(t__reserved=1), 2), (dict(t__k=BASE + 8), 3),
    (dict(t__v=BASE + 4), 3), (dict(t__mask=BASE + 2), 3), (dict(t__mask_words=0), 2), (dict(d__max_q=33), 2),
    (dict(t__k_stride=pkv._i64x3(-8, 128, 256)), 2), (dict(t__v_stride=pkv._i64x3(4, 128, 256)), 3),
    (dict(t__k_stride=pkv._i64x3(0, 0, (1 << 25) + 8)), 2), (dict(out=BASE + 2 * GB), 4), (dict(out=BASE + 3 * GB), 4), (dict(out=BASE + 4 * GB), 4), (dict(out=BASE + 6 * GB), 4),
    (dict(head_dim=96), 5), (dict(d__dtype=3), 5), (dict(d__window=-1), 2), (dict(n_kv_heads=3), 2), (dict(scale=float("nan")), 2),
]


@needs_no_gpu
@pytest.mark.parametrize("form", [dict(), dict(paged=True), dict(quant=True)])
@pytest.mark.parametrize("kw,status", ATTENTION_REFUSALS)
def test_attention_refusals(kw, status, form):
    assert pkv.pkv_tree_attention(**attention_args(**form, **kw)) == status
    assert pkv.pkv_last_error()


@needs_no_gpu
@pytest.mark.parametrize("form,kw,status", [
    (dict(quant=True), dict(paging=None), 1), (dict(quant=True), dict(s__block_tokens=16), 2), (dict(quant=True), dict(d__dtype=1), 5),
    (dict(paged=True), dict(d__dtype=1), 5), (dict(paged=True), dict(d__kv_base=BASE), 2), (dict(paged=True), dict(pg__page_size=48), 2),
    (dict(mla=True), dict(t__v=BASE + 3 * GB), 2), (dict(mla=True), dict(t__v_stride=pkv._i64x3(0, 0, 576)), 2),
    (dict(mla=True), dict(d__dtype=1), 5), (dict(quant=True, mla=True), dict(), 5)])
def test_attention_refusals_of_forms(form, kw, status):
    assert pkv.pkv_tree_attention(**attention_args(**form, **kw)) == status


def test_attention_workspace():
    """A record per split and row: always one at least, none without a cache."""
    a = attention_args()
    rows = 2 * 30 * 8
    size = pkv.pkv_tree_attention_workspace_size(a["desc"], 8, 2, 128, 0)
    assert size >= rows * 129 * 4 and size % (rows * 129 * 4) == 0
    for n in (1, 3):
        a["desc"].n_splits = n
        assert pkv.pkv_tree_attention_workspace_size(a["desc"], 8, 2, 128, 0) == n * rows * 129 * 4
        assert pkv.pkv_tree_attention_workspace_size(a["desc"], 8, 2, 128, 1) == n * rows * 129 * 4
    a["desc"].max_kv_len = 0
    assert pkv.pkv_tree_attention_workspace_size(a["desc"], 8, 2, 128, 0) == 0
    assert pkv.pkv_tree_attention_workspace_size(a["desc"], 8, 3, 128, 0) == 0
    assert pkv.pkv_tree_attention_workspace_size(None, 8, 2, 128, 0) == 0


# ---- verification ---------------------------------------------------------------

def verify_args(**kw):
    d = pkv.pkv_verify_desc(0, 3, 30, 12, 1000, 5, BASE, 1000, 1000, None, 0)
    a = dict(target_probs=BASE + GB, draft_probs=BASE + 2 * GB, tokens=BASE, parent=BASE, u_accept=BASE, u_sample=BASE, path=BASE,
             n_accepted=BASE, next_token=BASE, desc=d, workspace=BASE + 3 * GB, workspace_bytes=1 << 20)
    return apply(a, dict(d=d), kw)


@needs_no_gpu
@pytest.mark.parametrize("kw,status", [
    (dict(desc=None), 1), (dict(target_probs=None), 1), (dict(tokens=None), 1), (dict(parent=None), 1), (dict(u_accept=None), 1),
    (dict(u_sample=None), 1), (dict(path=None), 1), (dict(n_accepted=None), 1), (dict(next_token=None), 1), (dict(workspace=None), 1),
    (dict(workspace_bytes=64), 2), (dict(workspace=BASE + 8), 3), (dict(target_probs=BASE + 1), 3), (dict(draft_probs=BASE + 1), 3),
    (dict(d__dtype=1, target_probs=BASE + 2), 3), (dict(d__dtype=2), 5), (dict(d__n_seqs=0), 2), (dict(d__vocab=0), 2),
    (dict(d__max_path=0), 2), (dict(d__total_q=-1), 2), (dict(d__max_q=-1), 2), (dict(d__reserved=1), 2), (dict(d__cu_q=None), 1),
    (dict(d__cu_q=None, d__n_seqs=1), 2), (dict(d__target_stride=-1), 2), (dict(d__max_q=1025), 5), (dict(d__n_seqs=65536), 5)])
def test_verify_refusals(kw, status):
    assert pkv.pkv_tree_verify(**verify_args(**kw)) == status
    assert pkv.pkv_last_error()


def test_verify_workspace():
    d = verify_args()["desc"]
    one = pkv.pkv_tree_verify_workspace_size(d)
    assert one > 0
    d.n_seqs = 6
    assert pkv.pkv_tree_verify_workspace_size(d) == 2 * one
    d.vocab = 0
    assert pkv.pkv_tree_verify_workspace_size(d) == 0


# ---- commit ---------------------------------------------------------------------

def commit_args(paged=False, quant=False, **kw):
    L = pkv.pkv_layout()
    L.dtype, L.n_layers, L.n_kv_heads, L.head_dim, L.v_dim, L.n_tokens, L.dst_capacity = 0, 2, 4, 128, 128, 30, 256
    L.src_k_stride = L.src_v_stride = pkv._i64x3(30 * 512, 128, 512)
    L.dst_k_stride = L.dst_v_stride = pkv._i64x3(20 * 64 * 512, 128, 512)
    pg = pkv.pkv_paged_cache()
    pg.page_size, pg.max_pages, pg.block_table, pg.n_pages = 64, 4, BASE, 20
    pg.page_stride_k = pg.page_stride_v = 64 * 512
    s = pkv.pkv_block_scales(64, 0, BASE + 10 * GB, BASE + 11 * GB, pkv._i64x4(80, 1, 4, 4), pkv._i64x4(80, 1, 4, 4))
    a = dict(draft_k=BASE + GB, draft_v=BASE + 2 * GB, cache_k=BASE + 3 * GB, cache_v=BASE + 4 * GB, path=BASE, n_accepted=BASE,
             kv_len=BASE, kv_base=None, n_seqs=3, max_path=5, layout=L, paging=pg if paged or quant else None,
             scales=s if quant else None, workspace=BASE + 9 * GB, workspace_bytes=1 << 20)
    return apply(a, dict(L=L, pg=pg, s=s), kw)


@needs_no_gpu
@pytest.mark.parametrize("form", [dict(), dict(paged=True), dict(quant=True)])
@pytest.mark.parametrize("kw,status", [
    (dict(layout=None), 1), (dict(draft_k=None), 1), (dict(draft_v=None), 1), (dict(cache_k=None), 1), (dict(path=None), 1),
    (dict(n_accepted=None), 1), (dict(kv_len=None), 1), (dict(n_seqs=0), 2), (dict(max_path=0), 2), (dict(max_path=65536), 5),
    (dict(L__dtype=2), 5), (dict(L__n_tokens=-1), 2), (dict(L__v_dim=0), 2), (dict(L__reserved=1), 2), (dict(draft_k=BASE + GB + 8), 3),
    (dict(cache_k=BASE + GB), 4), (dict(cache_v=BASE + 3 * GB), 4), (dict(L__src_k_stride=pkv._i64x3(-8, 128, 512)), 2)])
def test_commit_refusals(kw, status, form):
    assert pkv.pkv_tree_commit(**commit_args(**form, **kw)) == status
    assert pkv.pkv_last_error()


@needs_no_gpu
@pytest.mark.parametrize("form,kw,status", [
    (dict(quant=True), dict(paging=None), 1), (dict(quant=True), dict(n_seqs=65536), 5), (dict(quant=True), dict(kv_base=BASE), 2),
    (dict(paged=True), dict(kv_base=BASE), 2), (dict(paged=True), dict(L__dst_capacity=257), 2),
    (dict(quant=True), dict(L__head_dim=96), 5), (dict(paged=True), dict(pg__block_table=None), 1)])
def test_commit_refusals_of_forms(form, kw, status):
    assert pkv.pkv_tree_commit(**commit_args(**form, **kw)) == status


def test_commit_workspace():
    for quant in (0, 1):
        assert pkv.pkv_tree_commit_workspace_size(3, 5, quant) == 0


# ---- the binding ----------------------------------------------------------------

def test_binding_refuses_host_tensors():
    i, f = torch.zeros(4, dtype=torch.int32), torch.zeros(4)
    p = torch.zeros(4, 10)
    x = torch.zeros(1, 2, 4, 64)
    with pytest.raises(ValueError, match="parent is on cpu"):
        pkv.tree_masks(i, i)
    with pytest.raises(ValueError, match="q is on cpu"):
        pkv.tree_attention(x, x, x, x, x, x, i, i, 1.0, 4)
    with pytest.raises(ValueError, match="target_probs is on cpu"):
        pkv.tree_verify(p, i, i, f, f, 4)
    with pytest.raises(ValueError, match="draft_k is on cpu"):
        pkv.tree_commit(x, x, x, x, i, i, i)
    with pytest.raises(TypeError):
        pkv.tree_masks([0], i)


# ---- the references -------------------------------------------------------------

def test_reference_masks():
    seen = T.ancestors(np.array([-1, 0, 0, 2, 7]))
    assert seen.astype(int).tolist() == [[1, 0, 0, 0, 0], [1, 1, 0, 0, 0], [1, 0, 1, 0, 0], [1, 0, 1, 1, 0], [0, 0, 0, 0, 1]]
    big = np.zeros((1, 40), bool)
    big[0, [0, 31, 39]] = True
    assert T.pack(big, 2).tolist() == [[1 - 2 ** 31, 128]]


def test_reference_verify():
    """One drafted token of probability 1/4 where the draft had 1/2: accepted below u = 1/2, else the rest."""
    p, q = np.array([[0.25, 0.5, 0.25], [0.1, 0.2, 0.7]]), np.array([[0.5, 0.25, 0.25], [1.0, 0.0, 0.0]])
    args = ([9, 0], [-1, 0])
    assert T.verify(p, q, *args, [0, 0.49], 0.5, 4) == ([0, 1], 2)
    assert T.verify(p, q, *args, [0, 0.51], 0.5, 4) == ([0], 1)         # max(p - q, 0) has token 1 alone
    assert T.verify(p, None, *args, [0, 0.24], 0.0, 4) == ([0, 1], 0)
    assert T.verify(p, None, *args, [0, 0.26], 0.0, 4) == ([0], 1)       # without the tried token 0
    assert T.verify(p, None, *args, [0, 0.24], 0.0, 1) == ([0], 0)       # no room for another row
    assert T.verify(np.array([[0.0, np.nan]]), None, [0], [-1], [0], 0.5, 4) == ([0], -1)
