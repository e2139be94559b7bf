"""Shapes that the tensor-level calls on trees refuse: the library takes its bounds from the key cache, so a value cache with fewer
slots, pages or heads, or more slots than there are, would be read or written past its end.  On the CPU: the library's entry points
are replaced, and only the checks in front of them run."""
import contextlib

import pytest
import torch

from paper_2606_17107_amd import pkv


@pytest.fixture(autouse=True)
def stand_ins(monkeypatch):
    monkeypatch.setattr(torch.cuda, "device", lambda d: contextlib.nullcontext())
    monkeypatch.setattr(pkv, "_gpu_device", lambda t, name: t.device)
    calls = []
    for name in ("pkv_tree_attention", "pkv_tree_commit"):
        monkeypatch.setattr(pkv, name, lambda *a, **k: calls.append(a) or 0)
    return calls


L, H, D, ROWS = 2, 4, 64, 6


def i32(*shape):
    return torch.zeros(shape, dtype=torch.int32)


def pool(pages, page, heads=H, kind="paged"):
    return torch.zeros((L, pages, page, heads, D), dtype=torch.uint8 if kind == "quant" else torch.bfloat16)


def cache(slots, heads=H):
    return torch.zeros((L, heads, slots, D), dtype=torch.bfloat16)


def attend(k, v, heads=H, **kw):
    q, x = torch.zeros(L, ROWS, heads, D, dtype=torch.bfloat16), torch.zeros(L, heads, ROWS, D, dtype=torch.bfloat16)
    pkv.tree_attention(q, k, v, x, x.clone(), q.clone(), i32(ROWS), i32(2), 1.0, 50, n_seqs=2, cu_q=i32(3), **kw)


def commit(k, v, heads=H, **kw):
    x = torch.zeros(L, heads, ROWS, D, dtype=torch.bfloat16)
    pkv.tree_commit(x, None if v is None else x.clone(), k, v, i32(2, 3), i32(2), i32(2), **kw)


CALLS = [attend, commit]
TABLE = i32(2, 4)


@pytest.mark.parametrize("call", CALLS)
def test_values_as_large_as_keys_or_larger(call, stand_ins):
    call(cache(90), cache(90))
    call(cache(90), cache(95))
    call(pool(9, 32), pool(9, 32), block_table=TABLE)
    call(pool(9, 32), pool(12, 32), block_table=TABLE, v_block_table=TABLE.clone())
    assert len(stand_ins) == 4


@pytest.mark.parametrize("call", CALLS)
def test_value_caches_with_fewer_slots(call, stand_ins):
    for slots in (89, 1, 0):
        with pytest.raises(ValueError, match="value cache has %d slots" % slots):
            call(cache(90), cache(slots))
    assert not stand_ins


@pytest.mark.parametrize("call", CALLS)
def test_value_pools_with_fewer_or_smaller_pages(call, stand_ins):
    for pages, page in ((8, 32), (9, 64), (18, 16), (1, 32)):
        with pytest.raises(ValueError, match="value pool has %d pages of %d slots" % (pages, page)):
            call(pool(9, 32), pool(pages, page), block_table=TABLE)
    assert not stand_ins


@pytest.mark.parametrize("call", CALLS)
def test_values_with_other_heads(call, stand_ins):
    with pytest.raises(ValueError):
        call(cache(90), cache(90, H - 1))
    with pytest.raises(ValueError):
        call(pool(9, 32), pool(9, 32, H - 1), block_table=TABLE)
    assert not stand_ins


@pytest.mark.parametrize("call", CALLS)
def test_value_tables_of_another_shape(call, stand_ins):
    for other in (i32(2, 3), i32(1, 4), i32(8)):
        with pytest.raises(ValueError, match="different shapes"):
            call(pool(9, 32), pool(9, 32), block_table=TABLE, v_block_table=other)
    assert not stand_ins


def test_more_slots_than_there_are(stand_ins):
    with pytest.raises(ValueError, match="91 slots, the caches have 90"):
        commit(cache(90), cache(90), slots=91)
    with pytest.raises(ValueError, match="91 slots, the caches have 90"):
        commit(cache(90), None, slots=91)
    with pytest.raises(ValueError, match="91 slots, the caches have 90"):
        attend(cache(90), cache(90), cache_slots=91)
    commit(cache(90), cache(90), slots=90)
    attend(cache(90), cache(90), cache_slots=30)
    assert len(stand_ins) == 2


@pytest.mark.parametrize("call", CALLS)
def test_pools_of_codes(call, stand_ins):
    """As before: one shape for both."""
    scale = torch.zeros(L, 9, 1, H, dtype=torch.uint8)
    with pytest.raises(ValueError, match="different shapes"):
        call(pool(9, 32, kind="quant"), pool(8, 32, kind="quant"), block_table=TABLE, k_scale=scale, v_scale=scale[:, :8])
    call(pool(9, 32, kind="quant"), pool(9, 32, kind="quant"), block_table=TABLE, k_scale=scale, v_scale=scale)
    assert len(stand_ins) == 1


@pytest.mark.skipif(torch.cuda.is_available(), reason="fake device addresses, so only without a GPU")
@pytest.mark.parametrize("form", [dict(), dict(paged=True), dict(quant=True)])
@pytest.mark.parametrize("v_dim", [128, 0])
def test_commit_without_drafted_rows_needs_no_tensors_of_them(form, v_dim, monkeypatch):
    """Past the checks, to the launch that there is no device for; with rows a missing tensor is refused as ever."""
    from test_tree_abi import commit_args
    monkeypatch.undo()
    values = {} if v_dim else dict(cache_v=None)
    a = commit_args(**form, draft_k=None, draft_v=None, L__v_dim=v_dim, L__n_tokens=0, **values)
    if not v_dim and a["scales"] is not None:
        a["scales"].v_scale = None
    assert pkv.pkv_tree_commit(**a) == pkv.PKV_ERR_DEVICE
    a["layout"].n_tokens = 1
    assert pkv.pkv_tree_commit(**a) == pkv.PKV_ERR_NULL
