"""Shapes that the tensor-level splices and suffix attention refuse: a destination, value tensor or block table that is smaller than
what the call reads or writes by the sizes of the others.  On the CPU: the library's entry points are replaced, and only the
checks in front of them run."""
import pytest
import torch

from paper_2606_17107_amd import pkv

L, H, D, DV, N = 2, 3, 64, 128, 10


@pytest.fixture(autouse=True)
def calls(monkeypatch):
    calls = []
    monkeypatch.setattr(pkv, "_gpu_device", lambda t, name: t.device)
    for name in ("pkv_reposition_splice", "pkv_reposition_splice_freqs", "pkv_reposition_splice_paged", "pkv_reposition_splice_batched",
                 "pkv_suffix_attention", "pkv_suffix_attention_paged"):
        monkeypatch.setattr(pkv, name, lambda *a, **k: calls.append(a) or 0)
    return calls


def bf16(*shape):
    return torch.zeros(shape, dtype=torch.bfloat16)


def i32(*shape):
    return torch.zeros(shape, dtype=torch.int32)


def splice(src_v, dst_k, dst_v):
    pkv.reposition_splice(bf16(L, H, N, D), src_v, dst_k, dst_v, i32(N), i32(N), 1e4, 64)


def freqs(src_v, dst_k, dst_v):
    pkv.reposition_splice_freqs(bf16(L, H, N, D), src_v, dst_k, dst_v, i32(N), i32(N), [1.0] * 32, 64)


def batched(src_v, dst_k, dst_v):
    pkv.reposition_splice_batched(bf16(L, H, N, D), src_v, dst_k, dst_v, torch.zeros(64, dtype=torch.uint8), 1, N, 1e4, 64)


def paged(src_v, dst_k, dst_v, table=None, v_table=None):
    pkv.reposition_splice_paged(bf16(L, H, N, D), src_v, dst_k, dst_v, i32(N), i32(N), i32(1, 4) if table is None else table, 1e4, 64,
                                v_block_table=v_table)


def less(shape):
    """The shape with one size one smaller, each in turn."""
    for i in range(len(shape)):
        yield tuple(n - (j == i) for j, n in enumerate(shape))


SRC, CACHE, POOL = (L, H, N, DV), (L, H, 50), (L, 6, 32, H)


@pytest.mark.parametrize("call", [splice, freqs, batched])
def test_splices(call, calls):
    call(bf16(*SRC), bf16(*CACHE, D), bf16(*CACHE, DV))
    call(bf16(*SRC), bf16(L + 1, H + 1, 50, D + 8), bf16(L + 1, H + 2, 60, DV + 8))
    call(None, bf16(*CACHE, D), None)
    assert len(calls) == 3
    for shape in less(SRC[:3]):
        with pytest.raises(ValueError, match="src_v"):
            call(bf16(*shape, DV), bf16(*CACHE, D), bf16(*CACHE, DV))
    for shape in ((L - 1, H, 50, D), (L, H - 1, 50, D), (L, H, 50, D - 1)):
        with pytest.raises(ValueError, match="dst_k"):
            call(bf16(*SRC), bf16(*shape), bf16(*CACHE, DV))
    for shape in less(CACHE + (DV,)):
        with pytest.raises(ValueError, match="dst_v"):
            call(bf16(*SRC), bf16(*CACHE, D), bf16(*shape))
    assert len(calls) == 3


def test_paged_splice(calls):
    paged(bf16(*SRC), bf16(*POOL, D), bf16(*POOL, DV))
    paged(None, bf16(*POOL, D), None)
    assert len(calls) == 2
    for shape in ((L - 1, 6, 32, H, D), (L, 6, 32, H - 1, D), (L, 6, 32, H, D - 1)):
        with pytest.raises(ValueError, match="dst_k"):
            paged(bf16(*SRC), bf16(*shape), bf16(*POOL, DV))
    for shape in less(POOL + (DV,)):
        with pytest.raises(ValueError, match="dst_v"):
            paged(bf16(*SRC), bf16(*POOL, D), bf16(*shape))
    for table, v_table in ((i32(0, 4), None), (i32(4), None), (i32(1, 4), i32(1, 3))):
        with pytest.raises(ValueError, match="block_table"):
            paged(bf16(*SRC), bf16(*POOL, D), bf16(*POOL, DV), table, v_table)
    assert len(calls) == 2


def attend(k, v, out=None, table=None, v_table=None, n_seqs=2):
    """Four query heads a KV head."""
    q = bf16(L, N, 4 * H, D)
    out = bf16(L, N, 4 * H, D) if out is None else out
    args = (q, k, v, out, i32(N), i32(2))
    if k.dim() == 5:
        pkv.suffix_attention_paged(*args, i32(2, 4) if table is None else table, 1.0, 0, n_seqs=n_seqs, cu_q=i32(3), v_block_table=v_table)
    else:
        pkv.suffix_attention(*args, 1.0, 0, n_seqs=n_seqs, cu_q=i32(3))


@pytest.mark.parametrize("cache", [CACHE, POOL])
def test_attention(cache, calls):
    full = cache + (D,)
    attend(bf16(*full), bf16(*full))
    attend(bf16(*full), bf16(*(n + 1 for n in cache), D))
    assert len(calls) == 2
    for shape in less(full):
        with pytest.raises(ValueError, match="v_cache"):
            attend(bf16(*full), bf16(*shape))
    for shape in ((L - 1,) + full[1:], full[:-1] + (D - 1,)):
        with pytest.raises(ValueError, match="k_cache"):
            attend(bf16(*shape), bf16(*full))
    for shape in less((L, N, 4 * H)):
        with pytest.raises(ValueError, match="out"):
            attend(bf16(*full), bf16(*full), bf16(*shape, D))
    assert len(calls) == 2


def test_attention_tables(calls):
    k = bf16(*POOL, D)
    attend(k, k, table=i32(3, 4))
    for table, v_table in ((i32(1, 4), None), (i32(8), None), (i32(2, 4), i32(2, 3))):
        with pytest.raises(ValueError, match="block_table"):
            attend(k, k, table=table, v_table=v_table)
    assert len(calls) == 1


def test_latent_rows(calls):
    k = bf16(L, 1, 50, 576)
    q, out = bf16(L, N, 16, 576), bf16(L, N, 16, 512)
    pkv.suffix_attention(q, k, k, out, i32(N), i32(2), 1.0, 0, n_seqs=2, cu_q=i32(3), variant=pkv.PKV_ATTN_MLA)
    assert len(calls) == 1
