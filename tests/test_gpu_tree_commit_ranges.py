"""Commits at the ends of their range: no drafted rows, a cache without slots, rows, lengths and page entries out of range.  Nothing
is written that is not accepted (codes and scale bytes), and whatever is accepted and cannot be written is flagged."""
import numpy as np
import pytest
import torch

import tree_ref as T
from paper_2606_17107_amd import pkv
from test_gpu_tree_commit import Case, quant_reference

pytestmark = pytest.mark.gpu

KINDS = ["contiguous", "paged", "quant"]


def tensors(c):
    return [t for t in (c.k, c.v, c.ks, c.vs) if t is not None]


def unchanged(c, before):
    return all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(tensors(c), before))


def flag():
    return torch.zeros(1, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("accepted", [True, False])
@pytest.mark.parametrize("field", ["dst_capacity", "n_tokens"])
def test_nothing_to_take_or_to_fill(kind, accepted, field):
    """A capacity of 0, or no drafted rows: every accepted row is out of range."""
    c = Case(kind, [0, 0], [3, 2], seed=31)
    before = [t.clone() for t in tensors(c)]
    f = flag()
    table = None if c.table is None else T.as_tensor(c.table)
    layout = pkv.make_commit_layout(c.dk, c.dv, c.k, c.v, table, c.k.shape[2] if table is None else 0, f)
    setattr(layout, field, 0)
    paging = None if table is None else pkv.make_paging(table, c.k, c.v)
    scales = pkv.make_block_scales(c.ks, c.vs, c.k.shape[2]) if kind == "quant" else None
    counts = T.as_tensor(c.counts if accepted else np.zeros(2, np.int32))
    assert pkv.pkv_tree_commit(c.dk, c.dv, c.k, c.v, T.as_tensor(c.path), counts, T.as_tensor(c.lens), None, 2, c.P, layout, paging,
                               scales, None, 0) == pkv.PKV_OK
    torch.cuda.synchronize()
    assert unchanged(c, before) and int(f) == int(accepted)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("values", [True, False])
@pytest.mark.parametrize("accepted", [True, False])
def test_no_drafted_rows(kind, values, accepted):
    """A step in which no sequence has rows, whose tensors have no address; a path that names rows all the same is flagged."""
    c = Case(kind, [10, 20], [3, 2], values=values, seed=30)
    before = [t.clone() for t in tensors(c)]
    c.dk = c.dk[:, :, :0]
    c.dv = c.dv[:, :, :0] if values else None
    f = flag()
    c.call(f, counts=None if accepted else np.zeros(2, np.int32))
    assert unchanged(c, before) and int(f) == int(accepted)
    c.dk = torch.empty_like(c.dk)
    c.dv = torch.empty_like(c.dv) if values else None
    assert c.dk.data_ptr() == 0
    c.call(f.zero_(), counts=None if accepted else np.zeros(2, np.int32))
    assert unchanged(c, before) and int(f) == int(accepted)


@pytest.mark.parametrize("kind", KINDS)
def test_nothing_accepted(kind):
    c = Case(kind, [10, 20], [3, 2], seed=32)
    before = [t.clone() for t in tensors(c)]
    f = flag()
    c.call(f, counts=np.array([0, -4], np.int32))
    assert unchanged(c, before) and int(f) == 0


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("length", [2 ** 31 - 2, 2 ** 30, 2 ** 20, -1, -500, -2 ** 31])
def test_lengths_out_of_range(kind, length):
    """One sequence's slots lie behind the capacity or before 0: nothing of it is written, the others are."""
    c = Case(kind, [10, 20, 40], [4, 4, 4], seed=33)
    lens = c.lens.copy()
    lens[1] = length
    good = [p for p in c.pairs() if p[0] != 1]
    if kind == "quant":
        want = quant_reference(c, [(row, s, 1, slot, slot) for s, slot, row in good], c.lens)
        want = [T.as_tensor(a) for a in (want[0][0], want[1][0], want[0][1], want[1][1])]
    else:
        want = c.expected(good)
    if kind == "contiguous":
        c.base[1] = 0
    f = flag()
    c.call(f, lens=lens)
    assert unchanged(c, want) and int(f) == 1


@pytest.mark.parametrize("page,block", [(32, 32), (64, 32), (128, 128)])
def test_codes_and_scales_beside_rows_out_of_range(page, block):
    """Rows of the path that do not exist leave their slots, and do not enter a block's scale; a block that gets none keeps its byte."""
    c = Case("quant", [10, 20, 40, 31], [4, 4, 4, 3], nodes=9, page=page, block=block, seed=34)
    path = c.path.copy()
    path[0, 1], path[1, 2], path[2, :4], path[3, 1] = 36, -1, 2 ** 31 - 1, -2 ** 31
    counts = np.array([4, 9, 4, 3], np.int32)
    good = [p for p in c.pairs(path, counts) if 0 <= p[2] < 36]
    want = quant_reference(c, [(row, s, 1, slot, slot) for s, slot, row in good], c.lens)
    f = flag()
    c.call(f, path, counts)
    assert unchanged(c, [T.as_tensor(a) for a in (want[0][0], want[1][0], want[0][1], want[1][1])]) and int(f) == 1


@pytest.mark.parametrize("kind", ["paged", "quant"])
@pytest.mark.parametrize("values", [True, False])
def test_page_entries_out_of_range(kind, values):
    """Codes, slots and scale bytes of page 0, which stands in for a page that is none, stay as they were."""
    c = Case(kind, [10, 20, 40], [4, 4, 4], values=values, seed=35)
    c.table[:, 0] = [-1, 10 ** 6, -5]
    c.table[:, 1] = [-1, c.k.shape[1], -2 ** 31]
    before = [t.clone() for t in tensors(c)]
    f = flag()
    c.call(f)
    assert unchanged(c, before) and int(f) == 1
