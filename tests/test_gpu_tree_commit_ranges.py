"""Commits at the ends of their range: no drafted rows, a cache without slots, rows, lengths and page entries out of range.  Nothing
is written that is not accepted (codes and scale bytes), and whatever is accepted and cannot be written is flagged."""
import numpy as np
import pytest
import torch

import tree_ref as T
from paper_2606_17107_amd import pkv
from test_gpu_tree_commit import Case

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
