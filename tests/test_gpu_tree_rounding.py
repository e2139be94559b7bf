"""What a sequence's result depends on beside its own rows: sizes of the call, for which only the rounding may change."""
import pytest
import torch

from test_gpu_tree_attention import Case, same

pytestmark = pytest.mark.gpu

KINDS = ["bf16", "f32", "paged", "quant", "mla", "mla_paged"]


def pad(c, extra):
    """`extra` rows more, that no sequence owns, behind the case's own."""
    for name, dim in (("q", 1), ("dk", 2), ("dv_rows", 2)):
        t = getattr(c, name)
        more = torch.full([extra if i == dim else n for i, n in enumerate(t.shape)], 3.0, dtype=t.dtype, device="cuda")
        setattr(c, name, torch.cat([t, more], dim))
    if c.mla:
        c.dv_rows = c.dk
    c.pos = torch.cat([torch.from_numpy(c.pos), torch.zeros(extra, dtype=torch.int32)]).numpy()
    c.rows += extra


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("lens,sizes", [([2000], [32]), ([1500, 90, 700], [9, 4, 30])])
def test_rows_of_no_sequence(kind, lens, sizes):
    """They count among the call's rows, by which the library cuts the keys; with the splits given nothing follows them."""
    c = Case(kind, lens, sizes, seed=70)
    own = c.rows
    given, given_lse = c.call(c.masks(), 3)
    c.check(given, given_lse)
    c.check(*c.call(c.masks()))
    pad(c, 4000)
    out, lse = c.call(c.masks(), 3)
    assert same(out.t[:, :own], given.t[:, :own]) and same(lse[:, :own], given_lse[:, :own])
    for splits in (3, 0):
        out, lse = c.call(c.masks(), splits)
        c.check(out, lse)
        assert out.untouched((slice(None), slice(own, None))) and bool((lse[:, own:] == 7.0).all())
        again, _ = c.call(c.masks(), splits)
        assert same(out.t, again.t)


@pytest.mark.parametrize("kind", KINDS)
def test_lengths_of_others(kind):
    """With the splits given a sequence's result does not follow the other sequences' lengths."""
    c = Case(kind, [900, 800, 64], [9, 14, 5], seed=71)
    want, _ = c.call(c.masks(), 4)
    c.lens[0], c.lens[2] = 17, 0
    c.pos[:9] -= 900 - 17
    c.pos[23:] -= 64
    out, lse = c.call(c.masks(), 4, max_kv=900)
    c.check(out, lse)
    assert same(out.t[:, 9:23], want.t[:, 9:23])
