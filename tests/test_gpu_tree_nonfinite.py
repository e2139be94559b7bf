"""Values of drafted rows that are no finite numbers behind weights that vanish: the weight is above 0 by definition, so the
channel of a row that sees one is NaN or infinite, in the join of one wave a row and head and in the join in tiles alike; a score of
-inf alone weighs nothing."""
import math

import pytest

from test_gpu_tree_attention import Case, Wide, same

pytestmark = pytest.mark.gpu

CHANNEL, ROW = 9, 4


def plant(c, s, seers, key, value):
    """Row ROW of tree s is seen by `seers` alone; its score is `key` times the scale, one of its values `value`."""
    c.seen[s][:, ROW] = False
    c.seen[s][seers, ROW] = True
    c.q[..., 0] = 1.0
    at = int(c.cu[s]) + ROW
    c.dk[:, :, at] = 0.0
    c.dk[:, :, at, 0] = key
    c.dv_rows[:, :, at] = 0.25
    c.dv_rows[:, :, at, CHANNEL] = value
    return at


def with_a_finite_value(c, at):
    c.dv_rows[:, :, at, CHANNEL] = 0.25
    return c.call(c.masks())[0]


def cases():
    for kind in ("bf16", "f32", "paged", "quant"):
        yield lambda kind=kind: (Case(kind, [100, 40], [6, 12], seed=51), 1, [5, 7, 9])
    for d in (64, 128):
        yield lambda d=d: (Wide("bf16", 52 + d, d), 3, [7, 9])
    yield lambda: (Wide("quant", 53), 3, [7, 9])


@pytest.mark.parametrize("make", cases())
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_vanished_weight(make, bad):
    c, s, seers = make()
    # exp(-30000 / 12) is 0 in 32 bits; a row's other scores are below 40 in size
    at = plant(c, s, seers, -30000.0, bad)
    out, lse = c.call(c.masks())
    assert bool(lse[:, :int(c.cu[-1])].isfinite().all())
    rows = [int(c.cu[s]) + i for i in seers]
    assert not bool(out.t[:, rows, :, CHANNEL].isfinite().any())
    clean = with_a_finite_value(c, at)
    rest = [r for r in range(int(c.cu[-1])) if r not in rows]
    assert same(out.t[:, rest], clean.t[:, rest])
    channels = [x for x in range(c.d) if x != CHANNEL]
    assert same(out.t[:, rows][..., channels], clean.t[:, rows][..., channels])
    assert bool(clean.t[:, rows].isfinite().all())


@pytest.mark.parametrize("make", cases())
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_score_of_minus_infinity(make, bad):
    c, s, seers = make()
    at = plant(c, s, seers, -math.inf, bad)
    out, lse = c.call(c.masks())
    clean = with_a_finite_value(c, at)
    n = int(c.cu[-1])
    assert bool(out.t[:, :n].isfinite().all()) and bool(lse[:, :n].isfinite().all())
    assert same(out.t[:, :n], clean.t[:, :n])


@pytest.mark.parametrize("make", cases())
def test_infinite_value_with_a_weight(make):
    c, s, seers = make()
    at = plant(c, s, seers, 0.0, math.inf)
    out, _ = c.call(c.masks())
    rows = [int(c.cu[s]) + i for i in seers]
    assert bool((out.t[:, rows, :, CHANNEL] == math.inf).all())
    x = out.t[:, :int(c.cu[-1])].clone()
    x[:, rows, :, CHANNEL] = 0
    assert bool(x.isfinite().all())
