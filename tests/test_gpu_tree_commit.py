"""Accepted rows appended to caches of every kind: copies bit for bit, codes as the quantising splice stores them; nothing else
is written."""
import numpy as np
import pytest
import torch

import quant_ref as R
import tree_ref as T
from paper_2606_17107_amd import pkv

pytestmark = pytest.mark.gpu


def bits(t):
    return t.contiguous().view(torch.uint8).cpu().numpy()


class Case:
    """Trees of `nodes` rows behind contexts of `lens` slots; counts[s] rows of each are accepted."""

    def __init__(self, kind, lens, counts, nodes=9, L=2, H=2, d=64, page=32, block=32, source=torch.bfloat16, values=True, seed=0,
                 max_path=None):
        self.rng = rng = np.random.default_rng(seed)
        self.kind, self.lens, self.counts, self.values = kind, np.array(lens, np.int32), np.array(counts, np.int32), values
        S = len(lens)
        self.P = max(1, max(counts)) if max_path is None else max_path
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        normal = lambda *shape: torch.empty(shape, device="cuda").normal_(generator=g)   # noqa: E731
        rows = S * nodes
        self.dk = normal(L, rows, H, d).to(source).transpose(1, 2)
        self.dv = normal(L, rows, H, d).to(source).transpose(1, 2) if values else None
        self.path = np.full((S, self.P), -1, np.int32)
        for s, n in enumerate(counts):
            picked = [0] + sorted(rng.choice(np.arange(1, nodes), n - 1, replace=False)) if n else []
            self.path[s, :n] = [s * nodes + r for r in picked]
        most = int(max(lens)) + self.P
        self.base = self.table = self.ks = self.vs = None
        if kind == "contiguous":
            self.k = normal(L, H, S * most + 3, d).to(source)
            self.v = normal(L, H, S * most + 3, d).to(source) if values else None
            self.base = rng.permutation(S).astype(np.int64) * most
        else:
            width = -(-most // page)
            pages = S * width + 3
            self.table = rng.permutation(pages)[:S * width].reshape(S, width).astype(np.int32)
            shape = (L, pages, page, H, d)
            if kind == "quant":
                self.k, self.v = (T.as_tensor(rng.integers(0, 256, shape).astype(np.uint8)) for _ in "kv")
                for t in (self.k, self.v):
                    t[(t & 127) == 127] = 3
                scales = (L, pages, page // block, H)
                self.ks, self.vs = (T.as_tensor(rng.integers(110, 125, scales).astype(np.uint8)) for _ in "kv")
                if not values:
                    self.v = self.vs = None
            else:
                self.k = normal(*shape).to(source)
                self.v = normal(*shape).to(source) if values else None
        self.page, self.block = page, block

    def call(self, flag=None, path=None, counts=None, lens=None, **kw):
        tables = {} if self.table is None else dict(block_table=T.as_tensor(self.table))
        pkv.tree_commit(self.dk, self.dv, self.k, self.v, T.as_tensor(self.path if path is None else path),
                        T.as_tensor(self.counts if counts is None else counts), T.as_tensor(self.lens if lens is None else lens),
                        kv_base=None if self.base is None else T.as_tensor(self.base), k_scale=self.ks, v_scale=self.vs, err_flag=flag,
                        **tables, **kw)
        torch.cuda.synchronize()

    def pairs(self, path=None, counts=None, lens=None):
        """(sequence, slot, row) of every accepted row."""
        path, counts, lens = (b if a is None else a for a, b in ((path, self.path), (counts, self.counts), (lens, self.lens)))
        return [(s, int(lens[s]) + i, int(path[s, i])) for s in range(len(counts)) for i in range(min(int(counts[s]), path.shape[1]))]

    def expected(self, pairs):
        out = []
        for t, new in ((self.k, self.dk), (self.v, self.dv)):
            if t is None:
                continue
            t = t.clone()
            for s, slot, row in pairs:
                if self.table is None:
                    t[:, :, int(self.base[s]) + slot] = new[:, :, row]
                else:
                    t[:, int(self.table[s, slot // self.page]), slot % self.page] = new[:, :, row]
            out.append(t)
        return out

    def check(self, want):
        for t, w in zip([t for t in (self.k, self.v) if t is not None], want):
            np.testing.assert_array_equal(bits(t), bits(w))


@pytest.mark.parametrize("kind", ["contiguous", "paged"])
@pytest.mark.parametrize("source", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("values", [True, False])
def test_copies(kind, source, values):
    for seed, (L, H, d) in enumerate([(1, 1, 64), (3, 2, 128), (2, 8, 64), (5, 1, 576)]):
        c = Case(kind, [0, 31, 30, 100, 64], [1, 4, 9, 0, 3], L=L, H=H, d=d, source=source, values=values, seed=seed)
        want = c.expected(c.pairs())
        c.call()
        c.check(want)


def quant_reference(c, segs, lens):
    out = []
    for new, pool, scale in ((c.dk, c.k, c.ks), (c.dv, c.v, c.vs)):
        if new is not None:
            out.append(R.store(new.double().cpu().numpy(), pool.cpu().numpy(), scale.cpu().numpy(), segs, lens, c.table, np.zeros(8), 0, 0,
                               c.table.shape[1] * c.page, False)[:2])
    return out


@pytest.mark.parametrize("source", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("page,block,d", [(32, 32, 64), (64, 32, 128), (128, 128, 64)])
def test_codes(source, page, block, d):
    """As the splice's definition says, byte for byte: blocks begun, continued and crossed."""
    for values in (True, False):
        c = Case("quant", [0, 31, 30, 127, 64, 5], [1, 4, 9, 3, 0, 2], L=2, d=d, page=page, block=block, source=source, values=values,
                 seed=page + d)
        want = quant_reference(c, [(row, s, 1, slot, slot) for s, slot, row in c.pairs()], c.lens)
        c.call()
        for (pool, scale), t, e in zip(want, (c.k, c.v), (c.ks, c.vs)):
            np.testing.assert_array_equal(t.cpu().numpy(), pool)
            np.testing.assert_array_equal(e.cpu().numpy(), scale)


@pytest.mark.parametrize("kind", ["contiguous", "paged", "quant"])
def test_nothing_accepted(kind):
    c = Case(kind, [10, 20], [3, 2], seed=5)
    before = [t.clone() for t in (c.k, c.v)]
    c.call(counts=np.array([0, -4], np.int32))
    c.check(before)


@pytest.mark.parametrize("kind", ["contiguous", "paged", "quant"])
def test_out_of_range(kind):
    """Rows, slots and page entries out of range are skipped and flagged; the others are written.  Counts above the path's
    length stop at it."""
    flag = torch.zeros(1, dtype=torch.int32, device="cuda")
    c = Case(kind, [10, 20, 40], [4, 4, 4], seed=6)
    path = c.path.copy()
    path[0, 1], path[1, 2] = 27, -1
    good = [p for p in c.pairs(path) if 0 <= p[2] < 27]
    counts = np.array([4, 9, 4], np.int32)
    if kind == "quant":
        want = quant_reference(c, [(row, s, 1, slot, slot) for s, slot, row in good], c.lens)
        want = [w[0] for w in want]
    else:
        want = c.expected(good)
    c.call(flag, path, counts)
    if kind == "quant":
        for t, w in zip((c.k, c.v), want):
            np.testing.assert_array_equal(t.cpu().numpy(), w)
    else:
        c.check(want)
    assert int(flag) == 1
    # slots behind the capacity, before 0, and far away
    c = Case(kind, [10, 20, 40], [4, 4, 4], seed=7)
    flag.zero_()
    before = [t.clone() for t in (c.k, c.v)]
    far = np.array([2 ** 31 - 2, -1, -2 ** 31], np.int32) if kind != "contiguous" else np.array([2 ** 31 - 2, -500, 2 ** 30], np.int32)
    if kind == "contiguous":
        c.base[:] = 0
    c.call(flag, lens=far)
    if kind == "paged" or kind == "contiguous":
        c.check(before)
        assert int(flag) == 1
    # a page entry outside the pool
    if kind != "contiguous":
        c = Case(kind, [10, 20, 40], [4, 4, 4], seed=8)
        flag.zero_()
        c.table[:, 0] = [-1, 10 ** 6, -5]
        c.table[:, 1] = -1
        before = [t.clone() for t in (c.k, c.v)]
        c.call(flag)
        c.check(before)
        assert int(flag) == 1


def test_value_pages_of_their_own():
    for kind in ("paged", "quant"):
        c = Case(kind, [10, 31], [4, 4], seed=9)
        other = Case(kind, [10, 31], [4, 4], seed=9)
        perm = torch.randperm(c.k.shape[1], generator=torch.Generator().manual_seed(1)).cuda()
        for t in ("v", "vs"):
            if getattr(c, t) is not None:
                moved = torch.empty_like(getattr(c, t))
                moved[:, perm] = getattr(c, t)
                setattr(c, t, moved)
        c.call(v_block_table=perm[T.as_tensor(c.table).long()].to(torch.int32).contiguous())
        other.call()
        assert torch.equal(c.k, other.k) and torch.equal(c.v[:, perm], other.v)


def test_offsets_past_32_bits():
    """Layers of the cache and of the drafted rows more than 2^32 bytes apart."""
    c = Case("contiguous", [3, 8], [2, 3], seed=10)
    want = c.expected(c.pairs())
    far = 2 ** 31 + 64
    for name in ("k", "dk"):
        t = getattr(c, name)
        buf = torch.empty(far + t.numel(), dtype=t.dtype, device="cuda")
        x = torch.as_strided(buf, t.shape, (far, t.shape[2] * t.shape[3], t.shape[3], 1))
        x.copy_(t)
        setattr(c, name, x)
    c.call()
    c.check(want)


def test_many_sequences():
    n = 65540
    c = Case("contiguous", [1] * n, [2] * n, nodes=2, L=1, H=1, d=64, seed=11)
    c.call()
    at = T.as_tensor(c.base)
    for i in range(2):
        assert torch.equal(c.k[0, 0, at + 1 + i], c.dk[0, 0, T.as_tensor(c.path[:, i]).long()])


def test_refusals_of_the_binding():
    c = Case("paged", [3, 8], [2, 3], seed=12)
    with pytest.raises(ValueError, match="both or not"):
        pkv.tree_commit(c.dk, None, c.k, c.v, T.as_tensor(c.path), T.as_tensor(c.counts), T.as_tensor(c.lens), block_table=T.as_tensor(c.table))
    with pytest.raises(ValueError, match="does not fit"):
        pkv.tree_commit(c.dk[..., :32], c.dv[..., :32], c.k, c.v, T.as_tensor(c.path), T.as_tensor(c.counts), T.as_tensor(c.lens),
                        block_table=T.as_tensor(c.table))
    with pytest.raises(ValueError, match="block_table"):
        pkv.tree_commit(c.dk, c.dv, c.k, c.v, T.as_tensor(c.path), T.as_tensor(c.counts), T.as_tensor(c.lens),
                        block_table=T.as_tensor(c.table[:1]))
    with pytest.raises(TypeError, match="kv_len"):
        pkv.tree_commit(c.dk, c.dv, c.k, c.v, T.as_tensor(c.path), T.as_tensor(c.counts), T.as_tensor(c.lens).long(),
                        block_table=T.as_tensor(c.table))
