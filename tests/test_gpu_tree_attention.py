"""Attention of trees of drafted tokens against a 64-bit reference on the values that the caches hold.

Tolerances.  bf16: as for the bf16 kernels, probabilities over the cache and outputs are each rounded to bf16 (half a step,
2^-9 relative to a weight, on average; rel-L2 below 1e-2, and for values of unit size max-abs 2e-2, mean-abs 2e-3).  fp32: a
score is a sum of 128 products of |q||k| about 1.5 in mean square, of size up to 10 after the scale; its rounding is below
130 * 2^-24 * 128 * 1.5 / sqrt(128) = 1.3e-4, so a weight is off by that much of itself at worst, an output by twice as much of
the largest value (about 5): 1.3e-3 at most, rel-L2 below 2.6e-4."""
import math

import numpy as np
import pytest
import torch

import quant_ref as R
import tree_ref as T
from helpers import Guarded, check_attention_close, host_bits, log
from paper_2606_17107_amd import pkv

pytestmark = pytest.mark.gpu

KINDS = ["bf16", "f32", "paged", "quant", "mla", "mla_paged"]


def same(a, b):
    """Equal bit for bit."""
    return torch.equal(a.contiguous().view(torch.uint8), b.contiguous().view(torch.uint8))


class Case:
    """Caches of `lens` slots and trees of `sizes` rows behind them, with every slot and row of the tensors filled."""

    def __init__(self, kind, lens, sizes, G=4, Hkv=2, d=128, L=1, ways=2, seed=0, page=64, block=32, extra_rows=0, gap=0, gain=1.5):
        self.rng = rng = np.random.default_rng(seed)
        self.kind, self.lens, self.sizes, self.L = kind, list(lens), list(sizes), L
        self.mla = kind.startswith("mla")
        if self.mla:
            Hkv, d, G = 1, 576, G * 4
        self.Hkv, self.d, self.dv, self.H = Hkv, d, 512 if self.mla else d, Hkv * G
        self.scale = 1 / math.sqrt(192 if self.mla else d)
        self.dtype = torch.float32 if kind == "f32" else torch.bfloat16
        g = torch.Generator(device="cuda")
        g.manual_seed(seed + 1)
        normal = lambda *shape: torch.empty(shape, device="cuda").normal_(generator=g).to(self.dtype)   # noqa: E731
        S, most = len(lens), max(1, max(lens))
        self.table = self.base = self.ks = self.vs = None
        if kind in ("paged", "quant", "mla_paged"):
            width = -(-most // page)
            P = S * width + 3
            self.table = T.as_tensor(rng.permutation(P)[:S * width].reshape(S, width).astype(np.int32))
            if kind == "quant":
                shape = (L, P, page // block, Hkv)
                ks, vs = (rng.integers(119, 123, shape).astype(np.uint8) for _ in "kv")
                self.ks, self.vs = T.as_tensor(ks), T.as_tensor(vs)
                fill = lambda e: (normal(L, P, page, Hkv, d).float()   # noqa: E731
                                  * torch.exp2(127.0 - e.float()).repeat_interleave(block, 2)[..., None]).clamp(-448, 448)
                self.k, self.v = (fill(e).to(torch.float8_e4m3fn).view(torch.uint8) for e in (self.ks, self.vs))
            else:
                self.k = normal(L, P, page, Hkv, d)
                self.v = self.k if self.mla else normal(L, P, page, Hkv, d)
        else:
            self.k = normal(L, Hkv, S * most + 5, d)
            self.v = self.k if self.mla else normal(L, Hkv, S * most + 5, d)
            self.base = T.as_tensor(rng.permutation(S).astype(np.int64) * most)
        self.starts = np.cumsum([gap] + [n + gap for n in sizes])[:-1] if gap else np.cumsum([0] + list(sizes))[:-1]
        self.cu = np.concatenate([self.starts, [self.starts[-1] + sizes[-1]]]).astype(np.int32)
        assert not gap or len(sizes) == 1, "rows in front of the first sequence only"
        self.rows = rows = int(self.cu[-1]) + extra_rows
        self.q = (normal(L, rows, self.H, d).float() * gain).to(self.dtype)
        self.dk = normal(L, rows, Hkv, d).transpose(1, 2)     # as a projection leaves them
        self.dv_rows = self.dk if self.mla else normal(L, rows, Hkv, d).transpose(1, 2)
        self.parents = [T.random_tree(rng, n, ways) for n in sizes]
        self.seen = [T.ancestors(p) for p in self.parents]
        self.pos = np.zeros(rows, np.int32)
        for s, seen in enumerate(self.seen):
            self.pos[self.cu[s]:self.cu[s] + sizes[s]] = lens[s] + seen.sum(1) - 1
        self.words = max(1, -(-max(sizes) // 32))

    def masks(self):
        m = np.full((self.rows, self.words), -1, np.int32)      # rows that no sequence owns: any bits
        for s, seen in enumerate(self.seen):
            m[self.cu[s]:self.cu[s] + self.sizes[s]] = T.pack(seen, self.words)
        return T.as_tensor(m)

    def call(self, mask, splits=0, window=0, max_kv=None, max_q=None, stream=None, guard=True, **kw):
        shape = (self.L, self.rows, self.H, self.dv)
        out = Guarded(shape, self.dtype)
        lse = torch.full(shape[:3], 7.0, device="cuda")
        max_kv = max(self.lens) if max_kv is None else max_kv
        most = max(self.sizes) if max_q is None else max_q
        variant = pkv.PKV_ATTN_MLA if self.mla else pkv.PKV_ATTN_GQA
        args = dict(n_seqs=len(self.lens), cu_q=T.as_tensor(self.cu), max_q=most, variant=variant, n_splits=splits, window=window,
                    kv_base=self.base, block_table=self.table)
        desc = pkv.make_tree_desc(self.q, self.k, self.v, out.t, max_kv, **args)
        need = pkv.pkv_tree_attention_workspace_size(desc, self.H, self.Hkv, self.d, self.kind == "quant")
        ws = Guarded((need,), torch.uint8) if need else None
        pkv.tree_attention(self.q, self.k, self.v, self.dk, self.dv_rows, out.t, T.as_tensor(self.pos),
                           T.as_tensor(np.array(self.lens, np.int32)), self.scale, max_kv, mask=mask, lse_out=lse,
                           workspace=None if ws is None else ws.t, k_scale=self.ks, v_scale=self.vs, stream=stream, **args, **kw)
        torch.cuda.synchronize()
        out.check("output")
        if ws is not None:
            ws.check("workspace")
        return out, lse

    def cache(self, name, layer, s, kv):
        """Keys or values of one sequence, [Hkv][kv][*] in 64 bits."""
        t = {"k": self.k, "v": self.v}[name]
        if self.table is None:
            b = int(self.base[s])
            x = t[layer, :, b:b + kv].double().cpu().numpy()
        elif self.kind == "quant":
            scale = {"k": self.ks, "v": self.vs}[name]
            x = R.logical(t[layer:layer + 1].cpu().numpy(), scale[layer:layer + 1].cpu().numpy(), self.table[s].cpu().numpy(), kv)[0]
        else:
            page = t.shape[2]
            j = torch.arange(kv, device="cuda")
            x = t[layer, self.table[s].long()[j // page], j % page].double().permute(1, 0, 2).cpu().numpy()
        return x[..., :self.dv] if name == "v" else x

    def check(self, out, lse, window=0, max_kv=None, **bf16_tol):
        got = out.t.float().cpu().numpy().astype(np.float64)
        for l in range(self.L):
            for s, n in enumerate(self.sizes):
                if n == 0:
                    continue
                kv = self.lens[s] if max_kv is None else min(self.lens[s], max_kv)
                at = slice(int(self.cu[s]), int(self.cu[s]) + n)
                want, want_lse = T.attention(self.q[l, at].double().cpu().numpy(), self.cache("k", l, s, kv), self.cache("v", l, s, kv),
                                             self.dk[l, :, at].double().cpu().numpy(),
                                             self.dv_rows[l, :, at].double().cpu().numpy()[..., :self.dv], self.pos[at], self.seen[s],
                                             self.scale, window)
                empty = np.isneginf(want_lse)
                assert not got[l, at][empty].any() and np.isneginf(lse[l, at].cpu().numpy()[empty]).all()
                assert not out.t[l, at].isnan().any()
                full = ~empty
                if full.any():
                    tol = dict(max_abs=1.3e-3, mean_abs=1.3e-3, rel_l2=2.6e-4) if self.kind == "f32" else bf16_tol
                    check_attention_close(got[l, at][full], want[full], **tol)
                    np.testing.assert_allclose(lse[l, at].cpu().numpy()[full], want_lse[full], atol=1.3e-4 if self.kind == "f32" else 2e-2)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("splits", [0, 1, 3])
def test_trees(kind, splits):
    """Ragged caches from no slot on, trees from one row on; two layers."""
    c = Case(kind, [700, 0, 33, 1, 250], [9, 5, 1, 40, 17], L=2, seed=splits)
    out, lse = c.call(c.masks(), splits)
    c.check(out, lse)
    again, _ = c.call(c.masks(), splits)
    assert same(out.t, again.t)


@pytest.mark.parametrize("kind", ["bf16", "f32", "paged", "quant"])
@pytest.mark.parametrize("G", [1, 3, 7, 16])
@pytest.mark.parametrize("d", [64, 128])
def test_heads(kind, G, d):
    """Few and many rows a KV head, groups of every kind."""
    c = Case(kind, [300], [3], G=G, d=d, seed=G)
    c.check(*c.call(c.masks()))
    c = Case(kind, [40, 1500], [33, 8], G=G, d=d, seed=G + 1)
    c.check(*c.call(c.masks()))


@pytest.mark.parametrize("heads", [1, 2, 32])
def test_latent_heads(heads):
    c = Case("mla", [300, 70], [3, 6], G=heads, seed=heads)
    c.check(*c.call(c.masks()))


@pytest.mark.parametrize("kind", KINDS)
def test_one_row(kind):
    """A tree that is its root: token-by-token generation with the token's keys beside the cache."""
    c = Case(kind, [2000, 5, 64, 0], [1, 1, 1, 1], seed=3)
    c.check(*c.call(c.masks()))
    c.check(*c.call(None))


@pytest.mark.parametrize("kind", KINDS)
def test_no_cache(kind):
    """No slot anywhere: the trees alone, without a workspace."""
    c = Case(kind, [0, 0], [20, 3], seed=4)
    c.check(*c.call(c.masks()))
    c.check(*c.call(c.masks(), max_kv=1))


@pytest.mark.parametrize("kind", KINDS)
def test_chain(kind):
    """Without a mask a row sees the rows up to itself, as with a chain's mask."""
    c = Case(kind, [130, 64], [70, 2], ways=1, seed=5)
    out, lse = c.call(None)
    c.check(out, lse)
    other, _ = c.call(c.masks())
    assert same(out.t, other.t)


@pytest.mark.parametrize("n", [31, 32, 33, 63, 64, 65, 200])
def test_words(n):
    """Masks that end in, at and behind a word."""
    for kind in ("bf16", "f32", "mla"):
        c = Case(kind, [50], [n], G=2, d=64, seed=n)
        c.check(*c.call(c.masks()))


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("window", [1, 3, 40, 600])
def test_window(kind, window):
    c = Case(kind, [700, 10], [40, 9], ways=1, seed=6)
    for splits in (0, 2):
        c.check(*c.call(c.masks(), splits, window), window=window)


@pytest.mark.parametrize("kind", KINDS)
def test_any_bits(kind):
    """Masks that are no trees: rows that see nothing (zeros, -inf), rows that see later ones, bits behind the
    sequence's end and behind the words' use."""
    c = Case(kind, [0, 90], [35, 12], seed=7)
    c.seen = [c.rng.random(s.shape) < 0.3 for s in c.seen]
    c.seen[0][[0, 5, 34]] = False
    c.seen[1][3] = False
    mask = c.masks().cpu().numpy().view(np.uint32)
    mask[:35, 1] |= np.uint32(0xffffffff) << np.uint32(3)    # columns 35.. of the first sequence
    mask[35:, 0] |= np.uint32(0xffffffff) << np.uint32(12)
    mask[35:, 1] = 0xffffffff
    c.pos[35 + 3] = -1                                       # nor does it see the cache
    out, lse = c.call(T.as_tensor(mask.view(np.int32)))
    c.check(out, lse)
    assert np.isneginf(lse.cpu().numpy()[0, [0, 5, 34, 38]]).all()


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_nonfinite_rows(kind, bad):
    """What a row does not see does not reach it: unseen drafted rows, rows of other sequences, rows of none.  A NaN that
    is seen makes the row NaN."""
    c = Case(kind, [100, 40], [6, 5], seed=8, extra_rows=2)
    c.seen[0][:, 4] = False
    c.seen[0][4] = False
    c.seen[0][4, 0] = True
    clean, _ = c.call(c.masks())
    for t in (c.dk, c.dv_rows):
        t[:, :, [4, 11, 12]] = bad
    c.q[:, 11:] = bad
    out, lse = c.call(c.masks())
    assert same(out.t[:, :11], clean.t[:, :11])
    assert out.untouched((slice(None), slice(11, None))) and bool((lse[:, 11:] == 7.0).all())
    c.seen[0][5, 4] = True
    out, _ = c.call(c.masks())
    if math.isnan(bad):
        assert bool(out.t[:, 5].isnan().all())
    rest = [0, 1, 2, 3, 4, 6, 7, 8, 9, 10]
    assert same(out.t[:, rest], clean.t[:, rest])


@pytest.mark.parametrize("kind", ["bf16", "f32", "paged", "mla"])
def test_nan_in_the_cache(kind):
    """A NaN in a seen slot reaches the rows of its sequence and head, through the partials of one or several splits."""
    for splits in (1, 3):
        c = Case(kind, [300, 200], [5, 4], seed=9)
        clean, _ = c.call(c.masks(), splits)
        if c.table is None:
            c.k[0, 0, int(c.base[0]) + 7] = math.nan
        else:
            c.k[0, int(c.table[0, 0]), 7, 0] = math.nan
        out, _ = c.call(c.masks(), splits)
        G = c.H // c.Hkv
        assert bool(out.t[:, :5, :G].isnan().all())
        assert same(out.t[:, 5:], clean.t[:, 5:])
        assert same(out.t[:, :5, G:], clean.t[:, :5, G:])


@pytest.mark.parametrize("kind", ["bf16", "quant", "mla"])
def test_rows_of_no_sequence(kind):
    """Rows in front of the first sequence and behind the last are left as they were; bounds that do not fit own none."""
    c = Case(kind, [90], [7], seed=10, extra_rows=3, gap=4)
    out, lse = c.call(c.masks())
    c.check(out, lse)
    assert out.untouched((slice(None), slice(0, 4))) and out.untouched((slice(None), slice(11, None)))
    assert bool((lse[:, :4] == 7.0).all()) and bool((lse[:, 11:] == 7.0).all())
    c.cu = np.array([4, c.rows + 1], np.int32)
    out, lse = c.call(c.masks())
    assert out.untouched((slice(None), slice(None))) and bool((lse == 7.0).all())


def test_scales():
    """Scale 0, a negative one, large scores."""
    for kind in ("bf16", "f32", "mla"):
        for scale, gain in ((0.0, 1.5), (-0.1, 1.5), (1.0, 3.0)):
            c = Case(kind, [70], [12], seed=11, gain=gain)
            c.scale = scale
            if scale == 1.0:   # one key carries a row: weights and outputs follow the scores' own rounding
                out, lse = c.call(c.masks())
                assert not out.t.isnan().any() and not lse.isnan().any()
            else:
                c.check(*c.call(c.masks()))


def test_positions_at_the_ends():
    """Positions and windows of any int32 value."""
    for kind in ("bf16", "f32", "mla"):
        for window in (0, 1, 2 ** 31 - 1):
            c = Case(kind, [70], [6], seed=12)
            c.pos[:] = [2 ** 31 - 1, -2 ** 31, 0, 69, 70, 2 ** 31 - 1]
            c.check(*c.call(c.masks(), 0, window), window=window)


@pytest.mark.parametrize("kind", ["bf16", "f32"])
def test_strides(kind):
    """Rows, heads and layers apart, in other orders; offsets of drafted rows past 2^32 bytes."""
    c = Case(kind, [90, 30], [8, 3], L=2, seed=13, d=64)
    want, _ = c.call(c.masks())
    wide = torch.zeros(c.rows, c.H, c.L, 80, dtype=c.dtype, device="cuda")   # [row][head][layer][channel]
    wide[..., :64] = c.q.permute(1, 2, 0, 3)
    c.q = wide[..., :64].permute(2, 0, 1, 3)
    far = 2 ** 31 + 64
    for name in ("dk", "dv_rows"):
        t = getattr(c, name)
        buf = torch.empty(far + t.numel(), dtype=c.dtype, device="cuda")
        x = torch.as_strided(buf, t.shape, (far, c.rows * 64, 64, 1))
        x.copy_(t)
        setattr(c, name, x)
    got, _ = c.call(c.masks())
    assert same(got.t, want.t)


@pytest.mark.parametrize("kind", ["bf16", "paged", "mla"])
def test_more_sequences_than_lanes(kind):
    """More sequences than a wave has lanes: all are cut alike.

    Many of these rows see a few slots only, so their outputs are as large as the values, not of unit size: with every probability
    and the output off by half a step of bf16, 2^-8 of itself, an output is off by 2^-8 sum(p |v|) + 2^-8 |o| <= 2^-7 max |v|;
    the largest of 3 million normal values is below 6 (two-sided tail 2e-9 each): 6 / 128 = 0.047."""
    rng = np.random.default_rng(20)
    c = Case(kind, rng.integers(0, 200, 100), rng.integers(1, 4, 100), G=2, Hkv=1, d=64, seed=20)
    for splits in (0, 2):
        c.check(*c.call(c.masks(), splits), max_abs=0.047)


@pytest.mark.parametrize("kind", ["bf16", "f32", "mla"])
def test_many_splits(kind):
    """More records of a row than a wave has lanes."""
    c = Case(kind, [7000, 130], [3, 2], G=1, Hkv=1, d=64, seed=21)
    c.check(*c.call(c.masks(), 100))


class Wide(Case):
    """Enough rows for the join in tiles: 30 sequences of up to 27 rows, 16 heads a KV head (24576 rows of a head or more, 64 or
    more of each KV head).  Rows see few slots: bf16 outputs are off by up to 2^-7 max |v|, as above, and the probabilities of
    drafted rows are rounded like those of the cache."""

    def check(self, out, lse, **kw):
        super().check(out, lse, max_abs=0.047, **kw)

    def __init__(self, kind, seed, d=128, ways=2, most=40, nodes=27, **kw):
        rng = np.random.default_rng(seed)
        sizes = rng.integers(1, nodes + 1, 30)
        sizes[3], sizes[4] = nodes, 0
        lens = rng.integers(0, most + 1, 30)
        lens[5] = 0
        super().__init__(kind, lens, sizes, G=16, d=d, ways=ways, seed=seed, **kw)
        assert 30 * max(self.sizes) * self.H >= 24576


@pytest.mark.parametrize("kind", ["bf16", "paged", "quant"])
@pytest.mark.parametrize("d", [64, 128])
def test_wide(kind, d):
    c = Wide(kind, 22 + d, d)
    for splits in (0, 3):
        out, lse = c.call(c.masks(), splits)
        c.check(out, lse)
    again, _ = c.call(c.masks(), splits)
    assert same(out.t, again.t)
    c = Wide(kind, 23 + d, d, ways=1)
    out, lse = c.call(None)
    c.check(out, lse)
    other, _ = c.call(c.masks())
    assert same(out.t, other.t)


@pytest.mark.parametrize("window", [1, 5, 30])
def test_wide_window(window):
    c = Wide("bf16", 24, ways=1)
    c.check(*c.call(c.masks(), 0, window), window=window)


def test_wide_rows_of_more_than_a_tile():
    """Rows that see drafted rows of several tiles, or none of the first."""
    for d in (64, 128):
        c = Case("bf16", [20] * 9, [70, 33, 64, 1, 90, 32, 31, 65, 90], G=16, d=d, seed=25 + d)
        assert 9 * 90 * c.H >= 24576
        c.check(*c.call(c.masks()), max_abs=0.047)
        c.seen = [c.rng.random(s.shape) < 0.1 for s in c.seen]
        c.seen[4][:, :40] = False
        c.seen[0][7] = False
        c.pos[7] = -1
        out, lse = c.call(c.masks())
        c.check(out, lse, max_abs=0.047)
        assert np.isneginf(lse.cpu().numpy()[0, 7]).all()


@pytest.mark.parametrize("most", [0, 40])
@pytest.mark.parametrize("kind", ["bf16", "paged", "quant"])
def test_wide_of_few_rows(kind, most):
    """Many small trees whose rows have one record, or none."""
    rng = np.random.default_rng(31)
    for d in (64, 128):
        c = Case(kind, rng.integers(0, most + 1, 60), np.r_[9, rng.integers(1, 10, 59)], G=4, Hkv=4, d=d, seed=31 + d)
        assert 60 * 9 * c.H >= 8192
        out, lse = c.call(c.masks())
        c.check(out, lse, max_abs=0.047)


@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_wide_nonfinite_rows(bad):
    """In the join in tiles a value that is no finite number is left out of the tile and reaches the rows that see it,
    by hand; keys that a row does not see do not matter."""
    for d in (64, 128):
        c = Wide("bf16", 26 + d, d)
        at = int(c.cu[3])
        c.seen[3][:, 4] = False
        c.seen[3][4] = False
        c.seen[3][4, 0] = True
        clean, _ = c.call(c.masks())
        c.dk[:, :, at + 4] = bad
        c.dv_rows[:, :, at + 4] = bad
        out, lse = c.call(c.masks())
        assert same(out.t, clean.t)
        # one value of the row, seen by two rows
        c.dk[:, :, at + 4] = 0.5
        c.dv_rows[:, :, at + 4] = 0.25
        c.dv_rows[0, 1, at + 4, 9] = bad
        c.seen[3][[7, 9], 4] = True
        out, lse = c.call(c.masks())
        assert not lse.isnan().any()
        x = out.t[0].float().cpu().numpy()
        for i in (7, 9):
            assert np.isnan(x[at + i, 16:, 9]).all() if math.isnan(bad) else (x[at + i, 16:, 9] == bad).all()
        x[[at + 7, at + 9], 16:, 9] = 0
        assert np.isfinite(x).all()
        rest = [r for r in range(c.rows) if r not in (at + 7, at + 9)]
        assert same(out.t[:, rest], clean.t[:, rest])


def test_many_sequences():
    """More sequences than a grid dimension holds."""
    n = 65540
    c = Case("f32", [1] * n, [1] * n, G=1, Hkv=1, d=64, seed=14)
    out, lse = c.call(c.masks())
    x = torch.stack([c.k[0, 0, c.base], c.dk[0, 0]], 1).double()
    v = torch.stack([c.v[0, 0, c.base], c.dv_rows[0, 0]], 1).double()
    p = torch.softmax((x * c.q[0, :, 0].double()[:, None]).sum(-1) * c.scale, -1)
    assert float(((p[..., None] * v).sum(1) - out.t[0, :, 0]).abs().max()) < 1.3e-3


@pytest.mark.parametrize("kind", ["bf16", "quant"])
def test_more_rows_than_stated(kind):
    """Rows behind the stated bound are left as they were; the others still see all that their masks say."""
    c = Case(kind, [90], [9], seed=15)
    c.seen[0][2, 8] = True
    out, lse = c.call(c.masks(), max_q=5)
    assert out.untouched((slice(None), slice(5, None))) and bool((lse[:, 5:] == 7.0).all())
    at = slice(0, 5)
    want, _ = T.attention(c.q[0, at].double().cpu().numpy(), c.cache("k", 0, 0, 90), c.cache("v", 0, 0, 90), c.dk[0].double().cpu().numpy(),
                          c.dv_rows[0].double().cpu().numpy(), c.pos, c.seen[0][at], c.scale)
    check_attention_close(host_bits(out.t[0, at]), want)


def test_value_pages_of_their_own():
    c = Case("paged", [100, 40], [6, 4], seed=16)
    want, _ = c.call(c.masks())
    P = c.k.shape[1]
    perm = torch.randperm(P, generator=torch.Generator().manual_seed(1)).cuda()
    moved = torch.empty_like(c.v)
    moved[:, perm] = c.v
    c.v = moved
    got, _ = c.call(c.masks(), v_block_table=perm[c.table.long()].to(torch.int32).contiguous())
    assert same(got.t, want.t)


def test_value_pages_of_their_own_in_8_bits():
    c = Case("quant", [100, 40], [6, 4], seed=19)
    want, _ = c.call(c.masks())
    perm = torch.randperm(c.k.shape[1], generator=torch.Generator().manual_seed(1)).cuda()
    for t in ("v", "vs"):
        moved = torch.empty_like(getattr(c, t))
        moved[:, perm] = getattr(c, t)
        setattr(c, t, moved)
    got, _ = c.call(c.masks(), v_block_table=perm[c.table.long()].to(torch.int32).contiguous())
    assert same(got.t, want.t)


@pytest.mark.parametrize("kind", ["bf16", "quant", "mla"])
def test_another_stream(kind):
    c = Case(kind, [3000, 70], [8, 5], seed=17)
    want, _ = c.call(c.masks())
    s = torch.cuda.Stream()
    mask = c.masks()
    torch.cuda.synchronize()
    got, _ = c.call(mask, stream=s)
    assert same(got.t, want.t)


def test_refusals_of_the_binding():
    c = Case("bf16", [70], [6], seed=18)
    with pytest.raises(ValueError, match="mask"):
        c.call(torch.zeros(c.rows - 1, 1, dtype=torch.int32, device="cuda"))
    with pytest.raises(TypeError, match="mask"):
        c.call(torch.zeros(c.rows, 1, dtype=torch.int64, device="cuda"))
    dk = c.dk
    c.dk = dk[:, :, :-1]
    with pytest.raises(ValueError, match="draft_k"):
        c.call(c.masks())
    c.dk = dk.float()
    with pytest.raises(TypeError, match="draft_k"):
        c.call(c.masks())
    c.dk = dk.cpu()
    with pytest.raises(ValueError, match="draft_k"):
        c.call(c.masks())
    log("  refused")
