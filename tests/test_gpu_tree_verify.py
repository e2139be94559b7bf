"""Ancestor masks and verification of trees of drafted tokens against their definitions.  The results are whole numbers and have
to be equal; sums are in 64 bits on both sides, and inputs whose result could hang on their order (a comparison closer than
1e-12) are told apart by the reference, not by the kernels."""
import math

import numpy as np
import pytest
import torch

import tree_ref as T
from helpers import log
from paper_2606_17107_amd import pkv

pytestmark = pytest.mark.gpu


# ---- masks ----------------------------------------------------------------------

@pytest.mark.parametrize("ways", [1, 2, 5])
@pytest.mark.parametrize("sizes", [[1], [32], [33, 1, 0, 64, 65], [1024, 3], [256, 1000, 255]])
def test_masks(sizes, ways):
    rng = np.random.default_rng(sum(sizes) + ways)
    parents = [T.random_tree(rng, n, ways)[:n] for n in sizes]
    lens = rng.integers(0, 2 ** 20, len(sizes)).astype(np.int32)
    cu = np.concatenate([[2], 2 + np.cumsum(sizes)]).astype(np.int32)
    rows = int(cu[-1]) + 3
    parent = np.full(rows, 77, np.int32)
    parent[2:cu[-1]] = np.concatenate(parents)
    words = -(-max(sizes) // 32) + 1                        # one more than needed
    mask = torch.full((rows, words), 0x55, dtype=torch.int32, device="cuda")
    pos = torch.full((rows,), -9, dtype=torch.int32, device="cuda")
    flag = torch.zeros(1, dtype=torch.int32, device="cuda")
    pkv.tree_masks(T.as_tensor(parent), T.as_tensor(lens), n_seqs=len(sizes), cu_q=T.as_tensor(cu), max_q=max(sizes), mask=mask,
                   q_pos=pos, err_flag=flag)
    got, at = mask.cpu().numpy(), pos.cpu().numpy()
    for s, p in enumerate(parents):
        seen = T.ancestors(p)
        np.testing.assert_array_equal(got[cu[s]:cu[s + 1]], T.pack(seen, words))
        np.testing.assert_array_equal(at[cu[s]:cu[s + 1]], lens[s] + seen.sum(1) - 1)
    edge = [0, 1, rows - 3, rows - 2, rows - 1]
    assert (got[edge] == 0x55).all() and (at[edge] == -9).all() and int(flag) == 0


def test_masks_of_bad_parents():
    """Parents that are no earlier row count as none and are flagged; several roots are not."""
    flag = torch.zeros(1, dtype=torch.int32, device="cuda")
    kv = torch.tensor([10], dtype=torch.int32, device="cuda")
    p = np.array([-1, -1, 0, 1, 2], np.int32)
    mask, pos = pkv.tree_masks(T.as_tensor(p), kv, err_flag=flag)
    assert int(flag) == 0 and pos.tolist() == [10, 10, 11, 11, 12]
    p = np.array([0, 5, -2, 2, 2 ** 31 - 1], np.int32)
    mask, pos = pkv.tree_masks(T.as_tensor(p), kv, err_flag=flag)
    assert int(flag) == 1 and mask[:, 0].tolist() == [1, 2, 4, 12, 16] and pos.tolist() == [10, 10, 10, 11, 10]
    mask, pos = pkv.tree_masks(torch.zeros(0, dtype=torch.int32, device="cuda"), kv)
    assert mask.shape[0] == 0
    # bounds that do not fit the call own no rows, rows behind the bound are left alone
    mask = torch.full((6, 1), 9, dtype=torch.int32, device="cuda")
    pkv.tree_masks(T.as_tensor(np.array([-1, 0, 1, 2, 3, 4], np.int32)), torch.zeros(3, dtype=torch.int32, device="cuda"), n_seqs=3,
                   cu_q=T.as_tensor(np.array([0, 4, 9, 3], np.int32)), max_q=2, mask=mask)
    assert mask[:, 0].tolist() == [1, 3, 9, 9, 9, 9]


# ---- verification ---------------------------------------------------------------

class Case:
    def __init__(self, sizes, vocab, ways, drawn, dtype=torch.float32, seed=0, pad=0, gain=2.0, noise=0.7):
        self.rng = rng = np.random.default_rng(seed)
        self.sizes, self.V, self.dtype = list(sizes), vocab, dtype
        self.cu = np.concatenate([[0], np.cumsum(sizes)]).astype(np.int32)
        rows = self.rows = int(self.cu[-1])
        self.parents = [T.random_tree(rng, n, ways)[:n] for n in sizes]
        logits = rng.normal(size=(rows, vocab)) * gain
        soft = lambda x: np.exp(x - x.max(1, keepdims=True)) / np.exp(x - x.max(1, keepdims=True)).sum(1, keepdims=True)   # noqa: E731
        self.target = self.tensor(soft(logits), pad)
        self.draft = self.tensor(soft(logits + noise * rng.normal(size=logits.shape)), pad) if drawn else None
        self.tokens = np.zeros(rows, np.int32)
        q = (self.draft if drawn else self.target).double().cpu().numpy()
        for s, p in enumerate(self.parents):
            for i in range(1, len(p)):
                row = q[self.cu[s] + p[i]]
                self.tokens[self.cu[s] + i] = min(vocab - 1, np.searchsorted(np.cumsum(row), rng.random() * row.sum(), "right"))
        self.u_accept = rng.random(rows).astype(np.float32)
        self.u_sample = rng.random(len(sizes)).astype(np.float32)

    def tensor(self, p, pad):
        """Rows `pad` elements apart, from an address that only the type aligns."""
        rows, V = p.shape
        buf = torch.full((rows * (V + pad) + 1,), math.nan, dtype=self.dtype, device="cuda")
        t = torch.as_strided(buf, (rows, V), (V + pad, 1), 1 if pad else 0)
        t.copy_(torch.from_numpy(p))
        return t

    def call(self, max_path, **kw):
        parent = np.concatenate(self.parents).astype(np.int32) if self.rows else np.zeros(0, np.int32)
        flag = torch.zeros(1, dtype=torch.int32, device="cuda")
        out = pkv.tree_verify(self.target, T.as_tensor(self.tokens), T.as_tensor(parent), T.as_tensor(self.u_accept),
                              T.as_tensor(self.u_sample), max_path, self.draft, n_seqs=len(self.sizes), cu_q=T.as_tensor(self.cu),
                              max_q=max(self.sizes), err_flag=flag, **kw)
        torch.cuda.synchronize()
        return [t.cpu().numpy() for t in out] + [int(flag)]

    def check(self, max_path=8, flag=0):
        """Equal to the definition; returns the lengths of the paths."""
        path, count, after, raised = self.call(max_path)
        p = self.target.double().cpu().numpy()
        q = None if self.draft is None else self.draft.double().cpu().numpy()
        close = 0
        for s, parent in enumerate(self.parents):
            at = slice(self.cu[s], self.cu[s + 1])
            args = (p[at], None if q is None else q[at], self.tokens[at], parent, self.u_accept[at], self.u_sample[s], max_path)
            want = T.verify(*args)
            got = ([int(r) - int(self.cu[s]) for r in path[s][:count[s]]], int(after[s]))
            assert (path[s][count[s]:] == -1).all()
            if got != want:
                close += 1
                assert T.near_tie(*args), (s, got, want)
        assert raised == flag
        assert close <= len(self.sizes) // 100
        return count


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("drawn", [True, False])
@pytest.mark.parametrize("vocab", [1, 2, 31, 4095, 4096, 4097, 20011])
def test_vocabularies(vocab, drawn, dtype):
    n = 40 if vocab < 5000 else 6
    for ways in (1, 3):
        c = Case([7] * n, vocab, ways, drawn, dtype, seed=vocab)
        c.check()


@pytest.mark.parametrize("drawn", [True, False])
@pytest.mark.parametrize("ways", [1, 2, 4])
def test_trees(drawn, ways):
    """Trees of every size in one call, no rows among them."""
    sizes = [1, 2, 0, 5, 63, 64, 65, 130, 3, 200]
    counts = Case(sizes, 50, ways, drawn, seed=ways, gain=1.0).check(16)
    assert counts[2] == 0 and (counts[[0, 1, 3]] > 0).all()
    Case([1024, 1], 20, ways, drawn, seed=ways + 9, gain=1.0).check(64)


def test_large_vocabulary():
    for drawn in (True, False):
        for dtype in (torch.float32, torch.bfloat16):
            Case([9, 4, 6], 150001, 2, drawn, dtype, seed=3).check()


@pytest.mark.parametrize("drawn", [True, False])
def test_strides(drawn):
    """Rows at addresses that only the type aligns."""
    for dtype in (torch.float32, torch.bfloat16):
        for pad in (1, 3, 8):
            Case([5, 9, 2, 17], 1003, 2, drawn, dtype, seed=pad, pad=pad).check()


@pytest.mark.parametrize("drawn", [True, False])
@pytest.mark.parametrize("u", [0.0, 1.0 - 2.0 ** -24, 1.0, 2.0, -1.0, math.nan])
def test_random_numbers_at_the_ends(drawn, u):
    """0 takes every child that has a weight and the first token with one; numbers outside [0, 1) stay defined."""
    c = Case([9] * 30, 40, 2, drawn, seed=5)
    c.u_accept[:] = u
    c.u_sample[:] = u
    c.check()


@pytest.mark.parametrize("limit", [1, 2, 3])
def test_path_limit(limit):
    for drawn in (True, False):
        c = Case([9] * 30, 10, 1, drawn, seed=6, gain=0.5)
        c.u_accept[:] *= 0.3
        counts = c.check(limit)
        assert counts.max() == limit


def test_equal_distributions():
    """Where target and draft agree every drawn token is accepted; refused by force, nothing is left and the row's own
    probabilities are drawn from."""
    c = Case([5] * 20, 33, 1, True, seed=7, noise=0.0)
    assert (c.check() == 5).all()
    c = Case([4] * 20, 33, 9, True, seed=8, noise=0.0)
    c.u_accept[:] = 3.0
    assert (c.check() == 1).all()


def test_all_tokens_tried():
    """Children that cover the vocabulary, all refused; the same token twice."""
    for V in (1, 2, 3):
        c = Case([1 + 2 * V] * 10, V, 50, False, seed=V)
        c.parents = [np.array([-1] + [0] * (2 * V), np.int32)] * 10
        c.tokens = np.array(([0] + list(range(V)) * 2) * 10, np.int32)
        c.u_accept[:] = 5.0
        assert (c.check() == 1).all()
        c.u_accept[:] = 0.9
        c.check()


def test_probabilities_that_are_none():
    """NaN, infinities, negative numbers and zeros count as 0; a row without any weight gives -1 and the flag."""
    for drawn in (True, False):
        for dtype in (torch.float32, torch.bfloat16):
            c = Case([8] * 24, 37, 2, drawn, dtype, seed=9)
            for t in (c.target,) if c.draft is None else (c.target, c.draft):
                bad = torch.from_numpy(c.rng.random((c.rows, 37)) < 0.3).cuda()
                t[bad] = torch.tensor([math.nan, math.inf, -math.inf, -0.5, 0.0, -0.0], dtype=dtype, device="cuda")[
                    torch.from_numpy(c.rng.integers(0, 6, (c.rows, 37))).cuda()][bad]
            c.check()
            c.target[:] = 0
            assert (c.check(flag=1) == 1).all()


def test_rows_out_of_range():
    """Rows with a parent or token out of range are nobody's children, and flagged."""
    for drawn in (True, False):
        c = Case([9] * 12, 40, 2, drawn, seed=10)
        c.u_accept[:] *= 0.2
        c.tokens[3::9] = 40
        c.tokens[5::9] = -1
        c.parents = [np.where(np.arange(9) == 7, 7, p).astype(np.int32) for p in c.parents]
        c.check(flag=1)
        c = Case([9] * 12, 40, 2, drawn, seed=11)
        c.parents = [np.where(np.arange(9) == 4, -1, p).astype(np.int32) for p in c.parents]
        c.tokens[::9] = -5                                    # a root's own token is not looked at
        c.check()


def test_no_rows():
    """Sequences without rows, and a call without any."""
    for sizes in ([0, 3, 0], [0, 0]):
        c = Case(sizes, 50, 1, True, seed=14)
        path, count, after, flag = c.call(4)
        assert (count[np.array(sizes) == 0] == 0).all() and (after[np.array(sizes) == 0] == -1).all() and flag == 0
        assert (path[np.array(sizes) == 0] == -1).all()


def test_nothing_is_written_elsewhere():
    c = Case([4, 3], 100, 1, True, seed=12)
    need = pkv.pkv_tree_verify_workspace_size(pkv.make_verify_desc(c.target, c.draft, T.as_tensor(c.cu), 2, 4, 3))
    buf = torch.full((need + 8192,), 0xA5, dtype=torch.uint8, device="cuda")
    outs = [torch.full((n + 128,), 77, dtype=torch.int32, device="cuda") for n in (6, 2, 2)]
    inside = [outs[0][64:70].view(2, 3), outs[1][64:66], outs[2][64:66]]
    first = c.call(3)
    got = c.call(3, path=inside[0], n_accepted=inside[1], next_token=inside[2], workspace=buf[4096:4096 + need])
    for a, b in zip(first, got):
        np.testing.assert_array_equal(a, b)
    assert bool((buf[:4096] == 0xA5).all()) and bool((buf[4096 + need:] == 0xA5).all())
    for t in outs:
        assert bool((t[:64] == 77).all()) and bool((t[-62:] == 77).all())


def test_same_distribution_as_the_target():
    """The token after the root is distributed as the target's, whatever the draft: 60000 contexts, tokens of a vocabulary of
    5; each frequency within 5 standard deviations."""
    n, V = 60000, 5
    p = np.array([0.05, 0.4, 0.1, 0.25, 0.2])
    q = np.array([0.5, 0.1, 0.2, 0.15, 0.05])
    rng = np.random.default_rng(13)
    target = torch.tensor(p, dtype=torch.float32, device="cuda").expand(4 * n, V)
    for drawn in (True, False):
        draft = torch.tensor(q, dtype=torch.float32, device="cuda").expand(4 * n, V) if drawn else None
        children = rng.choice(V, size=(n, 3), p=q) if drawn else np.array([rng.permutation(V)[:3] for _ in range(n)])
        tokens = np.concatenate([np.zeros((n, 1)), children], 1).astype(np.int32).ravel()
        parent = np.tile(np.array([-1, 0, 0, 0], np.int32), n)
        cu = np.arange(0, 4 * n + 1, 4).astype(np.int32)
        path, count, after = (t.cpu().numpy() for t in pkv.tree_verify(
            target, T.as_tensor(tokens), T.as_tensor(parent), T.as_tensor(rng.random(4 * n).astype(np.float32)),
            T.as_tensor(rng.random(n).astype(np.float32)), 2, draft, n_seqs=n, cu_q=T.as_tensor(cu), max_q=4))
        first = np.where(count == 2, tokens[np.maximum(path[:, 1], 0)], after)
        freq = np.bincount(first, minlength=V) / n
        assert (np.abs(freq - p) < 5 * np.sqrt(p * (1 - p) / n)).all(), freq
        log("  accepted", float((count == 2).mean()), freq)


def test_captured_and_replayed():
    """Two graphs with a workspace each, replayed in turn with new inputs, against eager calls."""
    cases = [Case([8] * 5, 9000, 2, drawn, seed=20 + drawn) for drawn in (True, False)]
    graphs = []
    for c in cases:
        parent, cu = T.as_tensor(np.concatenate(c.parents)), T.as_tensor(c.cu)
        tokens, ua, us = T.as_tensor(c.tokens), T.as_tensor(c.u_accept), T.as_tensor(c.u_sample)
        outs = [torch.zeros(s, dtype=torch.int32, device="cuda") for s in ((5, 8), (5,), (5,))]
        ws = torch.empty(pkv.pkv_tree_verify_workspace_size(pkv.make_verify_desc(c.target, c.draft, cu, 5, 8, 8)), dtype=torch.uint8,
                         device="cuda")
        run = lambda o, w, c=c, a=(tokens, parent, ua, us), cu=cu: pkv.tree_verify(   # noqa: E731
            c.target, a[0], a[1], a[2], a[3], 8, c.draft, n_seqs=5, cu_q=cu, max_q=8, path=o[0], n_accepted=o[1], next_token=o[2],
            workspace=w)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            run(outs, ws)
        graphs.append((graph, run, outs, ua, us))
    for i in range(6):
        for graph, run, outs, ua, us in graphs:
            ua.uniform_(0, 1)
            us.uniform_(0, 1)
        torch.cuda.synchronize()
        for graph, *_ in graphs:
            graph.replay()
        torch.cuda.synchronize()
        for graph, run, outs, ua, us in graphs:
            for a, b in zip(run([None] * 3, None), outs):
                assert torch.equal(a, b), i
