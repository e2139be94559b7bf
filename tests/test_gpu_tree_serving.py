"""Speculative decoding as a serving program runs it: a chunk spliced into the cache, then steps of masks, tree attention,
verification and commit, eagerly against the references and as a captured step that is replayed."""
import math

import numpy as np
import pytest
import torch

import tree_ref as T
from helpers import check_attention_close, host_bits, log
from paper_2606_17107_amd import pkv, synth
from test_gpu_tree_attention import Case, same

pytestmark = pytest.mark.gpu

L, G, HKV, D, PAGE, BLOCK, WIDTH, V, S, NODES, PATH = 2, 4, 2, 128, 64, 32, 8, 500, 3, 12, 6


class Server:
    """Caches of S sequences, held in bf16 pages or in 8 bits, and a step over one tree each."""

    def __init__(self, quant, seed=3):
        self.quant, self.d = quant, synth.Draws(seed, "cuda")
        pages = S * WIDTH + 2
        shape = (L, pages, PAGE, HKV, D)
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        self.table = torch.randperm(pages, generator=torch.Generator().manual_seed(seed))[:S * WIDTH].view(S, WIDTH).to(torch.int32).cuda()
        self.kv_len = torch.tensor([70, 0, 31], dtype=torch.int32, device="cuda")
        self.ks = self.vs = None
        if quant:
            self.k, self.v = (torch.full(shape, 0x7f, dtype=torch.uint8, device="cuda") for _ in "kv")
            self.ks, self.vs = (torch.zeros((L, pages, PAGE // BLOCK, HKV), dtype=torch.uint8, device="cuda") for _ in "kv")
            src = [self.d.normal((L, HKV, 101, D)) for _ in "kv"]
            zero = torch.zeros(S, dtype=torch.int32, device="cuda")
            segs = pkv.make_segments_quant([dict(src_slot0=0, seq=0, n_tokens=70, src_pos0=0, dst_pos0=0),
                                            dict(src_slot0=70, seq=2, n_tokens=31, src_pos0=500, dst_pos0=0)], "cuda")
            pkv.reposition_splice_quant(*src, self.k, self.v, self.ks, self.vs, segs, 2, 70, zero, self.table, 1e4, D)
        else:
            self.k, self.v = (torch.full(shape, math.nan, dtype=torch.bfloat16, device="cuda") for _ in "kv")
            for s, n in ((0, 70), (2, 31)):
                src = [self.d.normal((L, HKV, n, D)) for _ in "kv"]
                at = torch.arange(n, dtype=torch.int32, device="cuda")
                pkv.reposition_splice_paged(*src, self.k, self.v, at + 9, at, self.table[s:s + 1].contiguous(), 1e4, D)
        rows = S * NODES
        i32 = lambda *shape: torch.zeros(shape, dtype=torch.int32, device="cuda")   # noqa: E731
        self.cu = torch.arange(0, rows + 1, NODES, dtype=torch.int32, device="cuda")
        self.parent, self.tokens = i32(rows), i32(rows)
        self.q = torch.zeros((L, rows, HKV * G, D), dtype=torch.bfloat16, device="cuda")
        self.dk, self.dv = (torch.zeros((L, rows, HKV, D), dtype=torch.bfloat16, device="cuda") for _ in "kv")
        self.target, self.draft = (torch.zeros((rows, V), device="cuda") for _ in "td")
        self.ua, self.us = torch.zeros(rows, device="cuda"), torch.zeros(S, device="cuda")
        self.mask, self.pos = i32(rows, 1), i32(rows)
        self.out = torch.zeros_like(self.q)
        self.path, self.count, self.next = i32(S, PATH), i32(S), i32(S)
        self.flag = i32(1)

    def draw(self, rng):
        """What the models bring to a step."""
        trees = [T.random_tree(rng, NODES, 2) for _ in range(S)]
        logits = rng.normal(size=(S * NODES, V)) * 2
        soft = lambda x: torch.softmax(torch.from_numpy(x).float().cuda(), -1)   # noqa: E731
        self.target.copy_(soft(logits))
        self.draft.copy_(soft(logits + 0.3 * rng.normal(size=logits.shape)))
        self.parent.copy_(torch.from_numpy(np.concatenate(trees)))
        at = torch.from_numpy(np.concatenate([np.maximum(t, 0) + NODES * s for s, t in enumerate(trees)])).cuda()
        e = torch.from_numpy(rng.exponential(size=(S * NODES, V))).cuda()
        self.tokens.copy_((self.draft[at] / e).argmax(-1))
        self.ua.copy_(torch.from_numpy(rng.random(S * NODES)) * 0.7)
        self.us.copy_(torch.from_numpy(rng.random(S)))
        for t in (self.q, self.dk, self.dv):
            t.copy_(torch.from_numpy(rng.normal(size=tuple(t.shape))))

    def step(self):
        dk, dv = self.dk.transpose(1, 2), self.dv.transpose(1, 2)
        pkv.tree_masks(self.parent, self.kv_len, n_seqs=S, cu_q=self.cu, max_q=NODES, mask=self.mask, q_pos=self.pos, err_flag=self.flag)
        pkv.tree_attention(self.q, self.k, self.v, dk, dv, self.out, self.pos, self.kv_len, 1 / math.sqrt(D), WIDTH * PAGE, mask=self.mask,
                           n_seqs=S, cu_q=self.cu, max_q=NODES, block_table=self.table, k_scale=self.ks, v_scale=self.vs)
        pkv.tree_verify(self.target, self.tokens, self.parent, self.ua, self.us, PATH, self.draft, n_seqs=S, cu_q=self.cu, max_q=NODES,
                        path=self.path, n_accepted=self.count, next_token=self.next, err_flag=self.flag)
        pkv.tree_commit(dk, dv, self.k, self.v, self.path, self.count, self.kv_len, block_table=self.table, k_scale=self.ks,
                        v_scale=self.vs, err_flag=self.flag)
        self.kv_len.add_(self.count)

    def state(self):
        return [t for t in (self.k, self.v, self.ks, self.vs, self.kv_len, self.mask, self.pos, self.out, self.path, self.count,
                            self.next) if t is not None]


@pytest.mark.parametrize("quant", [False, True])
def test_steps_against_the_references(quant):
    s, rng = Server(quant), np.random.default_rng(1)
    ref = Case.__new__(Case)     # the attention test's reading of caches and its comparison
    ref.kind, ref.L, ref.mla, ref.H, ref.Hkv, ref.d, ref.dv, ref.base = "quant" if quant else "paged", L, False, HKV * G, HKV, D, D, None
    ref.scale, ref.sizes, ref.cu = 1 / math.sqrt(D), [NODES] * S, s.cu.cpu().numpy()
    got = 0
    for step in range(5):
        s.draw(rng)
        lens = s.kv_len.tolist()
        before = [None if t is None else t.clone() for t in (s.k, s.v, s.ks, s.vs)]
        s.step()
        torch.cuda.synchronize()
        assert int(s.flag) == 0
        # attention saw the caches as they were before the step, and the trees
        ref.lens, ref.table, (ref.k, ref.v, ref.ks, ref.vs) = lens, s.table, before
        ref.q, ref.dk, ref.dv_rows = s.q, s.dk.transpose(1, 2), s.dv.transpose(1, 2)
        trees = s.parent.cpu().numpy().reshape(S, NODES)
        ref.seen = [T.ancestors(t) for t in trees]
        ref.pos = s.pos.cpu().numpy()
        assert ref.pos.tolist() == [lens[i] + int(r.sum()) - 1 for i, seen in enumerate(ref.seen) for r in seen]
        want = [T.attention(s.q[l, at].double().cpu().numpy(), ref.cache("k", l, i, lens[i]), ref.cache("v", l, i, lens[i]),
                            ref.dk[l, :, at].double().cpu().numpy(), ref.dv_rows[l, :, at].double().cpu().numpy(), ref.pos[at], ref.seen[i],
                            ref.scale)[0]
                for l in range(L) for i in range(S) for at in [slice(i * NODES, (i + 1) * NODES)]]
        want = np.stack(want).reshape(L, S * NODES, HKV * G, D)
        check_attention_close(host_bits(s.out), want)
        # the paths and what follows them
        for i in range(S):
            at = slice(i * NODES, (i + 1) * NODES)
            path, after = T.verify(s.target[at].double().cpu().numpy(), s.draft[at].double().cpu().numpy(), s.tokens[at].tolist(), trees[i],
                                   s.ua[at].tolist(), float(s.us[i]), PATH)
            n = int(s.count[i])
            assert [int(r) - i * NODES for r in s.path[i][:n]] == path and int(s.next[i]) == after
            assert int(s.kv_len[i]) == lens[i] + n
            got += n
            # the accepted rows' keys follow the context
            for name, rows_of in (("k", ref.dk), ("v", ref.dv_rows)):
                ref.k, ref.v, ref.ks, ref.vs = s.k, s.v, s.ks, s.vs
                have = ref.cache(name, 0, i, lens[i] + n)[:, lens[i]:]
                new = rows_of[0, :, [i * NODES + r for r in path]].double().cpu().numpy()
                if quant:   # to the nearest code: half a step of 2^-3 relative, or of the block's smallest step
                    step_of = 2.0 ** (128 - 127) * 2.0 ** -9
                    assert (np.abs(have - new) <= np.maximum(np.abs(new) * 2.0 ** -4, step_of / 2)).all()
                else:
                    assert np.array_equal(have, new)
    assert got > 5 * S   # some drafted tokens were accepted
    log("  accepted rows", got)


@pytest.mark.parametrize("quant", [False, True])
def test_captured_step(quant):
    """The whole step in a graph, replayed with the models' new inputs, equals eager steps bit for bit."""
    g, e = Server(quant), Server(quant)
    rng = np.random.default_rng(2)
    warm = Server(quant)
    warm.draw(np.random.default_rng(3))
    warm.step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        g.step()
    for i in range(8):
        seed = int(rng.integers(1 << 30))
        for x in (g, e):
            x.draw(np.random.default_rng(seed))
        graph.replay()
        e.step()
        torch.cuda.synchronize()
        for a, b in zip(g.state(), e.state()):
            assert same(a, b), i
    assert g.kv_len.tolist() == e.kv_len.tolist() and min(g.kv_len.tolist()) >= 8


def test_steps_of_two_servers_at_once():
    """Two captured steps, replayed on streams of their own at the same time, and an eager one on a third."""
    servers = [Server(q, seed) for q, seed in ((False, 4), (True, 5), (False, 6))]
    alone = [Server(q, seed) for q, seed in ((False, 4), (True, 5), (False, 6))]
    warm = Server(False)
    warm.draw(np.random.default_rng(3))
    warm.step()
    torch.cuda.synchronize()
    graphs = [torch.cuda.CUDAGraph() for _ in "ab"]
    for graph, x in zip(graphs, servers):
        with torch.cuda.graph(graph):
            x.step()
    streams = [torch.cuda.Stream() for _ in "abc"]
    for i in range(4):
        for s, a, seed in zip(servers, alone, range(10 * i, 10 * i + 3)):
            s.draw(np.random.default_rng(seed))
            a.draw(np.random.default_rng(seed))
        torch.cuda.synchronize()
        for st, run in zip(streams, [g.replay for g in graphs] + [servers[2].step]):
            with torch.cuda.stream(st):
                run()
        torch.cuda.synchronize()
        for s, a in zip(servers, alone):
            a.step()
            torch.cuda.synchronize()
            for x, y in zip(s.state(), a.state()):
                assert same(x, y), i


def test_the_same_sequence_twice():
    """Two trees over one stretch of a cache (two drafts of one context) attend as each alone, also when a row bound is high."""
    c = Case("bf16", [300, 300], [7, 7], seed=30)
    c.base[1] = c.base[0]
    out, lse = c.call(c.masks())
    c.check(out, lse)
    out, lse = c.call(c.masks(), max_q=32, max_kv=5000)
    c.check(out, lse)
