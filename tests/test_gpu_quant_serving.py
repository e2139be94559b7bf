"""The 8-bit cache as a serving program uses it: chunks composed into a sequence, branches forked, tokens appended
and attended over, branches dropped, the pool compacted, more tokens; each attention against the oracle on what the
caches then hold, eagerly and as a captured step that is replayed."""
import math

import numpy as np
import pytest
import torch

import quant_ref as R
from helpers import check_attention_close, host_bits, log
from paper_2606_17107_amd import pkv, synth

pytestmark = pytest.mark.gpu

L, H, HKV, D, PAGE, BLOCK, ROWS, WIDTH, P = 2, 8, 2, 128, 64, 32, 6, 12, 60


class Server:
    def __init__(self):
        self.k, self.v = (torch.full((L, P, PAGE, HKV, D), 0x7f, dtype=torch.uint8, device="cuda") for _ in "kv")
        self.ks, self.vs = (torch.zeros((L, P, PAGE // BLOCK, HKV), dtype=torch.uint8, device="cuda") for _ in "kv")
        self.table = torch.full((ROWS, WIDTH), -1, dtype=torch.int32, device="cuda")
        self.ref = torch.zeros(P, dtype=torch.int32, device="cuda")
        self.kv_len = torch.zeros(ROWS, dtype=torch.int32, device="cuda")
        self.pools = [self.k, self.v, self.ks, self.vs]
        self.flag = torch.zeros(1, dtype=torch.int32, device="cuda")
        self.g = synth.Draws(77, "cuda")

    def give(self, seq, pages):
        """The host's own allocation for a sequence that grows: pages at its end."""
        used = (self.ref > 0).cpu().numpy()
        free = [p for p in range(P - 1, -1, -1) if not used[p]][:pages]
        row = self.table[seq].cpu().numpy()
        row[np.nonzero(row < 0)[0][:pages]] = free
        self.table[seq] = torch.from_numpy(row).cuda()
        self.ref[torch.tensor(free).cuda()] = 1

    def splice(self, segs, src_k, src_v, longest):
        recs = pkv.make_segments_quant([dict(src_slot0=a, seq=b, n_tokens=n, src_pos0=p, dst_pos0=e)
                                        for a, b, n, p, e in segs], "cuda")
        pkv.reposition_splice_quant(src_k, src_v, *self.pools, recs, len(segs), longest, self.kv_len, self.table, 1e4, D,
                                    err_flag=self.flag)

    def attend(self, seqs, n):
        """The last n tokens of each sequence, against the oracle."""
        idx = torch.tensor(seqs, device="cuda")
        q = self.g.normal((L, len(seqs) * n, H, D)) * 1.5
        lens = self.kv_len[idx].cpu().tolist()
        pos = torch.tensor([m - n + i for m in lens for i in range(n)], dtype=torch.int32, device="cuda")
        out = torch.zeros_like(q)
        cu = torch.arange(0, len(seqs) * n + 1, n, dtype=torch.int32, device="cuda")
        pkv.suffix_attention_quant(q, *self.pools, out, pos, self.kv_len[idx].contiguous(), self.table[idx].contiguous(),
                                   1 / math.sqrt(D), max_kv_len=max(lens), n_seqs=len(seqs), cu_q=cu, max_q=n)
        torch.cuda.synchronize()
        assert int(self.flag.item()) == 0
        k, v, ks, vs = (t.cpu().numpy() for t in self.pools)
        table, got, qb, p = self.table.cpu().numpy(), host_bits(out), host_bits(q), pos.cpu().numpy()
        for i, s in enumerate(seqs):
            at = slice(i * n, (i + 1) * n)
            for l in range(L):
                want, _ = R.attention(qb[l, at], k[l], v[l], ks[l], vs[l], table[s], table[s], p[at], lens[i],
                                      1 / math.sqrt(D))
                check_attention_close(got[l, at], want)
        return out


def test_compose_fork_generate_compact():
    s = Server()
    lib_k, lib_v = s.g.normal((L, HKV, 300, D)), s.g.normal((L, HKV, 300, D))
    # two skills composed back to back into row 0
    s.give(0, 5)
    s.splice([(0, 0, 101, 0, 0), (150, 0, 150, 900, 101)], lib_k, lib_v, 150)
    s.kv_len[0] = 251
    s.attend([0], 64)
    # three branches
    forks = pkv.make_forks([dict(parent=0, child=c, n_tokens=251) for c in (1, 2, 3)], "cuda")
    pkv.pages_fork(s.pools, s.ref, s.table, PAGE, forks, 3, err_flag=s.flag)
    s.kv_len[1:4] = 251
    rows = s.table.cpu().numpy()
    assert (rows[1:4, :3] == rows[0, :3]).all() and len(set(rows[:4, 3])) == 4
    # each branch goes its own way: a token at a time over the page's end
    history = [[] for _ in range(4)]
    for step in range(8):
        if step == 5:
            for c in (1, 2, 3):
                s.give(c, 1)
        new_k, new_v = s.g.normal((L, HKV, 3, D)) * (1 + step), s.g.normal((L, HKV, 3, D))
        s.splice([(c - 1, c, 1, 251 + step, 251 + step) for c in (1, 2, 3)], new_k, new_v, 1)
        s.kv_len[1:4] += 1
        s.attend([1, 2, 3], 1)
    # the parent's own cache is what it was
    s.attend([0], 64)
    # two branches end, the pool is compacted, the last one is as before
    before = s.attend([3], 1)
    gone = torch.tensor([1, 2], dtype=torch.int32, device="cuda")
    pkv.pages_free(s.pools, s.ref, s.table, PAGE, gone, err_flag=s.flag)
    state = R.logical(s.k.cpu().numpy(), s.ks.cpu().numpy(), s.table[3].cpu().numpy(), 259)
    used = pkv.pages_compact(s.pools, s.ref, s.table, PAGE, err_flag=s.flag)
    torch.cuda.synchronize()
    assert int(used.item()) == 5 + 2 and int((s.ref > 0).sum()) == 7 and int(s.table.max()) < 7
    np.testing.assert_array_equal(R.logical(s.k.cpu().numpy(), s.ks.cpu().numpy(), s.table[3].cpu().numpy(), 259), state)
    s.attend([3], 1)
    s.attend([0, 3], 40)
    log("  composed, forked, generated, compacted")


def test_captured_generation_step():
    """A step (store a token for each sequence, attend) in a graph: lengths, segments and tables are device data that
    advance between the replays, and every replay equals the eager step."""
    s, e = Server(), Server()
    n = 3
    for x in (s, e):
        x.g = synth.Draws(78, "cuda")
        for c in range(n):
            x.give(c, 3)
        k, v = x.g.normal((L, HKV, 100, D)), x.g.normal((L, HKV, 100, D))
        x.splice([(0, c, 60 + 7 * c, 0, 0) for c in range(n)], k, v, 80)
        x.kv_len[:n] = torch.tensor([60, 67, 74], dtype=torch.int32)
    step_k, step_v = (torch.zeros((L, HKV, n, D), dtype=torch.bfloat16, device="cuda") for _ in "kv")
    q = torch.zeros((L, n, H, D), dtype=torch.bfloat16, device="cuda")
    out = {}
    calls = {}
    for name, x in (("graph", s), ("eager", e)):
        recs = pkv.make_segments_quant([dict(src_slot0=c, seq=c, n_tokens=1, src_pos0=60 + 7 * c, dst_pos0=60 + 7 * c)
                                        for c in range(n)], "cuda")
        pos = torch.tensor([60, 67, 74], dtype=torch.int32, device="cuda")
        o = out[name] = torch.zeros_like(q)
        cu = torch.arange(n + 1, dtype=torch.int32, device="cuda")
        words = recs.view(torch.int32).view(n, 6)

        def step(x=x, recs=recs, pos=pos, o=o, cu=cu, words=words):
            pkv.reposition_splice_quant(step_k, step_v, *x.pools, recs, n, 1, x.kv_len, x.table, 1e4, D)
            x.kv_len[:n] += 1
            pkv.suffix_attention_quant(q, *x.pools, o, pos, x.kv_len, x.table, 1 / math.sqrt(D), max_kv_len=WIDTH * PAGE,
                                       n_seqs=n, cu_q=cu, max_q=1)
            pos.add_(1)
            words[:, 4:] += 1

        calls[name] = step
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls["graph"]()
    for i in range(20):
        step_k.copy_(s.g.normal(step_k.shape) * (1 + i % 3))
        step_v.copy_(s.g.normal(step_k.shape))
        q.copy_(s.g.normal(q.shape))
        graph.replay()
        calls["eager"]()
        torch.cuda.synchronize()
        assert torch.equal(out["graph"], out["eager"]), i
        assert all(torch.equal(a, b) for a, b in zip(s.pools, e.pools)), i
        assert bool((out["graph"] != 0).any())
    assert s.kv_len[:n].cpu().tolist() == [80, 87, 94]
