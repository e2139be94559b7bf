"""Calls on a stream beside torch's current one, which is busy: what a call makes for itself (masks, positions, paths, scratch
memory) does not meet the current stream's work, neither a fill nor writes that are still under way into memory freed there."""
import math

import numpy as np
import pytest
import torch

import tree_ref as T
from paper_2606_17107_amd import pkv
from test_gpu_tree_attention import Case, same
from test_gpu_tree_verify import Case as VerifyCase

pytestmark = pytest.mark.gpu


class Busy:
    """The current stream under work of some tenths of a second, and blocks that it still writes when they are freed."""

    def __init__(self):
        self.x = torch.randn(8192, 8192, device="cuda")
        self.y = torch.empty_like(self.x)
        torch.mm(self.x, self.x, out=self.y)
        torch.cuda.synchronize()

    def start(self, *sizes):
        for _ in range(15):
            torch.mm(self.x, self.x, out=self.y)
        blocks = [torch.empty(n, dtype=torch.uint8, device="cuda") for n in sizes for _ in range(4)]
        for t in blocks:
            t.fill_(0x5a)


def test_masks_and_positions():
    rng = np.random.default_rng(1)
    sizes = [40, 1, 70, 33]
    parent = T.as_tensor(np.concatenate([T.random_tree(rng, n, 2) for n in sizes]))
    cu = T.as_tensor(np.concatenate([[0], np.cumsum(sizes)]).astype(np.int32))
    kv = T.as_tensor(np.array([5, 0, 1000, 77], np.int32))
    run = lambda stream=None: pkv.tree_masks(parent, kv, n_seqs=4, cu_q=cu, max_q=70, stream=stream)   # noqa: E731
    mask, pos = run()
    assert bool(mask.any()) and bool(pos.any())
    busy, side = Busy(), torch.cuda.Stream()
    for stream in (side, side.cuda_stream):
        busy.start(mask.numel() * 4, pos.numel() * 4)
        got = run(stream)
        torch.cuda.synchronize()
        assert torch.equal(got[0], mask) and torch.equal(got[1], pos)


@pytest.mark.parametrize("drawn", [True, False])
def test_verification(drawn):
    c = VerifyCase([8] * 5, 9000, 2, drawn, seed=40)
    args = [c.target, T.as_tensor(c.tokens), T.as_tensor(np.concatenate(c.parents)), T.as_tensor(c.u_accept), T.as_tensor(c.u_sample)]
    cu = T.as_tensor(c.cu)
    run = lambda stream=None: pkv.tree_verify(*args, 8, c.draft, n_seqs=5, cu_q=cu, max_q=8, stream=stream)   # noqa: E731
    want = run()
    need = pkv.pkv_tree_verify_workspace_size(pkv.make_verify_desc(c.target, c.draft, cu, 5, 8, 8))
    busy, side = Busy(), torch.cuda.Stream()
    for _ in range(2):
        busy.start(5 * 8 * 4, 5 * 4, need)
        got = run(side)
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert torch.equal(a, b)


@pytest.mark.parametrize("kind", ["bf16", "quant", "mla"])
def test_scratch_of_attention(kind):
    c = Case(kind, [3000, 70], [8, 5], seed=41)
    want, _ = c.call(c.masks())
    mask, pos, lens, cu = c.masks(), T.as_tensor(c.pos), T.as_tensor(np.array(c.lens, np.int32)), T.as_tensor(c.cu)
    out = torch.zeros_like(want.t)
    args = dict(n_seqs=2, cu_q=cu, max_q=8, variant=pkv.PKV_ATTN_MLA if c.mla else pkv.PKV_ATTN_GQA, kv_base=c.base, block_table=c.table)
    desc = pkv.make_tree_desc(c.q, c.k, c.v, out, 3000, **args)
    need = pkv.pkv_tree_attention_workspace_size(desc, c.H, c.Hkv, c.d, kind == "quant")
    assert need
    busy, side = Busy(), torch.cuda.Stream()
    for _ in range(2):
        busy.start(need)
        pkv.tree_attention(c.q, c.k, c.v, c.dk, c.dv_rows, out, pos, lens, c.scale, 3000, mask=mask, k_scale=c.ks, v_scale=c.vs,
                           stream=side, **args)
        torch.cuda.synchronize()
        assert same(out, want.t)


def test_steps_on_a_stream():
    """Masks made by one call and read by the next on the same stream, while the current one is busy; then on the current stream."""
    c = Case("paged", [500, 70], [8, 5], ways=2, seed=42)
    want, _ = c.call(c.masks())
    parent, lens, cu = T.as_tensor(np.concatenate(c.parents)), T.as_tensor(np.array(c.lens, np.int32)), T.as_tensor(c.cu)
    out = torch.zeros_like(want.t)
    busy, side = Busy(), torch.cuda.Stream()
    for _ in range(2):
        busy.start(c.rows * 4)
        mask, pos = pkv.tree_masks(parent, lens, n_seqs=2, cu_q=cu, max_q=8, stream=side)
        pkv.tree_attention(c.q, c.k, c.v, c.dk, c.dv_rows, out, pos, lens, 1 / math.sqrt(c.d), 500, mask=mask, n_seqs=2, cu_q=cu, max_q=8,
                           block_table=c.table, stream=side)
        torch.cuda.current_stream().wait_stream(side)
        kept = mask.clone()
        del mask, pos
        torch.cuda.synchronize()
        assert same(out, want.t)
        assert torch.equal(kept, c.masks())


def test_a_stream_inside_a_capture():
    """A call on a stream that a capture forked makes its tensors in the graph's memory; replays follow their inputs."""
    c = VerifyCase([8] * 5, 3000, 2, True, seed=43)
    parent, tokens, ua, us, cu = (T.as_tensor(a) for a in (np.concatenate(c.parents), c.tokens, c.u_accept, c.u_sample, c.cu))
    kv = T.as_tensor(np.array([3, 0, 9, 77, 5], np.int32))
    run = lambda stream=None: (*pkv.tree_masks(parent, kv, n_seqs=5, cu_q=cu, max_q=8, stream=stream),   # noqa: E731
                               *pkv.tree_verify(c.target, tokens, parent, ua, us, 8, c.draft, n_seqs=5, cu_q=cu, max_q=8, stream=stream))
    run()
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        side.wait_stream(torch.cuda.current_stream())
        outs = run(side)
        torch.cuda.current_stream().wait_stream(side)
    for i in range(4):
        ua.uniform_(0, 1)
        us.uniform_(0, 1)
        kv += 1
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(run(), outs):
            assert torch.equal(a, b), i
