"""Freeing, forking and compacting pages against a reference that works entry by entry: tables, counts and the
contents of every page, bit for bit, over bf16, fp32 and 8-bit pools of any strides."""
import numpy as np
import pytest
import torch

import quant_ref as R
from helpers import log
from paper_2606_17107_amd import pkv

pytestmark = pytest.mark.gpu


def random_pool(rng, n_seqs, width, page, extra, lens=None):
    """Counts and tables: sequences of lens slots on pages of their own, some sharing the pages of one before."""
    lens = [int(rng.integers(0, width * page + 1)) for _ in range(n_seqs)] if lens is None else lens
    P = n_seqs * width + extra
    ids = iter(rng.permutation(P).tolist())
    table, ref = np.full((n_seqs, width), -1, np.int32), np.zeros(P, np.int32)
    for s, n in enumerate(lens):
        donor = int(rng.integers(0, s)) if s and rng.random() < 0.4 else None
        for e in range(-(-n // page)):
            if donor is not None and e < lens[donor] // page and e < n // page:
                table[s, e] = table[donor, e]
            else:
                table[s, e] = next(ids)
            ref[table[s, e]] += 1
    return table, ref, lens


def tensors(rng, P, page, kind, L=2, H=3, d=64):
    def raw(shape, dtype):
        t = torch.from_numpy(rng.integers(0, 256, shape + (torch.empty(0, dtype=dtype).element_size(),)).astype(np.uint8)).cuda()
        return t.view(dtype)[..., 0]

    if kind == "e4m3":      # codes and scales; a page of scales is a few odd bytes
        return [raw((L, P, page, H, d), torch.uint8), raw((L, P, page, H, d), torch.uint8),
                raw((L, P, page // 32, H), torch.uint8), raw((L, P, page // 32, H), torch.uint8)]
    if kind == "bf16":
        return [raw((L, P, page, H, d), torch.int16).view(torch.bfloat16) for _ in "kv"]
    if kind == "mla":       # one tensor of 576 channels
        return [raw((L, P, page, 1, 576), torch.int16).view(torch.bfloat16)]
    if kind == "f32 heads":  # [layer][head][page][slot][channel]
        return [raw((L, H, P, page, d), torch.int32).view(torch.float32).permute(0, 2, 3, 1, 4) for _ in "kv"]
    assert kind == "gaps"   # rows, heads and pages apart, at odd bytes
    return [raw((L, P + 1, page + 1, H + 1, d + 3), torch.uint8)[:, 1:, 1:, 1:, 3:]]


KINDS = ["e4m3", "bf16", "mla", "f32 heads", "gaps"]


def as_bytes(t):
    return t.contiguous().view(torch.uint8).cpu().numpy() if t.dtype != torch.uint8 else t.cpu().numpy()


def apply(before, copies, page):
    out = [b.copy() for b in before]
    for c in copies:
        for o, b in zip(out, before):
            n = -(-(c[2] if len(c) > 2 else page) * o.shape[2] // page)
            o[:, c[1], :n] = b[:, c[0], :n]
    return out


def check_tensors(ts, before, copies, page):
    for t, w in zip(ts, apply(before, copies, page)):
        np.testing.assert_array_equal(as_bytes(t), w)


def cuda(a):
    return torch.from_numpy(np.asarray(a)).cuda()


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("page", [32, 128])
@pytest.mark.parametrize("out_of_place", [False, True])
def test_fork(kind, page, out_of_place):
    rng = np.random.default_rng(page + len(kind))
    table, ref, lens = random_pool(rng, 7, 5, page, 30, [page * 2, 77, page * 5, 1, 0, page * 3 + 31, 4 * page])
    forks = [(0, 4, page * 2), (5, 1, page * 3 + 31), (5, 3, 40), (2, 6, page * 5 - 1), ]
    if out_of_place:
        forks = [(0, 1, page + 5), (1, 0, 77), (5, 5, page * 3 + 1), (5, 6, 0)]
    out = rng.integers(-1, 5, table.shape).astype(np.int32) if out_of_place else table
    ts = tensors(rng, len(ref), page, kind)
    before = [as_bytes(t) for t in ts]
    want_ref, want, copies, bad = R.fork(ref, table, out, forks, page, not out_of_place)
    assert not bad
    g_ref, g_in, flag = cuda(ref), cuda(table), torch.zeros(1, dtype=torch.int32, device="cuda")
    g_out = cuda(out) if out_of_place else g_in
    pkv.pages_fork(ts, g_ref, g_in, page, pkv.make_forks([dict(parent=a, child=b, n_tokens=n) for a, b, n in forks], "cuda"),
                   len(forks), block_table_out=g_out if out_of_place else None, err_flag=flag)
    torch.cuda.synchronize()
    np.testing.assert_array_equal(g_out.cpu().numpy(), want)
    np.testing.assert_array_equal(g_ref.cpu().numpy(), want_ref)
    check_tensors(ts, before, copies, page)
    assert int(flag.item()) == 0


@pytest.mark.parametrize("row,dtype", [(67, torch.uint8), (5, torch.int16), (64, torch.int32)])
def test_fork_tails_of_many_tiles(row, dtype):
    """Pages that lie in one piece in each layer and take many tiles there, in units of 1, 2 and 16 bytes; last pages of
    one slot, of one short of a page, and between."""
    rng = np.random.default_rng(row)
    page, L, H = 1024, 3, 3
    table, ref, lens = random_pool(rng, 8, 2, page, 12, [page + 1, page + 511, 2 * page - 1, page, 0, 0, 0, 0])
    forks = [(0, 4, page + 1), (1, 5, page + 511), (2, 6, 2 * page - 1), (3, 7, 300)]
    size = torch.empty(0, dtype=dtype).element_size()
    ts = [torch.from_numpy(rng.integers(0, 256, (L, len(ref), page, H, row, size)).astype(np.uint8)).cuda().view(dtype)[..., 0]]
    before = [as_bytes(t) for t in ts]
    want_ref, want, copies, bad = R.fork(ref, table, table, forks, page, True)
    assert not bad and len(copies) == 4
    g_ref, g = cuda(ref), cuda(table)
    pkv.pages_fork(ts, g_ref, g, page, pkv.make_forks([dict(parent=a, child=b, n_tokens=n) for a, b, n in forks], "cuda"), 4)
    torch.cuda.synchronize()
    np.testing.assert_array_equal(g.cpu().numpy(), want)
    check_tensors(ts, before, copies, page)


def test_fork_many():
    """More records than one round of the plan, over more pages than one round of its scan."""
    rng = np.random.default_rng(1)
    page, n, width = 32, 1500, 8
    table, ref, lens = random_pool(rng, 40, width, page, 0)
    table = np.concatenate([table, np.full((n, width), -1, np.int32)])
    ref = np.concatenate([ref, np.zeros(9000, np.int32)])
    ref[rng.permutation(9300)[:7000]] += 1
    forks = [(int(p), 40 + i, int(rng.integers(0, lens[p] + 1))) for i, p in enumerate(rng.integers(0, 40, n))]
    ts = tensors(rng, len(ref), page, "e4m3", L=1, H=1)
    before = [as_bytes(t) for t in ts]
    want_ref, want, copies, bad = R.fork(ref, table, table, forks, page, True)
    g_ref, g, flag = cuda(ref), cuda(table), torch.zeros(1, dtype=torch.int32, device="cuda")
    pkv.pages_fork(ts, g_ref, g, page, pkv.make_forks([dict(parent=a, child=b, n_tokens=m) for a, b, m in forks], "cuda"), n,
                   err_flag=flag)
    torch.cuda.synchronize()
    np.testing.assert_array_equal(g.cpu().numpy(), want)
    np.testing.assert_array_equal(g_ref.cpu().numpy(), want_ref)
    check_tensors(ts, before, copies, page)
    assert int(flag.item()) == int(bad)
    log("  %d forks, %d copies" % (n, len(copies)))


@pytest.mark.parametrize("what", ["parent", "child", "length", "negative", "twice", "chain", "full", "hole", "far entry"])
def test_fork_refused_records(what):
    rng = np.random.default_rng(2)
    page = 32
    table, ref, lens = random_pool(rng, 6, 4, page, 0 if what == "full" else 9, [100, 60, 33, 64, 0, 0])
    forks = {"parent": [(6, 4, 3), (0, 5, 99)], "child": [(0, -1, 3), (0, 5, 99)], "length": [(0, 4, 129), (0, 5, 99)],
             "negative": [(0, 4, -1), (0, 5, 99)], "twice": [(0, 4, 99), (1, 4, 60), (2, 5, 33)],
             "chain": [(0, 4, 99), (4, 5, 50), (1, 3, 60)], "full": [(0, 4, 99), (1, 5, 60)],
             "hole": [(1, 4, 120), (0, 5, 99)], "far entry": [(1, 4, 60), (0, 5, 99)]}[what]
    if what == "full":
        ref[np.nonzero(ref == 0)[0][1:]] = 1       # one page is left for two copies
    if what == "far entry":
        table[1, 1] = len(ref) + 2
    ts = tensors(rng, len(ref), page, "bf16")
    before = [as_bytes(t) for t in ts]
    want_ref, want, copies, bad = R.fork(ref, table, table, forks, page, True)
    assert bad
    g_ref, g, flag = cuda(ref), cuda(table), torch.zeros(1, dtype=torch.int32, device="cuda")
    pkv.pages_fork(ts, g_ref, g, page, pkv.make_forks([dict(parent=a, child=b, n_tokens=m) for a, b, m in forks], "cuda"),
                   len(forks), err_flag=flag)
    torch.cuda.synchronize()
    np.testing.assert_array_equal(g.cpu().numpy(), want)
    np.testing.assert_array_equal(g_ref.cpu().numpy(), want_ref)
    check_tensors(ts, before, copies, page)
    assert int(flag.item()) == 1


def test_free():
    rng = np.random.default_rng(3)
    page = 64
    table, ref, lens = random_pool(rng, 9, 300, page, 5, [300 * page, 5, 0, 64, 65, 1000, 19200, 7, 300])
    ts = tensors(rng, len(ref), page, "e4m3", L=1, H=1)
    for seqs, keep in (([0, 3], None), ([6, 5, 1], [64, 65, 0]), ([4, 4, 7, 4], [64, 0, -3, 70]), ([8], [10 ** 9]), ([], None)):
        want_ref, want, bad = R.free(ref, table, seqs, keep, page)
        g_ref, g, flag = cuda(ref), cuda(table), torch.zeros(1, dtype=torch.int32, device="cuda")
        pkv.pages_free(ts, g_ref, g, page, cuda(np.asarray(seqs, np.int32)),
                       None if keep is None else cuda(np.asarray(keep, np.int32)), err_flag=flag)
        torch.cuda.synchronize()
        np.testing.assert_array_equal(g.cpu().numpy(), want)
        np.testing.assert_array_equal(g_ref.cpu().numpy(), want_ref)
        assert int(flag.item()) == int(bad) == 0
        ref, table = want_ref, want
    table[8, 2], table[8, 3], table[8, 4] = len(ref), -7, int(np.nonzero(ref == 0)[0][0])
    for seqs in ([8], [9, 5], [-1]):
        want_ref, want, bad = R.free(ref, table, seqs, None, page)
        g_ref, g, flag = cuda(ref), cuda(table), torch.zeros(1, dtype=torch.int32, device="cuda")
        pkv.pages_free(ts, g_ref, g, page, cuda(np.asarray(seqs, np.int32)), err_flag=flag)
        torch.cuda.synchronize()
        np.testing.assert_array_equal(g.cpu().numpy(), want)
        np.testing.assert_array_equal(g_ref.cpu().numpy(), want_ref)
        assert bad and int(flag.item()) == 1


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("in_place", [False, True])
def test_compact(kind, in_place):
    rng = np.random.default_rng(4)
    page = 64
    table, ref, lens = random_pool(rng, 8, 6, page, 70)
    ts = tensors(rng, len(ref), page, kind)
    before = [as_bytes(t) for t in ts]
    want_ref, want, copies, n, bad = R.compact(ref, table)
    assert copies and not bad
    g_ref, g, flag = cuda(ref), cuda(table), torch.zeros(1, dtype=torch.int32, device="cuda")
    o_ref, o = (g_ref, g) if in_place else (torch.full_like(g_ref, 9), torch.full_like(g, 9))
    used = pkv.pages_compact(ts, g_ref, g, page, ref_out=o_ref, block_table_out=o, err_flag=flag)
    torch.cuda.synchronize()
    assert int(used.item()) == n and int(flag.item()) == 0
    np.testing.assert_array_equal(o.cpu().numpy(), want)
    np.testing.assert_array_equal(o_ref.cpu().numpy(), want_ref)
    check_tensors(ts, before, copies, page)


@pytest.mark.parametrize("P,used", [(1, 0), (1, 1), (2, 1), (8191, 4000), (20011, 9000), (64, 64), (64, 0)])
def test_compact_sizes(P, used):
    """Pools of one page, full and empty ones, and more pages than a round of the scan; entries of every kind."""
    rng = np.random.default_rng(P + used)
    ref = np.zeros(P, np.int32)
    ref[rng.permutation(P)[:used]] = rng.integers(1, 5, used)
    table = rng.integers(-3, P + 3, (50, 40)).astype(np.int32)
    ts = tensors(rng, P, 32, "e4m3", L=1, H=1)
    before = [as_bytes(t) for t in ts]
    want_ref, want, copies, n, bad = R.compact(ref, table)
    g_ref, g, flag = cuda(ref), cuda(table), torch.zeros(1, dtype=torch.int32, device="cuda")
    got = pkv.pages_compact(ts, g_ref, g, 32, err_flag=flag)
    torch.cuda.synchronize()
    assert int(got.item()) == n and int(flag.item()) == int(bad)
    np.testing.assert_array_equal(g.cpu().numpy(), want)
    np.testing.assert_array_equal(g_ref.cpu().numpy(), want_ref)
    check_tensors(ts, before, copies, 32)


def test_graph_of_free_fork_compact():
    """A captured step replayed on tables that change between the replays, each against the reference."""
    rng = np.random.default_rng(5)
    page = 32
    table, ref, lens = random_pool(rng, 10, 6, page, 60, [150, 33, 190, 64, 0, 0, 0, 0, 0, 0])
    ts = tensors(rng, len(ref), page, "e4m3")
    g_ref, g = cuda(ref), cuda(table)
    seqs = cuda(np.arange(4, 10, dtype=np.int32))
    forks = [(i % 4, 4 + i, lens[i % 4]) for i in range(6)]
    recs = pkv.make_forks([dict(parent=a, child=b, n_tokens=n) for a, b, n in forks], "cuda")
    used = torch.zeros(1, dtype=torch.int32, device="cuda")
    ws = [torch.empty(1 << 16, dtype=torch.uint8, device="cuda") for _ in range(2)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        pkv.pages_free(ts, g_ref, g, page, seqs)
        pkv.pages_fork(ts, g_ref, g, page, recs, len(forks), workspace=ws[0])
        pkv.pages_compact(ts, g_ref, g, page, n_used=used, workspace=ws[1])
    for step in range(4):
        before = [as_bytes(t) for t in ts]
        ref, table, _ = R.free(ref, table, range(4, 10), None, page)
        ref, table, copies, bad = R.fork(ref, table, table, forks, page, True)
        after = apply(before, copies, page)
        ref, table, moves, n, _ = R.compact(ref, table)
        assert not bad
        graph.replay()
        torch.cuda.synchronize()
        np.testing.assert_array_equal(g.cpu().numpy(), table)
        np.testing.assert_array_equal(g_ref.cpu().numpy(), ref)
        assert int(used.item()) == n
        check_tensors(ts, after, moves, page)
        # the host scatters the pool again: sequence 0 moves to the last pages
        ids = [p for p in range(len(ref) - 1, -1, -1) if ref[p] == 0][:5]
        for e, p in zip(range(5), ids):
            old = table[0, e]
            table[table == old] = p
            ref[p], ref[old] = ref[old], 0
            for t in ts:
                t[:, p] = t[:, int(old)].clone()
        g.copy_(cuda(table))
        g_ref.copy_(cuda(ref))


def test_offsets_past_32_bits():
    """Pages at the end of a pool of more than 4 GiB: a fork's copy and a compaction's moves."""
    P, page, H, d = 70000, 64, 8, 128
    pool = torch.empty((1, P, page, H, d), dtype=torch.uint8, device="cuda")
    rng = np.random.default_rng(60)
    body = torch.from_numpy(rng.integers(0, 256, (page, H, d)).astype(np.uint8)).cuda()
    pool[0, P - 1], pool[0, P - 2], pool[0, 0] = body, 0, 0
    ref = torch.ones(P, dtype=torch.int32, device="cuda")
    ref[P - 2] = 0
    table = torch.tensor([[P - 1, -1], [-1, -1]], dtype=torch.int32, device="cuda")
    pkv.pages_fork([pool], ref, table, page, pkv.make_forks([dict(parent=0, child=1, n_tokens=41)], "cuda"), 1)
    assert table.tolist() == [[P - 1, -1], [P - 2, -1]] and int(ref[P - 2]) == 1
    assert torch.equal(pool[0, P - 2, :41], body[:41]) and not pool[0, P - 2, 41:].any()
    ref[0] = 0
    used = pkv.pages_compact([pool], ref, table, page)[-1]
    assert table.tolist() == [[0, -1], [P - 2, -1]] and int(ref[P - 1]) == 0 and int(ref[0]) == 1 and int(used) == P - 1
    assert torch.equal(pool[0, 0], body)
