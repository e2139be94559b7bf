"""Attention over an 8-bit cache against the oracle on the dequantised keys and values, which bf16 holds exactly.
Tolerances as for the bf16 kernels: probabilities and outputs are each rounded to bf16 (2^-9 relative at most on
average, 2^-8 at worst: rel-L2 below 1e-2), values are of unit size (max-abs 2e-2, mean-abs 2e-3)."""
import math

import numpy as np
import pytest
import torch

import quant_ref as R
from helpers import Guarded, check_attention_close, dev, host_bits, log
from paper_2606_17107_amd import pkv, synth

pytestmark = pytest.mark.gpu


class Cache:
    """Random codes of unit size under scales that differ from block to block, every slot of the pool filled."""

    def __init__(self, L, Hkv, d, page, block, lens, seed, extra=4, width=None):
        rng = np.random.default_rng(seed)
        width = width or max(1, max(-(-n // page) for n in lens))
        self.P = len(lens) * width + extra
        self.table = rng.permutation(self.P)[: len(lens) * width].reshape(len(lens), width).astype(np.int32)
        self.vtable = None
        self.ks, self.vs = (rng.integers(119, 123, (L, self.P, page // block, Hkv)).astype(np.uint8) for _ in "kv")
        self.k, self.v = (self.fill(rng, (L, self.P, page, Hkv, d), s) for s in (self.ks, self.vs))
        self.lens, self.page, self.block = lens, page, block

    @staticmethod
    def fill(rng, shape, scale):
        e = np.repeat(scale, shape[2] // scale.shape[2], axis=2)[..., None]
        x = rng.normal(size=shape).astype(np.float32) * np.exp2(127.0 - e).astype(np.float32)
        return torch.from_numpy(np.clip(x, -448, 448)).to(torch.float8_e4m3fn).view(torch.uint8).numpy()


def run(c, H, nqs, scale=None, splits=0, window=0, q_pos=None, max_kv=None, lse=True, pools=None, seed=5, cu=None, rows=None,
        cache_slots=None, gain=1.5):
    """The call, guarded, and the oracle: returns (output bits, log-sum-exps) after the comparison."""
    L, d = c.k.shape[0], c.k.shape[4]
    scale = 1 / math.sqrt(d) if scale is None else scale
    rows = sum(nqs) if rows is None else rows
    q = host_bits(synth.Draws(seed, "cpu").normal((L, rows, H, d)) * gain)
    starts = np.concatenate([[0], np.cumsum(nqs)]) if cu is None else np.asarray(cu)
    if q_pos is None:
        q_pos = np.zeros(rows, np.int64)
        for s, n in enumerate(nqs):
            q_pos[starts[s]:starts[s] + n] = np.arange(c.lens[s] - n, c.lens[s])
    q_pos = q_pos.astype(np.int32)
    k, v, ks, vs = (torch.from_numpy(t).cuda() for t in (c.k, c.v, c.ks, c.vs)) if pools is None else pools
    out = Guarded((L, rows, H, d), torch.bfloat16)
    lse_t = torch.full((L, rows, H), 7.0, device="cuda") if lse else None
    table = torch.from_numpy(c.table).cuda()
    vt = None if c.vtable is None else torch.from_numpy(c.vtable).cuda()
    pkv.suffix_attention_quant(dev(q), k, v, ks, vs, out.t, torch.from_numpy(q_pos).cuda(),
                               torch.tensor(c.lens, dtype=torch.int32, device="cuda"), table, scale,
                               max_kv_len=max(c.lens) if max_kv is None else max_kv, n_seqs=len(c.lens),
                               cu_q=torch.from_numpy(starts.astype(np.int32)).cuda() if len(c.lens) > 1 or cu is not None else None,
                               max_q=max(nqs), n_splits=splits, lse_out=lse_t, window=window, cache_slots=cache_slots,
                               v_block_table=vt)
    torch.cuda.synchronize()
    out.check("attention output")
    got = host_bits(out.t)
    stats = None
    for l in range(L):
        for s, n in enumerate(nqs):
            if n == 0:
                continue
            at = slice(starts[s], starts[s] + n)
            kv = min(c.lens[s], max(c.lens) if max_kv is None else max_kv)
            if kv == 0:
                assert not got[l, at].any()
                continue
            want, want_lse = R.attention(q[l, at], c.k[l], c.v[l], c.ks[l], c.vs[l], c.table[s],
                                         (c.table if c.vtable is None else c.vtable)[s], q_pos[at], kv, scale, window)
            stats = check_attention_close(got[l, at], want)
            if lse:
                np.testing.assert_allclose(lse_t.cpu().numpy()[l, at], want_lse, atol=2e-2)
    log("  ", stats)
    return out, lse_t


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("page,block", [(32, 32), (64, 32), (128, 128), (256, 64)])
def test_suffix(d, page, block):
    """Many rows a KV head, in one pass and in splits."""
    c = Cache(2, 2, d, page, block, [731], seed=d + page)
    for splits in (0, 1, 3):
        run(c, 8, [45], splits=splits)


@pytest.mark.parametrize("G", [1, 4, 7, 32])
@pytest.mark.parametrize("d", [64, 128])
def test_one_token(d, G):
    """Few rows: whole items, cut items, ragged lengths down to one slot."""
    run(Cache(1, 2, d, 64, 64, [500], seed=G), 2 * G, [1])
    run(Cache(2, 2, d, 32, 32, [3001], seed=G + 1), 2 * G, [1])
    run(Cache(1, 2, d, 64, 32, [1, 33, 5000, 64, 900], seed=G + 2), 2 * G, [1] * 5)


def test_few_rows_long_and_many_sequences():
    """Scale windows of 64 tiles a wave move on; 64 sequences; up to 32 rows."""
    run(Cache(1, 1, 64, 32, 32, [40000], seed=21), 4, [3])
    run(Cache(1, 1, 128, 32, 32, [70000], seed=22), 8, [1])
    lens = [int(n) for n in np.random.default_rng(23).integers(1, 2500, 64)]
    run(Cache(1, 2, 64, 64, 64, lens, seed=24), 8, [1] * 64)
    run(Cache(1, 2, 128, 64, 64, lens[:20], seed=25), 8, [min(8, n) for n in lens[:20]])


@pytest.mark.parametrize("d", [64, 128])
def test_many_rows_long(d):
    """More than 256 tiles in one pass: the scale window moves on in the pipelined loop and in the masked one."""
    run(Cache(1, 1, d, 32, 32, [9300], seed=26), 4, [40], splits=1)
    run(Cache(1, 1, d, 64, 64, [9300], seed=27), 4, [40], splits=1, window=8700)


@pytest.mark.parametrize("window", [1, 50, 700])
@pytest.mark.parametrize("nq", [1, 40])
def test_window(window, nq):
    c = Cache(1, 2, 128, 32, 32, [1500], seed=28)
    for splits in (0, 1, 2):
        run(c, 8, [nq], splits=splits, window=window)


def test_ragged_prefill():
    """Sequences of every size in one call; enough of them that the longest are dispatched first."""
    lens = [300, 1000, 77, 513, 1, 2048, 64, 32]
    nqs = [17, 40, 77, 64, 1, 300, 5, 32]
    run(Cache(2, 2, 128, 64, 32, lens, seed=29), 8, nqs)
    lens = [int(n) for n in np.random.default_rng(30).integers(1500, 3000, 24)]
    run(Cache(1, 8, 64, 64, 64, lens, seed=31), 16, [130] * 24)


def test_rows_that_see_nothing():
    """Empty caches, positions before the cache, windows past its end: zeros and -inf.  Rows that no sequence owns are
    left as they were."""
    c = Cache(1, 2, 128, 32, 32, [0, 100, 64], seed=32, width=4)
    for splits in (0, 1):
        out, lse = run(c, 8, [3, 2, 4], splits=splits, cu=[2, 5, 7, 11], rows=13, max_kv=100,
                       q_pos=np.array([0, 0, -1, 0, 5, 98, 99, 60, 61, 62, 63, 0, 0]))
        assert out.untouched((slice(None), [0, 1, 11, 12])) and bool((lse[:, [0, 1, 11, 12]] == 7.0).all())
        assert bool((lse[:, 2:5] == -math.inf).all())
    c = Cache(1, 2, 64, 32, 32, [70], seed=33)
    for nq in (3, 40):
        pos = np.full(nq, -5)
        pos[1] = 10 ** 9
        out, lse = run(c, 8, [nq], q_pos=pos, window=20, lse=False)
        assert not host_bits(out.t).any()


@pytest.mark.parametrize("nq,H,kv", [(1, 8, 900), (1, 8, 300), (4, 8, 2000), (40, 8, 500), (130, 2, 300)])
@pytest.mark.parametrize("d", [64, 128])
def test_unseen_slots_do_not_matter(nq, H, kv, d):
    """NaN codes behind the length, and in keys and values of slots that only later queries see: earlier rows are
    bit for bit what they are without them, later rows NaN exactly where the value channel is."""
    c = Cache(1, 2, d, 64, 32, [kv], seed=34)
    kw = dict(splits=0, lse=True)
    out, lse = run(c, H, [nq], **kw)
    base = host_bits(out.t)
    slots = np.arange(c.table.shape[1] * 64)
    ids, at = c.table[0][slots // 64], slots % 64
    pools = [torch.from_numpy(t.copy()).cuda() for t in (c.k, c.v, c.ks, c.vs)]
    tail = torch.from_numpy(slots >= kv)
    for p in pools[:2]:
        p[:, torch.from_numpy(ids).long()[tail], torch.from_numpy(at)[tail]] = 0x7f
    out, lse2 = run(c, H, [nq], pools=pools, **kw)
    np.testing.assert_array_equal(host_bits(out.t), base)
    assert torch.equal(lse, lse2)
    if nq < 4:
        return
    hidden = kv - nq + nq // 2           # the first query that sees it is nq // 2
    pools[1][0, ids[hidden], at[hidden], 0, 3] = 0xff
    q = synth.Draws(5, "cpu").normal((1, nq, H, d)) * 1.5
    got = Guarded((1, nq, H, d), torch.bfloat16)
    pkv.suffix_attention_quant(q.cuda(), *pools, got.t, torch.arange(kv - nq, kv, dtype=torch.int32, device="cuda"),
                               torch.tensor([kv], dtype=torch.int32, device="cuda"), torch.from_numpy(c.table).cuda(),
                               1 / math.sqrt(d), max_kv_len=kv)
    torch.cuda.synchronize()
    x = got.t.float().cpu()
    G = H // 2
    nan = torch.zeros_like(x, dtype=torch.bool)
    nan[0, nq // 2:, :G, 3] = True
    assert torch.equal(torch.isnan(x), nan)
    same = host_bits(got.t)
    np.testing.assert_array_equal(same[0, : nq // 2], base[0, : nq // 2])
    np.testing.assert_array_equal(same[0, :, G:], base[0, :, G:])
    pools[1][0, ids[hidden], at[hidden], 0, 3] = 0
    pools[0][0, ids[hidden], at[hidden], 1, 0] = 0x7f          # a NaN key of KV head 1
    pkv.suffix_attention_quant(q.cuda(), *pools, got.t, torch.arange(kv - nq, kv, dtype=torch.int32, device="cuda"),
                               torch.tensor([kv], dtype=torch.int32, device="cuda"), torch.from_numpy(c.table).cuda(),
                               1 / math.sqrt(d), max_kv_len=kv)
    torch.cuda.synchronize()
    x = got.t.float().cpu()
    assert bool(torch.isnan(x[0, nq // 2:, G:]).all()) and not bool(torch.isnan(x[0, : nq // 2]).any())


def test_scales_of_the_softmax():
    """Negative, zero and large softmax scales; sharp rows."""
    c = Cache(1, 2, 128, 32, 32, [700], seed=35)
    for nq in (1, 40):
        for s in (-0.1, 0.0, 0.5):
            run(c, 8, [nq], scale=s)


def test_far_apart_block_scales():
    """Blocks whose scales differ by 2^40: the large ones decide, nothing overflows."""
    c = Cache(1, 1, 64, 32, 32, [400], seed=36)
    c.vs[:] = np.where(np.arange(c.vs.size).reshape(c.vs.shape) % 2, 101, 121)
    c.ks[:, ::3] = 90
    for nq in (1, 40):
        run(c, 4, [nq])


def test_strides_and_tables():
    """Pools with room between rows, head-major pools, values through their own table, entries outside the pool
    (clamped into it) and tables wider than the cache."""
    c = Cache(2, 2, 128, 64, 32, [700], seed=37, width=20)
    wide = [torch.zeros(t.shape[:-1] + (160,), dtype=torch.uint8, device="cuda") for t in (c.k, c.v)]
    for a, t in zip(wide, (c.k, c.v)):
        a[..., :128] = torch.from_numpy(t).cuda()
    scales = [torch.from_numpy(np.ascontiguousarray(t.transpose(0, 3, 1, 2))).cuda().permute(0, 2, 3, 1) for t in (c.ks, c.vs)]
    heads = [torch.from_numpy(np.ascontiguousarray(t.transpose(0, 3, 1, 2, 4))).cuda().permute(0, 2, 3, 1, 4) for t in (c.k, c.v)]
    for nq in (1, 50):
        run(c, 8, [nq], pools=[wide[0][..., :128], wide[1][..., :128]] + scales)
        run(c, 8, [nq], pools=heads + scales)
    c.vtable = np.roll(c.table, 3, axis=1)
    for nq in (1, 50):
        run(c, 8, [nq])
    c.table[0, 2], c.table[0, 4] = -9, c.P + 50
    pools = [torch.from_numpy(t).cuda() for t in (c.k, c.v, c.ks, c.vs)]
    clamped = np.clip(c.table, 0, c.P - 1)
    for nq in (1, 50):
        outs = []
        for t in (c.table, clamped):
            q = synth.Draws(6, "cuda").normal((2, nq, 8, 128))
            out = torch.zeros_like(q)
            pkv.suffix_attention_quant(q, *pools, out, torch.arange(700 - nq, 700, dtype=torch.int32, device="cuda"),
                                       torch.tensor([700], dtype=torch.int32, device="cuda"), torch.from_numpy(t).cuda(),
                                       0.1, max_kv_len=700)
            outs.append(out)
        torch.cuda.synchronize()
        assert torch.equal(*outs)


def test_many_sequences():
    """More than 64 sequences (the many-row kernel with one query each)."""
    lens = [int(n) for n in np.random.default_rng(38).integers(1, 400, 90)]
    run(Cache(1, 2, 64, 32, 32, lens, seed=39), 8, [1] * 90)


def test_large_pool_offsets():
    """Pages beyond 2^32 bytes of the pool."""
    page, H, d = 64, 8, 128
    P = (1 << 32) // (page * H * d) + 40
    k = torch.zeros((1, P, page, H, d), dtype=torch.uint8, device="cuda")
    v = torch.zeros_like(k)
    ks = torch.full((1, P, 2, H), 121, dtype=torch.uint8, device="cuda")
    vs = torch.full_like(ks, 120)
    c = Cache(1, H, d, page, 32, [600], seed=40, extra=0)
    far = np.array([P - 1 - i for i in range(c.table.shape[1])], np.int32)
    for t, s in ((k, c.k), (v, c.v), (ks, c.ks), (vs, c.vs)):
        t[:, torch.from_numpy(far).long().cuda()] = torch.from_numpy(np.ascontiguousarray(s[:, c.table[0]])).cuda()
    table = torch.from_numpy(far[None]).cuda()
    for nq in (1, 50):
        outs = []
        for pools, t in (([k, v, ks, vs], table), ([torch.from_numpy(x).cuda() for x in (c.k, c.v, c.ks, c.vs)],
                                                   torch.from_numpy(c.table).cuda())):
            q = synth.Draws(7, "cuda").normal((1, nq, 32, d))
            out = torch.zeros_like(q)
            pkv.suffix_attention_quant(q, *pools, out, torch.arange(600 - nq, 600, dtype=torch.int32, device="cuda"),
                                       torch.tensor([600], dtype=torch.int32, device="cuda"), t, 0.09, max_kv_len=600)
            outs.append(out)
        torch.cuda.synchronize()
        assert torch.equal(*outs)


def test_nothing_to_do():
    c = Cache(1, 2, 64, 32, 32, [0], seed=41)
    run(c, 4, [2], max_kv=0)
    q = torch.zeros(1, 0, 4, 64, dtype=torch.bfloat16, device="cuda")
    pools = [torch.from_numpy(x).cuda() for x in (c.k, c.v, c.ks, c.vs)]
    none = torch.zeros(0, dtype=torch.int32, device="cuda")
    pkv.suffix_attention_quant(q, *pools, torch.zeros_like(q), none, torch.zeros(1, dtype=torch.int32, device="cuda"),
                               torch.from_numpy(c.table).cuda(), 1.0, max_kv_len=0)
    torch.cuda.synchronize()


@pytest.mark.parametrize("nq", [1, 40])
def test_side_stream_and_graph(nq):
    c = Cache(1, 2, 128, 64, 64, [3000], seed=42)
    pools = [torch.from_numpy(x).cuda() for x in (c.k, c.v, c.ks, c.vs)]
    q = synth.Draws(8, "cuda").normal((1, nq, 8, 128))
    pos = torch.arange(3000 - nq, 3000, dtype=torch.int32, device="cuda")
    kv, table = torch.tensor([3000], dtype=torch.int32, device="cuda"), torch.from_numpy(c.table).cuda()

    def call(out, **kw):
        pkv.suffix_attention_quant(q, *pools, out, pos, kv, table, 0.09, max_kv_len=3000, **kw)

    want, got = torch.zeros_like(q), torch.zeros_like(q)
    call(want)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    call(got, stream=side)
    side.synchronize()
    assert torch.equal(got, want)
    desc = pkv.make_attn_desc_quant(q, pools[0], pools[1], got, table, 3000)
    ws = torch.empty(max(16, pkv.pkv_attention_quant_workspace_size(desc, 8, 2, 128)), dtype=torch.uint8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(got, workspace=ws)
    for n in (3000, 1234, 2999):
        q.mul_(-1.0)
        kv.fill_(n)
        graph.replay()
        call(want)
        torch.cuda.synchronize()
        assert torch.equal(got, want), n
