"""NaN, infinities and subnormals through every form of the 8-bit cache's splice, and NaN codes on both sides of a
window in its attention."""
import math

import numpy as np
import pytest
import torch

import quant_ref as R
from helpers import host_bits
from paper_2606_17107_amd import pkv, synth
from test_gpu_quant_attention import Cache
from test_gpu_quant_range import call_splice, expected
from test_gpu_quant_splice import HALF, INTER, Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("style", [HALF, INTER])
@pytest.mark.parametrize("delta", [0, 13])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
def test_nonfinite_rows(d, dtype, delta, style):
    """A turned pair with a NaN or an infinity is NaN where the formula makes it so; block scales come from the finite
    values alone, in blocks with and without infinities, and in one without any finite value."""
    c = Case(L=2, d=d, dtype=dtype, seed=70 + delta)
    for t in (c.src_k, c.src_v):
        t[0, 0, 3, 5], t[0, 0, 4, 6], t[0, 1, 9, d - 1] = float("nan"), float("inf"), float("-inf")
        t[1, 0, 2], t[1, 0, 33, 1] = float("inf"), float("nan")
        t[0, 0, 62:94] = float("nan")       # slots 64 .. 95
        t[1, 1, 62:94] = float("-inf")
    c.kv_len[0] = 2
    c.run([(0, 0, 130, 2 - delta, 2)], style=style)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("block", [32, 128])
def test_kept_nan_codes_under_a_growing_scale(block, dtype):
    c = Case(page=128, block=block, dtype=dtype, seed=72)
    rng = np.random.default_rng(72)
    for t in (c.k, c.v):
        t[rng.random(t.shape) < 0.05] = 0x7f
        t[rng.random(t.shape) < 0.05] = 0xff
    for t in (c.ks, c.vs):
        t[:] = rng.integers(80, 130, t.shape)     # blocks that grow by much, by little, and not at all
    c.kv_len[0] = 300
    c.run([(0, 0, 30, 5, 20), (50, 0, 1, 0, 130), (60, 0, 7, 200, 200)])


@pytest.mark.parametrize("delta", [0, 5])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_subnormal_sources(dtype, delta):
    """Values below the smallest normal number are stored like any others.  (There the rotation's products round to
    multiples of 2^-149: three roundings, 1.5 * 2^-149, beside the relative bound.)"""
    d, n = 64, 64
    x = synth.Draws(73, "cpu").normal((1, 1, n, d), torch.float32).double()
    x = (x * torch.logspace(-133, -118, n, 2, dtype=torch.float64)[:, None]).to(torch.bfloat16 if dtype == "bf16" else torch.float32)
    assert int(((x.double().abs() < 2.0 ** -126) & (x != 0)).sum()) > 1000
    omega = 1e4 ** (-2.0 * np.arange(d // 2) / d)
    (k, v, ks, vs), row = call_splice(x, x, delta, list(omega), block=32)
    for pool, scale, turn in ((k, ks, delta), (v, vs, 0)):
        y, err = R.turned(x[0, 0].double().numpy(), turn, omega, 0, 0)
        err = err + (1.5 * 2.0 ** -149 if turn else 0.0)
        for b in range(n // 32):
            rows, off = y[b * 32:(b + 1) * 32], err[b * 32:(b + 1) * 32]
            e, codes = expected(rows)
            lo, hi = (R.encode(z * 2.0 ** (127 - e)) for z in (rows - off, np.clip(rows + off, None, 448 * 2.0 ** (e - 127))))
            assert scale[0, row[0], b, 0] == e
            R.check_codes(pool[0, row[0], b * 32:(b + 1) * 32, 0], codes, lo, hi)


@pytest.mark.parametrize("splits", [0, 1, 2])
@pytest.mark.parametrize("nq,window,kv", [(4, 100, 1500), (8, 33, 300), (40, 100, 1500), (130, 500, 2300)])
@pytest.mark.parametrize("d", [64, 128])
def test_nan_values_in_front_of_a_window(d, nq, window, kv, splits):
    """A NaN value code in a slot that only the earlier queries' windows reach, and NaN codes in keys and values that no
    window reaches: NaN in those rows and that channel, every other output bit for bit as without."""
    c = Cache(1, 2, d, 64, 32, [kv], seed=74)
    H, G = 8, 4
    table = torch.from_numpy(c.table).cuda()
    pools = [torch.from_numpy(t.copy()).cuda() for t in (c.k, c.v, c.ks, c.vs)]
    q = synth.Draws(75, "cuda").normal((1, nq, H, d)) * 1.5
    pos = torch.arange(kv - nq, kv, dtype=torch.int32, device="cuda")

    def call():
        out, lse = torch.full_like(q, 9.0), torch.zeros(1, nq, H, device="cuda")
        pkv.suffix_attention_quant(q, *pools, out, pos, torch.tensor([kv], dtype=torch.int32, device="cuda"), table, 1 / math.sqrt(d),
                                   max_kv_len=kv, window=window, n_splits=splits, lse_out=lse)
        torch.cuda.synchronize()
        return out, lse

    def at(slot):
        return int(c.table[0][slot // 64]), slot % 64

    want, want_lse = call()
    for slot in range(max(0, kv - nq - window - 40), kv - nq - window + 1):       # before the first window
        page, i = at(slot)
        pools[0][:, page, i], pools[1][:, page, i] = 0x7f, 0xff
    got, lse = call()
    assert torch.equal(got, want) and torch.equal(lse, want_lse)
    page, i = at(kv - nq + nq // 2 - window)       # seen by queries before nq // 2
    pools[1][0, page, i, 1, 3] = 0x7f
    got, lse = call()
    nan = torch.zeros_like(want, dtype=torch.bool)
    nan[0, : nq // 2, G:, 3] = True
    assert torch.equal(torch.isnan(got), nan) and torch.equal(lse, want_lse)
    np.testing.assert_array_equal(host_bits(got)[~nan.cpu().numpy()], host_bits(want)[~nan.cpu().numpy()])
    pools[1][0, page, i, 1, 3] = 0
    pools[0][0, page, i, 0, 5] = 0xff              # a NaN key: whole rows of KV head 0
    got, lse = call()
    assert bool(torch.isnan(got[0, : nq // 2, :G]).all()) and bool(torch.isnan(lse[0, : nq // 2, :G]).all())
    assert not bool(torch.isnan(got[0, nq // 2:]).any()) and not bool(torch.isnan(got[0, :, G:]).any())
