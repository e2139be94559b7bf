"""The ends of the 8-bit cache's range: the largest finite inputs, scale bytes of every value, and codes that only a
block's scale makes large."""
import numpy as np
import pytest
import torch

import quant_ref as R
from paper_2606_17107_amd import pkv, synth

pytestmark = pytest.mark.gpu

TOP = 246                              # largest scale byte that is written
LIMIT = 448.0 * 2.0 ** (TOP - 127)     # largest magnitude that is stored


def expected(x, kept=0):
    """Scale byte and codes of one block's rows (`kept`: old byte where the block keeps a row)."""
    v = np.abs(x[np.isfinite(x)])
    e = max(min(R.need(min(v.max(initial=0.0), LIMIT)), TOP), kept)
    with np.errstate(invalid="ignore"):
        return e, R.encode(np.clip(x, -LIMIT, LIMIT, where=np.isfinite(x), out=x.copy()) * 2.0 ** (127 - e))


def call_splice(src_k, src_v, delta, omega, page=64, block=32, old=None, kv_len=0, at=0):
    """Rows of the sources at slots `at` .. of one sequence; returns pools and scales as numpy."""
    L, H, n, d = src_k.shape
    P = 4
    pools = [torch.full((L, P, page, H, d), 0x11, dtype=torch.uint8, device="cuda") for _ in "kv"]
    scales = [torch.full((L, P, page // block, H), 100 if old is None else old, dtype=torch.uint8, device="cuda") for _ in "kv"]
    table = torch.tensor([[2, 0, 3]], dtype=torch.int32, device="cuda")
    seg = pkv.make_segments_quant([dict(src_slot0=0, seq=0, n_tokens=n, src_pos0=at - delta, dst_pos0=at)], "cuda")
    pkv.reposition_splice_quant(src_k.cuda(), src_v.cuda(), *pools, *scales, seg, 1, n,
                                torch.tensor([kv_len], dtype=torch.int32, device="cuda"), table, 1e4, d, omega=omega)
    torch.cuda.synchronize()
    return [t.cpu().numpy() for t in pools + scales], table.cpu().numpy()[0]


@pytest.mark.parametrize("block", [32, 64])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("delta", [0, 7])
@pytest.mark.parametrize("d", [64, 128])
def test_largest_finite_inputs(d, delta, dtype, block):
    """Finite values beyond 448 * 2^119 are stored as it, beside NaN, infinities and ordinary values; so the stored values
    are finite in bf16.  (Frequencies of 0: moved rows go through the rotation and come out as they were.)"""
    L, H, n = 1, 2, 70
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    src = synth.Draws(61, "cpu").normal((2, L, H, n, d), torch.float32) * 2.0 ** 125
    big = [3.3895313892515355e38, -3.3895313892515355e38, LIMIT, 464 * 2.0 ** 119, -466 * 2.0 ** 119, 2.0 ** 127,
           float("nan"), float("inf"), float("-inf"), 3.0e38, -3.2e38, 2.0 ** 119, -2.0 ** 110]
    for t in range(0, n, 3):
        for i, x in enumerate(big):
            src[:, :, :, t, (5 * t + 7 * i) % d] = x
    src = src.to(dt)
    (k, v, ks, vs), row = call_splice(src[0], src[1], delta, [0.0] * (d // 2), block=block)
    for pool, scale, x, turn in ((k, ks, src[0], delta), (v, vs, src[1], 0)):
        x = R.turned(x.double().numpy(), turn, np.zeros(d // 2), 0, 0)[0]     # (0 * inf is NaN)
        for h in range(H):
            for b in range(-(-n // block)):
                rows = x[0, h, b * block:(b + 1) * block]
                e, codes = expected(rows)
                assert e == TOP
                slots = np.arange(b * block, b * block + len(rows))
                got = pool[0, row[slots // 64], slots % 64, h]
                assert scale[0, row[b * block // 64], b * block % 64 // block, h] == e
                R.check_codes(got, codes, codes, codes)
                stored = R.decode(got, np.uint8(e))
                assert np.array_equal(np.isfinite(stored), np.isfinite(rows))
                assert np.nanmax(np.abs(stored)) <= 255 * 2.0 ** 120      # bf16's largest finite value
