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


def meant(e):
    """The scale byte that a stored one counts as."""
    return np.clip(e, 1, TOP)


def attend(q, pools, q_pos, kv, window=0, splits=0, table=None, n=1):
    table = torch.tensor([list(range(pools[0].shape[1]))], dtype=torch.int32, device="cuda") if table is None else table
    out = torch.full_like(q, 3.0)
    lse = torch.zeros(q.shape[:3], device="cuda")
    pkv.suffix_attention_quant(q, *pools, out, torch.as_tensor(q_pos, dtype=torch.int32, device="cuda"),
                               torch.tensor([kv], dtype=torch.int32, device="cuda"), table, 1 / 8, max_kv_len=kv, window=window,
                               n_splits=splits, lse_out=lse)
    torch.cuda.synchronize()
    return out.cpu(), lse.cpu()


@pytest.mark.parametrize("nq", [1, 45])
@pytest.mark.parametrize("d", [64, 128])
def test_every_code_under_every_scale_byte(d, nq):
    """One slot in use whose value channels are all codes, the tile's other slots full of the largest one: the output is
    the value itself, as bf16 rounds it (the codes of bytes 1 and 2 fall between bf16's steps; below its normal numbers,
    2^-126, a result may also be 0)."""
    L, H = 256, 256 // d
    pools = [torch.zeros((L, 1, 32, H, d), dtype=torch.uint8, device="cuda") for _ in "kv"]
    pools[1][:] = 0x7e
    codes = np.arange(256).astype(np.uint8).reshape(H, d)
    pools[1][:, 0, 0] = torch.from_numpy(codes).cuda()
    scales = [torch.arange(256, dtype=torch.uint8, device="cuda").reshape(L, 1, 1, 1).repeat(1, 1, 1, H) for _ in "kv"]
    q = synth.Draws(62, "cuda").normal((L, nq, 2 * H, d))
    out, _ = attend(q, pools + scales, [0] * nq, 1)
    want = R.decode(codes[None], meant(np.arange(256))[:, None, None])                # [L, H, d]
    rounded = torch.from_numpy(want).to(torch.bfloat16).double().numpy()
    exact = np.arange(256) >= 3
    np.testing.assert_array_equal(rounded[exact], want[exact])
    got = out.double().numpy().reshape(L, nq, H, 2, d)
    rounded = np.broadcast_to(rounded[:, None, :, None], got.shape)
    small = np.abs(rounded) < 2.0 ** -126
    np.testing.assert_array_equal(got[~small], rounded[~small])
    assert ((got[small] == rounded[small]) | (got[small] == 0)).all()


@pytest.mark.parametrize("byte", [0, 246, 247, 254, 255])
@pytest.mark.parametrize("nq,kv,splits", [(1, 70, 0), (4, 2050, 0), (8, 300, 0), (45, 300, 0), (45, 300, 1), (130, 2050, 3)])
@pytest.mark.parametrize("d", [64, 128])
def test_unseen_slots_under_any_scale(d, nq, kv, splits, byte):
    """The largest codes, and NaN, in slots that a row does not see, in a block whose scale makes them infinite in bf16
    (or is no scale at all): the rows are bit for bit what they are without them.  Behind the length, and behind a
    query's own position."""
    page, H, G = 64, 2, 4
    pages = -(-kv // page)
    g = torch.Generator(device="cuda").manual_seed(kv + nq)
    pools = [torch.randint(0, 0x48, (1, pages, page, H, d), dtype=torch.uint8, device="cuda", generator=g) for _ in "kv"]
    scales = [torch.full((1, pages, page // 32, H), 122, dtype=torch.uint8, device="cuda") for _ in "kv"]
    hidden = kv - nq + nq // 2               # queries before nq // 2 do not see it
    first = hidden // 32                     # its block and those behind it get the byte, the slots in use codes of 0
    for t in scales:
        t.view(1, -1, H)[:, first:] = byte
    flat = [t.view(1, -1, H, d) for t in pools]
    for t in flat:
        t[:, first * 32:] = 0
    q = synth.Draws(63, "cuda").normal((1, nq, G * H, d))
    pos = np.arange(kv - nq, kv)
    want, want_lse = attend(q, pools + scales, pos, kv, splits=splits)
    assert bool(torch.isfinite(want.float()).all())
    start = kv if nq == 1 else hidden
    for codes in (0x7e, 0xfe, 0x7f, 0x78):
        for t in flat:
            t[:, start:] = codes
        got, lse = attend(q, pools + scales, pos, kv, splits=splits)
        rows = nq if start == kv else nq // 2
        assert torch.equal(got[:, :rows], want[:, :rows]), hex(codes)
        assert torch.equal(lse[:, :rows], want_lse[:, :rows]), hex(codes)


@pytest.mark.parametrize("nq", [4, 45])
@pytest.mark.parametrize("d", [64, 128])
def test_blocks_that_no_row_sees(d, nq):
    """Blocks between the windows of queries far apart hold anything: codes, scale bytes and table entries."""
    page, H, G, kv, window = 32, 2, 4, 1400, 40
    pages = -(-kv // page)
    g = torch.Generator(device="cuda").manual_seed(nq)
    pools = [torch.randint(0, 0x48, (1, pages, page, H, d), dtype=torch.uint8, device="cuda", generator=g) for _ in "kv"]
    scales = [torch.full((1, pages, 1, H), 122, dtype=torch.uint8, device="cuda") for _ in "kv"]
    pos = np.where(np.arange(nq) % 2, 1390 - np.arange(nq), 60 + np.arange(nq))
    q = synth.Draws(64, "cuda").normal((1, nq, G * H, d))
    for splits in (0, 1):
        want, want_lse = attend(q, pools + scales, pos, kv, window=window, splits=splits)
        seen = np.zeros(pages * page, bool)
        for p in pos:
            seen[max(0, p - window + 1): p + 1] = True
        free = torch.from_numpy(np.nonzero(~seen.reshape(pages, page).any(1))[0]).cuda()
        assert len(free) > 20
        other = [t.clone() for t in pools + scales]
        for t in other[:2]:
            t[:, free] = torch.randint(0, 256, t[:, free].shape, dtype=torch.uint8, device="cuda", generator=g)
        for byte in (0, 250, 255):
            for t in other[2:]:
                t[:, free] = byte
            got, lse = attend(q, other, pos, kv, window=window, splits=splits)
            assert torch.equal(got, want) and torch.equal(lse, want_lse), byte


@pytest.mark.parametrize("old", [0, 1, 246, 250, 255])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_kept_rows_under_any_scale_byte(dtype, old):
    """Rows spliced into a block that keeps rows under `old`: it counts as the nearest byte that is written."""
    d = 64
    x = synth.Draws(65, "cpu").normal((1, 1, 5, d), torch.float32) * (2.0 ** -100 if old < 2 else 1.0)
    x = x.to(torch.bfloat16 if dtype == "bf16" else torch.float32)
    (k, v, ks, vs), row = call_splice(x, x, 0, None, old=old, kv_len=20, at=20)
    rows = x[0, 0].double().numpy()
    e, codes = expected(rows, int(meant(old)))
    for pool, scale in ((k, ks), (v, vs)):
        assert meant(scale[0, row[0], 0, 0]) == e
        R.check_codes(pool[0, row[0], 20:25, 0], codes, codes, codes)
        kept = R.encode(np.full((20, d), R.VALUES[0x11]) * 2.0 ** float(int(meant(old)) - e))
        np.testing.assert_array_equal(pool[0, row[0], :20, 0], kept)
        assert (pool[0, row[0], 25:32, 0] == 0x11).all()
