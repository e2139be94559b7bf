"""The 8-bit references themselves (CPU): the E4M3 table against torch's, rounding to the nearest with ties to
even at every midpoint, and the scale rule at its boundaries."""
import numpy as np
import torch

import quant_ref as R


def test_values_are_torchs():
    want = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    np.testing.assert_array_equal(R.VALUES, want)


def test_encode_every_code_and_midpoint():
    v = R.VALUES[:127]
    np.testing.assert_array_equal(R.encode(v), np.arange(127))
    mid = (v[1:] + v[:-1]) / 2
    even = np.where(np.arange(126) % 2 == 0, np.arange(126), np.arange(1, 127))
    np.testing.assert_array_equal(R.encode(mid), even)
    np.testing.assert_array_equal(R.encode(mid * (1 - 1e-12)), np.arange(126))
    np.testing.assert_array_equal(R.encode(mid * (1 + 1e-12)), np.arange(1, 127))
    x = np.random.default_rng(1).normal(size=4000) * 60
    want = torch.from_numpy(x).float().to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    np.testing.assert_array_equal(R.encode(x.astype(np.float32)), want)
    np.testing.assert_array_equal(R.encode([np.nan, np.inf]), [127, 127])


def test_need_is_the_smallest_scale():
    for top in (448.0, 448.0001, 1.75, 1.7501, 3.5, 1e-38, 0.0, 3e38):
        e = R.need(top)
        assert 448 * 2.0 ** (e - 127) >= top and (e == 1 or 448 * 2.0 ** (e - 128) < top)


def test_pages_by_hand():
    ref = np.array([2, 1, 0, 1, 0], np.int32)
    table = np.array([[0, 1, -1], [0, 3, -1], [-1, -1, -1]], np.int32)
    r, t, copies, bad = R.fork(ref, table, table, [(0, 2, 40)], 32, True)
    assert r.tolist() == [3, 1, 1, 1, 0] and t[2].tolist() == [0, 2, -1] and copies == [(1, 2, 8)] and not bad
    r, t, bad = R.free(r, t, [2, 2], None, 32)
    assert r.tolist() == ref.tolist() and t.tolist() == table.tolist() and not bad
    after, renamed, copies, n, bad = R.compact(ref, table)
    assert n == 3 and copies == [(3, 2)] and after.tolist() == [2, 1, 1, 0, 0] and renamed[1].tolist() == [0, 2, -1]
