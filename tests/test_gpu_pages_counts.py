"""Forks of rows whose entries are not pages, or pages that nobody counts: those entries become -1 and are flagged, and
no page that a child gets is one that another child shares."""
import numpy as np
import pytest
import torch

from paper_2606_17107_amd import pkv

pytestmark = pytest.mark.gpu


def cuda(a):
    return torch.from_numpy(np.asarray(a)).cuda()


def run(table, ref, forks, page=32, out=None, rows=2):
    """The call over one tensor whose page p holds bytes p + 1; returns table, counts, first bytes of pages, flag."""
    pool = (torch.arange(len(ref), device="cuda") + 1).to(torch.uint8).reshape(1, -1, 1, 1, 1).repeat(1, 1, page, 1, rows)
    g_ref, g_in, flag = cuda(np.asarray(ref, np.int32)), cuda(np.asarray(table, np.int32)), torch.zeros(1, dtype=torch.int32, device="cuda")
    g_out = None if out is None else cuda(np.asarray(out, np.int32))
    pkv.pages_fork([pool], g_ref, g_in, page, pkv.make_forks([dict(parent=a, child=b, n_tokens=n) for a, b, n in forks], "cuda"),
                   len(forks), block_table_out=g_out, err_flag=flag)
    torch.cuda.synchronize()
    return (g_in if out is None else g_out).tolist(), g_ref.tolist(), pool[0, :, :, 0, 0].cpu().numpy(), int(flag.item())


def test_whole_entries_outside_the_pool():
    """They are -1 in the child; the pages beside them are shared and copied as ever."""
    for bad in (7, 100, -1, -5, -2 ** 31):
        table, ref, pool, flag = run([[3, bad, 5, 6], [0, 0, 0, 0]], [0, 0, 0, 1, 0, 1, 1], [(0, 1, 3 * 32 + 4)])
        assert table == [[3, bad, 5, 6], [3, -1, 5, 0]] and flag == 1
        assert ref == [1, 0, 0, 2, 0, 2, 1]
        assert (pool[0] == [7] * 4 + [1] * 28).all()
