"""Calls of many layers: layers and KV heads are beyond what a grid dimension holds together."""
import numpy as np
import pytest

import tree_ref as T
from helpers import check_attention_close
from test_gpu_tree_attention import Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("lens", [[3], [0]])
@pytest.mark.parametrize("L", [16383, 16384])
def test_layers_and_heads(L, lens):
    """16 rows of 4 KV heads: as many rows as go through the join in tiles, up to 65535 (layer, head) pairs.  Rows see a few
    slots and rows: outputs are off by up to 2^-7 max |v|, below 0.047, as in the attention tests."""
    c = Case("bf16", lens, [16], G=1, Hkv=4, d=64, L=L, seed=60)
    out, lse = c.call(c.masks())
    got = out.t[[0, 1, L // 2, L - 1]].double().cpu().numpy()
    for at, l in zip(got, (0, 1, L // 2, L - 1)):
        want, want_lse = T.attention(c.q[l].double().cpu().numpy(), c.cache("k", l, 0, lens[0]), c.cache("v", l, 0, lens[0]),
                                     c.dk[l].double().cpu().numpy(), c.dv_rows[l].double().cpu().numpy(), c.pos, c.seen[0], c.scale)
        check_attention_close(at, want, max_abs=0.047)
        np.testing.assert_allclose(lse[l].cpu().numpy(), want_lse, atol=2e-2)
