"""Attention over pages: groups of any size, and scores that are infinite."""
import numpy as np
import pytest
import torch

from tests.paged_common import f64, values
from tests.test_gpu_10_attention_paged import attend, check, held, tree_of

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H, H_kv, counts, d", [(7, 1, [64, 1, 37], 64), (71, 1, [3, 0, 1], 128), (339, 3, [2, 5], 64), (1023, 1, [9], 64),
                                                (4096, 1, [1, 2], 64), (65, 5, [1, 1, 1], 128)])
def test_groups_of_any_size(H, H_kv, counts, d, dtype):
    """Rows of a tile that divide into tokens and heads in odd ways, up to the largest group."""
    c, x = held([n + 45 * b for b, n in enumerate(counts)], counts, H_kv=H_kv, d=d, page=16, dtype=dtype, seed=H)
    q = values((sum(counts), H, d), dtype, 3)
    for masks in (None, tree_of(counts, np.random.default_rng(H))):
        check(c, x, q, d ** -0.5, 200, masks, dtype)
    assert c.status.item() == 0


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H, H_kv, n", [(4, 4, 1), (8, 1, 3), (8, 1, 9), (8, 2, 40)])
def test_infinite_scores(H, H_kv, n, dtype):
    """A score of -inf weighs nothing: the same bits as with a key so far off that its weight is zero.  Where all are, zeros; one of +inf
    makes its queries NaN."""
    def run(key, everywhere):
        c, x = held([n + 200, n], [n, n], H_kv=H_kv, d=64, page=16, dtype=dtype, seed=8)
        q = values((2 * n, H, 64), dtype, 9)
        q[:, :, 0] = 1
        row = x.plain[1][0]
        for t in range(n + 200) if everywhere else (0, 21, 150, 200):
            c.pools[0][int(c.oracle.table[row, t // 16]), :, t % 16, 0] = key
        return f64(attend(c, x, q, 0.125, n + 200))

    want, got = run(-1e30, False), run(-float("inf"), False)
    assert np.isfinite(want).all() and (got == want).all()
    far = run(-float("inf"), True)
    assert (far[:n] == 0).all() and (far[n:] == want[n:]).all()
    up = run(float("inf"), False)
    assert np.isnan(up[:n]).all() and (up[n:] == want[n:]).all()
