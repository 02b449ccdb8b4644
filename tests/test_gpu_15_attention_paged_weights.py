"""The softmax weights of attention over pages in the second product, up to 16 rows (tokens times heads of a group) to a key/value head.

Bound beside paged_common's, before any run: a weight p in bf16 is two parts, its upper bits and the rest of p (1 + 2^-20).  The rest is below
(2^-7 + 2^-20) p and rounded by at most 2^-8 of itself, so the parts make p (1 + e), |e| < 2^-15 + 2^-19; their sum divides the product of the
same parts, so the mean is off by less than twice that of the weighted mean of |v|: 2^-13 of it holds.  The result is rounded once, 2^-8 of it.
"""
import numpy as np
import pytest

from oracle import paged as orc
from tests.paged_common import W, attention_bound, assert_within, f64, values
from tests.test_gpu_10_attention_paged import attend, held, signed, tree_of

pytestmark = pytest.mark.gpu

CASES = [   # lens, tokens, H, H_kv, d, page
    ([3], [1], 1, 1, 64, 16), ([2, 5, 17, 33], [1] * 4, 32, 32, 128, 64), ([1000, 40], [1, 1], 32, 8, 128, 64), ([6000], [1], 8, 1, 64, 16),
    ([9, 300, 77], [2, 3, 4], 8, 2, 128, 16), ([31, 500], [4, 3], 4, 1, 64, 32), ([4, 2100], [1, 1], 16, 1, 128, 128), ([20, 900], [8, 2], 2, 1, 64, 64)]


@pytest.mark.parametrize("tree", [False, True])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_weights_keep_their_bits(case, tree):
    lens, counts, H, H_kv, d, page = CASES[case]
    assert max(counts) * H // H_kv <= 16
    c, x = held(lens, counts, H_kv=H_kv, d=d, page=page, dtype="bf16", seed=case)
    q = values((sum(counts), H, d), "bf16", 50 + case, 1.5)
    masks = tree_of(counts, np.random.default_rng(case)) if tree else None
    scale = float(np.float32(d ** -0.5))
    got = f64(attend(c, x, q, scale, max(lens), None if masks is None else signed(masks)))
    want, size, reach = orc.attention(c.oracle, f64(c.pools[0]), f64(c.pools[1]), *x.plain[:2], c.start(x).tolist(), f64(q), scale, masks)
    assert_within("o", got, want, attention_bound(want, size, reach, max(lens), d, "f32") + 2.0 ** -13 * size + W * np.abs(want))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H, H_kv, n", [(4, 4, 1), (16, 1, 2), (8, 1, 3), (8, 2, 40)])
def test_infinite_values_before_the_entry(dtype, H, H_kv, n):
    """Values of one sign among what all queries see make a result infinite, of both signs NaN, whatever bits a weight has (equal keys: all weights
    are one)."""
    for equal in (False, True):
        c, x = held([n + 300, n + 5], [n, n], H_kv=H_kv, d=64, page=16, dtype=dtype, seed=21)
        if equal:
            for p in range(c.oracle.n_pages):
                c.pools[0][p][c.pools[0][p].isfinite()] = 0.5
        t = c.oracle.table[x.plain[1][0]]
        for at, feature, bad in ((0, 0, float("inf")), (37, 9, -float("inf")), (64, 33, float("inf")), (140, 33, float("inf")), (250, 63, -float("inf")),
                                 (5, 63, float("inf"))):
            c.pools[1][int(t[at // 16]), :, at % 16, feature] = bad
        q = values((2 * n, H, 64), dtype, 22)
        got = f64(attend(c, x, q, 0.125, n + 300))
        with np.errstate(all="ignore"):
            want, size, reach = orc.attention(c.oracle, f64(c.pools[0]), f64(c.pools[1]), *x.plain[:2], c.start(x).tolist(), f64(q), 0.125)
        assert (want[:n, :, 0] == np.inf).all() and (want[:n, :, 9] == -np.inf).all() and np.isnan(want[:n, :, 63]).all()
        assert_within("o", got, want, attention_bound(want, size, reach, n + 300, 64, dtype))
