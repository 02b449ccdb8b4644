"""A paged cache at the sizes where its calls change their ways."""
import numpy as np
import pytest

from oracle import paged as orc
from tests.paged_common import assert_within, attention_bound, f64, values
from tests.test_gpu_10_attention_paged import attend, held

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_many_requests_that_may_draft_many(dtype):
    """More requests of up to 64 tokens, with more heads, than a 32-bit number of rows at a thousand bytes each would hold."""
    B, H, H_kv, d = 520, 64, 8, 64
    r = np.random.default_rng(1)
    counts = [64 if b in (7, 519) else int(r.integers(0, 3)) for b in range(B)]
    lens = [n + int(r.integers(0, 40)) for n in counts]
    c, x = held(lens, counts, H_kv=H_kv, d=d, page=16, dtype=dtype, seed=2)
    assert x.max_n == 64
    q = values((sum(counts), H, d), dtype, 3)
    got = f64(attend(c, x, q, 0.125, max(lens)))
    want, size, reach = orc.attention(c.oracle, f64(c.pools[0]), f64(c.pools[1]), *x.plain[:2], c.start(x).tolist(), f64(q), 0.125)
    assert c.status.item() == 0
    assert_within("o", got, want, attention_bound(want, size, reach, max(lens), d, dtype))
