"""How far a gate may be off where no result is in fp32 (include/dsla.h: 2^-18), seen through the rounding of the result: products are placed beside the
border between two bf16 numbers, further from it than the gate may be off, and have to round to their own side.

A gate's exponent is rounded once: below 128 by half of 2^-17, which is 44.4 U of its power (U = 2^-24); what the constant log2 e lacks is put back.  The
power 2 U, the sum 1, the inverse 2, the factor that puts back 2, the product with z 1, that with the feature 1: 54 U of the result.  (Where the factor
itself is below 2^-126 it has fewer bits: gates above -87.3 here.)
"""
import numpy as np
import pytest
import torch

import paper_2506_09316_amd as dsla
from oracle import block as orc
from tests.block_common import GATE, U

pytestmark = pytest.mark.gpu


def beside_borders(kind, low, high, seed):
    """Features and gates, and the bf16 numbers that their products round to: 57 U from a border, on either side."""
    rng = np.random.default_rng(seed)
    z = rng.uniform(low, high, (1 << 13, 128)).astype(np.float32)
    factor = orc.act(z.astype(np.float64), kind)
    below = 1 + rng.integers(0, 127, z.shape) / 128                      # a bf16 number, the next one is 1 / 128 further
    border = below + 1 / 256
    f = (border * (1 + np.where(rng.integers(0, 2, z.shape), 57, -57) * U) / factor).astype(np.float32)
    product = f * factor
    assert (np.abs(product / border - 1) >= 55 * U).all() and (np.abs(product / border - 1) <= 59 * U).all()
    return f, z, np.where(product > border, below + 1 / 128, below)


@pytest.mark.parametrize("kind, code", [("sigmoid", dsla.DSLA_ACT_SIGMOID), ("silu", dsla.DSLA_ACT_SILU)])
@pytest.mark.parametrize("low, high", [(-87.3, -80), (-80, -61), (-61, -44), (-44, -20), (-20, -3), (-3, -0.01), (0.01, 3), (3, 60)])
def test_gates_keep_their_bound(low, high, kind, code):
    assert GATE["bf16"] <= 55 * U
    f, z, want = beside_borders(kind, low, high, 7)
    o, g = torch.from_numpy(f).cuda(), torch.from_numpy(z).cuda()
    out = torch.zeros(len(f), 128, device="cuda", dtype=torch.bfloat16)
    heads = dsla.make_head_norm(1, 128, io_dtype=dsla.DSLA_F32, out_dtype=dsla.DSLA_BF16, gate_act=code)
    dsla.dsla_head_norm(heads, o.view(-1, 1, 128), out, gate=g.view(-1, 1, 128))
    wrong = out.double().cpu().numpy() != want
    assert not wrong.any(), (wrong.sum(), z[wrong][:4])
    # the border of a block: x' = 0 + y act(g)
    norm = dsla.make_norm(128, x_dtype=dsla.DSLA_BF16, y_dtype=dsla.DSLA_F32, h_dtype=dsla.DSLA_BF16, gate_act=code)
    x = torch.zeros_like(out)
    dsla.dsla_residual_norm(norm, x, o, x, None, gate=g)
    wrong = x.double().cpu().numpy() != want
    assert not wrong.any(), (wrong.sum(), z[wrong][:4])


@pytest.mark.parametrize("out", ["bf16", "f32"])
def test_gates_of_any_size(out):
    """Infinite, huge, tiny and signed gates: as the quotients have them."""
    inf, nan = float("inf"), float("nan")
    z = [0.0, -0.0, 1e-38, -1e-38, 1e-30, -3e-20, 88.0, 130.0, -130.0, 3e38, -3e38, inf, -inf, nan, 1e5, -1e5]
    g = torch.tensor(z * 4, device="cuda").view(1, 1, 64)
    o = torch.ones_like(g)
    for code, want in ((dsla.DSLA_ACT_SIGMOID, [.5, .5, .5, .5, .5, .5, 1, 1, 0, 1, 0, 1, 0, nan, 1, 0]),
                       (dsla.DSLA_ACT_SILU, [0, 0, .5e-38, -.5e-38, .5e-30, -1.5e-20, 88, 130, 0, 3e38, 0, inf, nan, nan, 1e5, 0])):
        result = torch.full((1, 64), 7.0, device="cuda", dtype=torch.bfloat16 if out == "bf16" else torch.float32)
        heads = dsla.make_head_norm(1, 64, io_dtype=dsla.DSLA_F32, out_dtype=dsla.DSLA_BF16 if out == "bf16" else dsla.DSLA_F32, gate_act=code)
        dsla.dsla_head_norm(heads, o, result, gate=g)
        got, want = result[0].double().cpu().numpy(), np.array(want * 4, np.float64)
        finite = np.isfinite(want)
        assert (np.isnan(got) == np.isnan(want)).all() and (got[np.isinf(want)] == inf).all()
        got, want = got[finite], want[finite]
        assert (np.abs(got - want) <= np.abs(want) * (2.0 ** -8 if out == "bf16" else 2.0 ** -21) + 2.0 ** -133).all()
