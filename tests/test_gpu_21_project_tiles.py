"""Every kernel of the product of e4m3 operands against its definition in 64 bits, at sizes that take it (tests/test_project_tiles.py).  Bounds:
test_gpu_18_project_fp8."""
import pytest
import torch

import paper_2506_09316_amd as dsla
from tests.block_common import SCALES, TORCH, U, values
from tests.project_sizes import SIZES
from tests.test_gpu_18_project_fp8 import _double, operand

pytestmark = pytest.mark.gpu


def operands(M, K, widths, scale, seed):
    """x, W with their scales, and the scales of every output."""
    xq, xs = operand(M, K, scale, 1, seed)
    parts = [operand(w, K, scale, 128, seed + 10 + 3 * j, 0.05) for j, w in enumerate(widths)]
    wq = torch.cat([p[0].view(torch.uint8) for p in parts]).view(torch.float8_e4m3fn)
    ws = torch.cat([p[1].view(torch.uint8) if scale == "e8m0" else p[1] for p in parts]).view(SCALES[scale])
    return xq, xs, wq, ws, parts


def roomy(M, widths, out):
    """Outputs with something behind their last row."""
    return [torch.full((M + 3, w), 5.0, device="cuda", dtype=TORCH[out]) for w in widths]


@pytest.mark.parametrize("mt, nt, scale, out, M, K, widths", SIZES)
def test_project(mt, nt, scale, out, M, K, widths):
    xq, xs, wq, ws, parts = operands(M, K, widths, scale, 50)
    b = values((sum(widths),), "f32", 3) if (M + K // 16) % 2 else None
    room = roomy(M, widths, out)
    outs = [o[:M] for o in room]
    dsla.dsla_project_fp8(xq, xs, wq, ws, outs, bias=b)
    x, at = _double(xq, xs, 1), 0
    for o, whole, (q, s) in zip(outs, room, parts):
        w = _double(q, s, 128)
        want, size = x @ w.t().contiguous(), x.abs() @ w.abs().t().contiguous()
        if b is not None:
            want, size = want + b[at:at + len(q)].double(), size + 2 * b.abs().max().double()
        bound = 2.0 ** -8 * want.abs() + 2.0 ** -11 * size if out == "bf16" else U * want.abs() + (128 + -(-K // 128) + 4) * U * size
        off = (o.double() - want).abs() - bound
        assert o.isfinite().all() and float(off.max()) <= 0, (float(off.max()), int(off.argmax()))
        assert bool((whole[M:] == 5).all())
        at += len(q)
