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


# A size with a few steps of 128 for every kernel.
FEW = [min((s for s in SIZES if s[:4] == kernel and s[5] > 128), key=lambda s: s[5]) for kernel in sorted({s[:4] for s in SIZES})]


@pytest.mark.parametrize("mt, nt, scale, out, M, K, widths", FEW)
def test_what_is_not_a_number_stays_where_it_is(mt, nt, scale, out, M, K, widths):
    """NaN in a row of x, in its scales of an even and of an odd step, in a column of W and in a scale of W; rows and columns of zeros."""
    xq, xs, wq, ws, _ = operands(M, K, widths, scale, 60)
    outs = [o[:M] for o in roomy(M, widths, out)]
    dsla.dsla_project_fp8(xq, xs, wq, ws, outs)
    clean, last, N = torch.cat(outs, 1), -(-K // 128) - 1, sum(widths)
    rows = {name: r for r, name in zip((0, M - 1, M // 2, M // 3, 2 * M // 3), ("zeros", "value", "even", "odd", "last")) if M > 4 or name in ("zeros", "value")}
    nan = 255 if scale == "e8m0" else float("nan")
    bits = xs.view(torch.uint8) if scale == "e8m0" else xs
    xq.view(torch.uint8)[rows["value"], K - 3] = 0x7f
    xq.view(torch.uint8)[rows["zeros"]] = 0
    for name, step in (("even", 2), ("odd", 1), ("last", last)):
        if name in rows:
            bits[rows[name], step] = nan
    dsla.dsla_project_fp8(xq, xs, wq, ws, outs)
    got = torch.cat(outs, 1)
    bad = [r for n, r in rows.items() if n != "zeros"]
    rest = torch.tensor([m for m in range(M) if m not in rows.values()], device="cuda", dtype=torch.long)
    assert got[bad].isnan().all() and (got[rows["zeros"]] == 0).all() and torch.equal(got[rest], clean[rest])
    # and in W: a column, one of zeros, and a block's scale (of the last output, whose block of columns is its last)
    at, block = N - widths[-1], sum(-(-w // 128) for w in widths[:-1])
    first = at + (widths[-1] - 1) // 128 * 128
    wq.view(torch.uint8)[0, K - 5] = 0xff
    if first > 1:
        wq.view(torch.uint8)[1] = 0
    wbits = ws.view(torch.uint8) if scale == "e8m0" else ws
    wbits[-1, 1] = nan
    dsla.dsla_project_fp8(xq, xs, wq, ws, outs)
    got = torch.cat(outs, 1)
    assert got[:, 0].isnan().all() and got[:, first:].isnan().all()
    if first > 1:
        assert (got[rest, 1] == 0).all() and torch.equal(got[rest][:, 2:first], clean[rest][:, 2:first])


@pytest.mark.parametrize("mt, nt, scale, out, M, K, widths", FEW)
def test_scales_far_apart(mt, nt, scale, out, M, K, widths):
    """Ones with scales whose product is the same in every block and far from both: exactly as many as there are, times that."""
    exponents = torch.tensor([127, -127, 0, 73, -101, 1, -1, 120], device="cuda") if scale == "e8m0" else torch.tensor([100, -100, 0, 73, -101, 1, -1, 90], device="cuda")
    P, blocks = -(-K // 512) * 4, [-(-w // 128) for w in widths]
    row, step, block = torch.arange(M, device="cuda"), torch.arange(P, device="cuda"), torch.arange(sum(blocks), device="cuda")
    one = torch.full((max(M, sum(widths)), K), 0x38, device="cuda", dtype=torch.uint8).view(torch.float8_e4m3fn)
    for c in (0, 90 if scale == "e8m0" else 20, -90 if scale == "e8m0" else -20):
        a = exponents[step % 8].expand(M, P)                      # x: 2^(a - row % 3)
        b = c - exponents[step % 8].expand(sum(blocks), P)        # W: 2^(c - a)
        a = a - (row % 3 * (c >= 0))[:, None] * (a > -120)
        keep = a.clamp(-127, 127) if scale == "e8m0" else a
        b = b.clamp(-127, 127) if scale == "e8m0" else b
        xs = (keep + 127).to(torch.uint8).view(torch.float8_e8m0fnu) if scale == "e8m0" else torch.exp2(keep.double()).float()
        ws = (b + 127).to(torch.uint8).view(torch.float8_e8m0fnu) if scale == "e8m0" else torch.exp2(b.double()).float()
        outs = [torch.zeros(M, w, device="cuda", dtype=TORCH[out]) for w in widths]
        dsla.dsla_project_fp8(one[:M], xs.contiguous(), one[:sum(widths)], ws.contiguous(), outs)
        steps = -(-K // 128)
        in_step = torch.tensor([min(128, K - 128 * s) for s in range(steps)], device="cuda", dtype=torch.float64)
        each = torch.exp2((keep[:, :steps] + b[:1, :steps]).double()) * in_step
        size, want = each.sum(1), each.sum(1)
        bound = (2.0 ** -8 + 2.0 ** -11 if out == "bf16" else (steps + 4) * U) * size
        for o in outs:
            assert bool(((o.double() - want[:, None]).abs() <= bound[:, None]).all()), c
