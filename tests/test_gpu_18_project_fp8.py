"""The product of e4m3 operands with block scales, against the oracle in 64 bits.

Bounds: results in bf16 are rounded (2^-8) after sums that the e4m3 instructions take in groups of eight products, each kept to 2^-14 of its
group's largest: at most 7 * 2^-14 of the largest magnitudes, so at most 2^-11 of the sum of all magnitudes; results in fp32 after sums
of exact products in fp32: 128 within a block and one for each block, each addition and each scale at most U of the sum of magnitudes.
"""
import numpy as np
import pytest
import torch

import paper_2506_09316_amd as dsla
from oracle import block as orc
from tests.block_common import SCALES, TORCH, U, assert_within, e4m3_room, f64, stored, values

pytestmark = pytest.mark.gpu


def operand(rows, cols, scale, block_rows, seed, std=1.0):
    """e4m3 values with scales of every size, from the library's own call."""
    x = values((rows, cols), "f32", seed, std) * torch.exp(values((rows, 1), "f32", seed + 1, 0.7)) * torch.exp(values((1, cols), "f32", seed + 2, 0.7))
    q, s = e4m3_room(rows, cols, scale, block_rows, fill=255 if scale == "e8m0" else 77)   # (behind a row's last scale: NaN)
    if scale == "f32":
        s.fill_(float("nan"))
    dsla.dsla_quantize(x, q, s, block_rows=block_rows)
    return q, s


def bound(want, size, K, out):
    if out == "bf16":
        return 2.0 ** -8 * np.abs(want) + 2.0 ** -11 * size
    return U * np.abs(want) + (128 + -(-K // 128) + 4) * U * size


def check(M, K, widths, scale, out, bias, seed=0):
    xq, xs = operand(M, K, scale, 1, seed + 10)
    parts = [operand(w, K, scale, 128, seed + 20 + 5 * j, 0.05) for j, w in enumerate(widths)]
    wq = torch.cat([p[0].view(torch.uint8) for p in parts]).view(torch.float8_e4m3fn)
    ws = torch.cat([p[1].view(torch.uint8) for p in parts]).view(SCALES[scale]) if scale == "e8m0" else torch.cat([p[1] for p in parts])
    b = values((sum(widths),), "f32", seed + 3) if bias else None
    outs = [torch.full((M, w), float("nan"), device="cuda", dtype=TORCH[out]) for w in widths]
    dsla.dsla_project_fp8(xq, xs, wq, ws, outs, bias=b)
    nc = -(-K // 128)
    want, size = orc.project(stored(xq), stored(xs)[:, :nc], stored(wq), stored(ws)[:, :nc], widths, f64(b))
    for j, o in enumerate(outs):
        assert_within(f"output {j}", f64(o), want[j], bound(want[j], size[j] + (0 if b is None else 2 * np.abs(f64(b)).max()), K, out))
    return xq, xs, wq, ws, outs, b


SIZES = [(1, 16, [16]), (1, 128, [128]), (3, 144, [16, 48]), (16, 4096, [1040]), (17, 640, [128, 256, 16]), (64, 1392, [208, 64, 128]), (65, 512, [512]),
         (100, 2064, [128, 384]), (129, 128, [144]), (200, 384, [272, 32, 32, 32, 32, 32, 32, 32]), (256, 256, [256, 256]), (300, 1024, [80, 640]), (513, 1392, [1200, 208, 208]),
         (520, 128, [256]), (600, 144, [400, 16]), (1025, 640, [512, 384])]


@pytest.mark.parametrize("out", ["bf16", "f32"])
@pytest.mark.parametrize("scale", ["e8m0", "f32"])
@pytest.mark.parametrize("M, K, widths", SIZES)
def test_project(M, K, widths, scale, out):
    check(M, K, widths, scale, out, bias=M % 2 == 1)


@pytest.mark.parametrize("out", ["bf16", "f32"])
@pytest.mark.parametrize("scale", ["e8m0", "f32"])
@pytest.mark.parametrize("M", [2, 40, 90, 700])
def test_nan_and_zeros_stay_in_their_rows_and_columns(M, scale, out):
    """A NaN in a row of x, or in a scale of it, makes that row NaN; in a row of W that column; a scale of W its block of columns.  Blocks of zeros
    give zeros."""
    K, widths = 400, [192, 64]
    xq, xs, wq, ws, outs, _ = check(M, K, widths, scale, out, bias=False)
    clean = [f64(o) for o in outs]
    xq.view(torch.uint8)[1, 390] = 0x7f
    xq.view(torch.uint8)[0] = 0
    wq.view(torch.uint8)[130, 7] = 0xff
    wq.view(torch.uint8)[200] = 0
    if scale == "e8m0":
        ws.view(torch.uint8)[0, 2] = 255
    else:
        ws[0, 2] = float("nan")
    dsla.dsla_project_fp8(xq, xs, wq, ws, outs)
    a, b = (f64(o) for o in outs)
    assert np.isnan(a[1]).all() and np.isnan(b[1]).all() and np.isnan(a[:, :128]).all() and np.isnan(a[:, 130]).all()
    rest = [m for m in range(M) if m > 1]
    keep = [c for c in range(128, 192) if c != 130]
    assert (a[np.ix_(rest, keep)] == clean[0][np.ix_(rest, keep)]).all() and (a[0][keep] == 0).all() and (b[0] == 0).all()
    others = [c for c in range(64) if c != 8]
    assert (b[np.ix_(rest, others)] == clean[1][np.ix_(rest, others)]).all() and (b[rest, 8] == 0).all()


def test_scales_far_apart():
    """E8M0 scales whose sum of exponents leaves fp32's on its way, and results that are its smallest and largest normal numbers."""
    K = 128
    for out in ("bf16", "f32"):
        for M in (1, 70, 600):
            xq = torch.full((M, K), 1.0, device="cuda").to(torch.float8_e4m3fn)
            wq = torch.full((256, K), 1.0, device="cuda").to(torch.float8_e4m3fn)
            xs, ws = torch.zeros(M, 4, device="cuda", dtype=torch.uint8), torch.zeros(2, 4, device="cuda", dtype=torch.uint8)
            for bx, bw in ((254, 10), (10, 254), (1, 130), (127, 127), (200, 170), (0, 200), (220, 0)):
                xs[:, 0], ws[:, 0] = bx, bw
                o = torch.zeros(M, 256, device="cuda", dtype=TORCH[out])
                dsla.dsla_project_fp8(xq, xs.view(torch.float8_e8m0fnu), wq, ws.view(torch.float8_e8m0fnu), [o])
                assert (f64(o) == 2.0 ** (7 + bx + bw - 254)).all(), (out, M, bx, bw)


@pytest.mark.parametrize("scale", ["e8m0", "f32"])
@pytest.mark.parametrize("M", [3, 100, 600])
def test_stacked_weights_quantized_where_they_lie(M, scale):
    """Every output's weights into their place among the stacked ones, whose scales then begin on any multiple of four bytes."""
    K, widths = 400, [144, 16, 272, 128]
    rows, blocks = sum(widths), sum(-(-w // 128) for w in widths)
    w = values((rows, K), "f32", 3, 0.1)
    wq, ws = e4m3_room(rows, K, scale)[0], e4m3_room(128 * blocks, K, scale, 128)[1]
    at, block = 0, 0
    for n in widths:
        b = -(-n // 128)
        dsla.dsla_quantize(w[at:at + n], wq[at:at + n], ws[block:block + b], block_rows=128)
        at, block = at + n, block + b
    xq, xs = operand(M, K, scale, 1, 5)
    outs = [torch.full((M, n), float("nan"), device="cuda") for n in widths]
    dsla.dsla_project_fp8(xq, xs, wq, ws, outs)
    want, size = orc.project(stored(xq), stored(xs)[:, :4], stored(wq), stored(ws), widths, None)
    for j, o in enumerate(outs):
        assert_within(f"output {j}", f64(o), want[j], bound(want[j], size[j], K, "f32"))
    at = 0
    for n, o in zip(widths, want):   # and they stand for the weights: half a step of e4m3 each, of what is not below its normal numbers
        off = np.abs(f64(w[at:at + n])) * 2.0 ** -4 + np.abs(f64(w)).max() / 448 * 2.0 ** -9
        x = orc.dequantize(stored(xq), stored(xs)[:, :4], 1)
        assert_within("weights", o, x @ f64(w[at:at + n]).T, np.abs(x) @ off.T + 1e-12)
        at += n


@pytest.mark.parametrize("scale", ["e8m0", "f32"])
@pytest.mark.parametrize("out", ["bf16", "f32"])
@pytest.mark.parametrize("M, K, N", [(5, 16384, 64), (150, 24640, 96), (700, 6272, 272), (2, 131072, 16)])
def test_long_rows(M, K, N, scale, out):
    """Scales in many pieces, of every kind of tile."""
    check(M, K, [N], scale, out, bias=True, seed=7)


def test_rows_past_four_gigabytes():
    """The last rows of x, and of W, lie beyond 2^32 bytes."""
    K, M = 1 << 20, 4100
    xq = torch.zeros(M, K, device="cuda", dtype=torch.uint8).view(torch.float8_e4m3fn)
    xs = torch.full((M, K // 128), 127, device="cuda", dtype=torch.uint8).view(torch.float8_e8m0fnu)
    tail, _ = operand(2, K, "e8m0", 1, 3)
    xq.view(torch.uint8)[-2:] = tail.view(torch.uint8)
    wq, ws = operand(16, K, "e8m0", 128, 4)
    o = torch.full((M, 16), float("nan"), device="cuda")
    dsla.dsla_project_fp8(xq, xs, wq, ws, [o])
    blocks = K // 128
    (want,), (size,) = orc.project(stored(tail), np.full((2, blocks), 127, np.uint8), stored(wq), stored(ws)[:, :blocks], [16], None)
    assert_within("x", f64(o[-2:]), want, bound(want, size, K, "f32"))
    assert not o[:-2].any()
    for M2, out in ((2, "bf16"), (2, "f32"), (300, "bf16")):   # the same rows as weights
        few, fs = xq.view(torch.uint8)[:M2].clone().view(torch.float8_e4m3fn), xs.view(torch.uint8)[:M2].clone().view(torch.float8_e8m0fnu)
        few.view(torch.uint8)[0] = wq.view(torch.uint8)[0]
        big = torch.full((33, blocks), 127, device="cuda", dtype=torch.uint8).view(torch.float8_e8m0fnu)
        y = torch.full((M2, 4096), float("nan"), device="cuda", dtype=TORCH[out])
        dsla.dsla_project_fp8(few, fs, xq[4:], big[:32], [y])
        (want,), (size,) = orc.project(stored(wq[:1]), np.full((1, blocks), 127, np.uint8), stored(tail), np.full((1, blocks), 127, np.uint8), [2], None)
        assert_within("W", f64(y[:1, -2:]), want, bound(want, size, K, out))
        assert not y[1:].any() and not y[0, :-2].any()


def _double(q, s, block_rows):
    """The values of e4m3 operands in 64 bits, on the GPU (the sums of so many products take too long on the host)."""
    rows, cols = q.shape
    n = torch.arange(256, device="cuda", dtype=torch.uint8).view(torch.float8_e4m3fn).double()
    f = torch.exp2(s.view(torch.uint8).double() - 127) if s.dtype != torch.float32 else s.double()
    i, j = torch.arange(rows, device="cuda") // block_rows, torch.arange(cols, device="cuda") // 128
    return n[q.view(torch.uint8).long()] * f[i][:, j]


@pytest.mark.parametrize("scale", ["e8m0", "f32"])
@pytest.mark.parametrize("bias", [False, True])
@pytest.mark.parametrize("M, K, widths", [(3000, 128, [4096, 1040, 16, 2048]), (2100, 144, [8192]), (3000, 1408, [4096, 1040, 16, 2048]), (2305, 1536, [1024] * 7 + [1040]),
                                          (2817, 2176, [144, 272, 6800]), (2400, 4112, [4096, 3104, 16]), (2304, 6144, [7168]), (2304, 6272, [7168])])
def test_many_rows_and_columns(M, K, widths, scale, bias):
    """Outputs that take several rounds of the largest tiles: steps of K in even and odd numbers, scales in several pieces, ragged blocks and rows."""
    xq, xs = operand(M, K, scale, 1, 30)
    parts = [operand(w, K, scale, 128, 40 + 3 * j, 0.05) for j, w in enumerate(widths)]
    cat = lambda i, t: torch.cat([p[i].view(torch.uint8) if t != torch.float32 else p[i] for p in parts]).view(t)
    wq, ws = cat(0, torch.float8_e4m3fn), cat(1, SCALES[scale])
    b = values((sum(widths),), "f32", 3) if bias else None
    outs = [torch.full((M, w), float("nan"), device="cuda", dtype=torch.bfloat16) for w in widths]
    dsla.dsla_project_fp8(xq, xs, wq, ws, outs, bias=b)
    x, at = _double(xq, xs, 1), 0
    for o, (q, s) in zip(outs, parts):
        w = _double(q, s, 128)
        want, size = x @ w.t().contiguous(), x.abs() @ w.abs().t().contiguous()
        if bias:
            want, size = want + b[at:at + len(q)].double(), size + 2 * b.abs().max().double()
        off = (o.double() - want).abs() - (2.0 ** -8 * want.abs() + 2.0 ** -11 * size)
        assert o.isfinite().all() and float(off.max()) <= 0, (float(off.max()), int(off.argmax()))
        at += len(q)
