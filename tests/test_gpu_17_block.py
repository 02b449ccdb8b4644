"""What stands around a layer, against the oracle in 64 bits (bounds: block_common): norms, gates and residual of a block's border, norm and
gate of heads, quantization with block scales."""
import numpy as np
import pytest
import torch

import paper_2506_09316_amd as dsla
from oracle import block as orc
from tests.block_common import (GATE, HALF, NORM, PART, PART_OF, TORCH, U, assert_quantized, assert_scales_behind_untouched, assert_within, e4m3_room, f64, stored,
                                values)

pytestmark = pytest.mark.gpu

CODE = {"f32": dsla.DSLA_F32, "bf16": dsla.DSLA_BF16, "e4m3": dsla.DSLA_E4M3}
ACT = {"none": dsla.DSLA_ACT_NONE, "sigmoid": dsla.DSLA_ACT_SIGMOID, "silu": dsla.DSLA_ACT_SILU}
SCALE = {"f32": dsla.DSLA_SCALE_F32, "e8m0": dsla.DSLA_SCALE_E8M0}
EPS = 1e-6


# ---------------------------------------------------------------------------------------------------------------
# quantization: byte for byte
@pytest.mark.parametrize("scale", ["e8m0", "f32"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows, cols, block_rows", [(1, 16, 1), (3, 112, 1), (5, 128, 1), (2, 144, 1), (33, 640, 1), (700, 1392, 1), (1, 4112, 1),
                                                    (1, 16, 128), (127, 128, 128), (128, 256, 128), (129, 144, 128), (300, 1392, 128)])
def test_quantize(rows, cols, block_rows, dtype, scale):
    x = values((rows, cols), "f32", 3)
    x *= torch.exp(values((rows, 1), "f32", 4, 3.0))    # rows of every size
    x[:, ::7] *= 1e-4                                     # and small values beside large ones
    x = x.to(TORCH[dtype])
    q, s = e4m3_room(rows, cols, scale, block_rows)
    dsla.dsla_quantize(x, q, s, block_rows=block_rows)
    want_q, want_s = orc.quantize(f64(x), block_rows, scale == "e8m0")
    assert (stored(s)[:, :want_s.shape[1]] == want_s).all()
    assert (stored(q) == want_q).all()
    assert_scales_behind_untouched(s, cols)


@pytest.mark.parametrize("scale", ["e8m0", "f32"])
@pytest.mark.parametrize("block_rows", [1, 128])
def test_quantize_unusual_values(block_rows, scale):
    """Blocks of zeros, of the smallest and largest numbers, with infinities and NaN, ties, the borders of scales."""
    rows, cols = 130, 1024
    x = np.random.default_rng(1).standard_normal((rows, cols)).astype(np.float32)
    b = slice(0, 128), slice(128, 256), slice(256, 384), slice(384, 512), slice(512, 640), slice(640, 768), slice(768, 896), slice(896, 1024)
    x[:, b[0]] = 0
    x[:, b[1]] *= 1e-38
    x[:, b[2]] *= 1e37
    x[:, b[3]] = np.where(np.arange(128) % 2, -0.0, 2.0 ** -101)
    x[::3, 512 + 5] = np.inf
    x[1::3, 512 + 9] = -np.inf
    x[2::4, 512 + 100] = np.nan
    x[:, b[5]] = np.where(np.arange(128) % 16 == 3, 448, (np.arange(128) % 100 + 0.5) * np.where(np.arange(128) % 2, 1, -1)).astype(np.float32)   # ties of the type
    x[:, b[6]] = 3.5 * 2.0 ** (np.arange(rows)[:, None] % 40 - 20)          # a scale's largest: 1.75 * 2^n, and the number behind it
    x[::2, 768] = np.nextafter(x[::2, 768], np.float32(np.inf))
    x[5:7, b[7]] = np.inf                                                     # a block with nothing finite in it
    x[7, b[7]] = np.nan
    t = torch.from_numpy(x).cuda()
    q, s = e4m3_room(rows, cols, scale, block_rows)
    dsla.dsla_quantize(t, q, s, block_rows=block_rows)
    want_q, want_s = orc.quantize(x, block_rows, scale == "e8m0")
    assert (stored(s)[:, :8] == want_s).all()
    got, nan = stored(q), np.isnan(orc.e4m3_values())
    assert (nan[got] == nan[want_q]).all() and (nan[got] == ~np.isfinite(x)).all()
    assert (got == want_q)[np.isfinite(x)].all()


# ---------------------------------------------------------------------------------------------------------------
# a block's border
def border(rows, D, x_dtype, y_dtype, out, *, post=True, pre=True, gate="none", scale="e8m0", residual=0.5, with_y=True, keep=True, seed=0, std=1.0):
    x, y = values((rows, D), x_dtype, seed + 1, 2.0 * std), values((rows, D), y_dtype, seed + 2, std) if with_y else None
    g = values((rows, D), y_dtype, seed + 3, 2.0) if gate != "none" and with_y else None
    wpost = 1 + 0.3 * values((D,), "f32", seed + 4) if post and with_y else None
    wpre = 1 + 0.3 * values((D,), "f32", seed + 5) if pre else None
    kind = "none" if gate == "linear" else gate
    norm = dsla.make_norm(D, x_dtype=CODE[x_dtype], y_dtype=CODE[y_dtype], h_dtype=CODE[out], scale_type=SCALE[scale], gate_act=ACT[kind], eps=EPS,
                          residual_scale=residual, post_weight=wpost, pre_weight=wpre)
    x_out = torch.full_like(x, float("nan")) if keep else None
    h, hs = e4m3_room(rows, D, scale) if out == "e4m3" else (torch.full((rows, D), float("nan"), device="cuda", dtype=TORCH[out]), None)
    dsla.dsla_residual_norm(norm, x, y, x_out, h, gate=g, h_scale=hs)
    r, want, part = orc.residual_norm(f64(x), f64(y), f64(g), kind, residual, f64(wpost), f64(wpre), EPS)
    off_r = U * np.abs(r) + PART_OF[(keep and x_dtype == "f32") or out == "f32"] * np.abs(part)
    off = off_r
    if wpre is not None:
        inv = 1 / np.sqrt((r * r).mean(-1, keepdims=True) + EPS) * np.abs(f64(wpre))
        off = inv * off_r + np.abs(want) * (NORM + np.linalg.norm(off_r, axis=-1, keepdims=True) / np.linalg.norm(r, axis=-1, keepdims=True))
    if keep:
        assert_within("x_out", f64(x_out), r, off_r + HALF[x_dtype] * np.abs(r))
    if out == "e4m3":
        assert_quantized("h", h, hs, want, off)
        assert_scales_behind_untouched(hs, D)
    else:
        assert_within("h", f64(h), want, off + HALF[out] * np.abs(want))


@pytest.mark.parametrize("out, scale", [("bf16", "e8m0"), ("f32", "e8m0"), ("e4m3", "e8m0"), ("e4m3", "f32")])
@pytest.mark.parametrize("x_dtype, y_dtype", [("bf16", "bf16"), ("f32", "bf16"), ("bf16", "f32"), ("f32", "f32")])
@pytest.mark.parametrize("rows, D, gate", [(5, 16, "silu"), (3, 112, "sigmoid"), (6, 512, "silu"), (2, 528, "linear"), (9, 1024, "none"), (3, 1040, "silu"),
                                           (4, 2064, "sigmoid"), (2, 4096, "silu"), (3, 8176, "linear"), (2, 9008, "silu"), (1, 16400, "silu"), (1, 32768, "silu")])
def test_border(rows, D, gate, x_dtype, y_dtype, out, scale):
    border(rows, D, x_dtype, y_dtype, out, gate=gate, scale=scale)


@pytest.mark.parametrize("out", ["bf16", "e4m3"])
@pytest.mark.parametrize("options", [dict(post=False), dict(pre=False), dict(post=False, pre=False, gate="silu"), dict(with_y=False), dict(with_y=False, pre=False, keep=False),
                                     dict(keep=False), dict(residual=0.0), dict(residual=-3.5), dict(std=1e-12), dict(std=1e17)])
def test_border_options(options, out):
    border(7, 640, "f32", "f32", out, **options)
    border(1001, 256, "bf16", "bf16", out, **options)


def test_border_without_h():
    x, y, w = values((9, 384), "bf16", 1), values((9, 384), "bf16", 2), 1 + 0.1 * values((384,), "f32", 3)
    norm = dsla.make_norm(384, x_dtype=dsla.DSLA_BF16, y_dtype=dsla.DSLA_BF16, h_dtype=dsla.DSLA_BF16, post_weight=w, pre_weight=w, eps=EPS)
    out = torch.empty_like(x)
    dsla.dsla_residual_norm(norm, x, y, out, None)
    r, _, part = orc.residual_norm(f64(x), f64(y), None, "none", 1.0, f64(w), None, EPS)
    assert_within("x_out", f64(out), r, (U + HALF["bf16"]) * np.abs(r) + PART * np.abs(part))


@pytest.mark.parametrize("D", [256, 1536, 5120])
def test_border_in_place(D):
    """x' over x and h over y, over the gate, or over x: the same bits."""
    x, y, g = (values((37, D), "bf16", i) for i in range(3))
    w = 1 + 0.1 * values((D,), "f32", 9)
    norm = dsla.make_norm(D, x_dtype=dsla.DSLA_BF16, y_dtype=dsla.DSLA_BF16, h_dtype=dsla.DSLA_BF16, gate_act=dsla.DSLA_ACT_SILU, post_weight=w, pre_weight=w)
    x_out, h = torch.empty_like(x), torch.empty_like(x)
    dsla.dsla_residual_norm(norm, x, y, x_out, h, gate=g)
    for to_x, to_h in ((0, 1), (0, 2), (1, 0), (None, 0), (2, None)):
        t = [x.clone(), y.clone(), g.clone()]
        dsla.dsla_residual_norm(norm, t[0], t[1], None if to_x is None else t[to_x], None if to_h is None else t[to_h], gate=t[2])
        assert to_x is None or torch.equal(t[to_x], x_out)
        assert to_h is None or torch.equal(t[to_h], h)


def test_border_not_finite():
    """An infinity or NaN stays in its row; the e4m3 result has NaN there and no other row changes."""
    D = 640
    x, y = values((6, D), "f32", 1), values((6, D), "f32", 2)
    w = torch.ones(D, device="cuda")
    norm = dsla.make_norm(D, x_dtype=dsla.DSLA_F32, y_dtype=dsla.DSLA_F32, h_dtype=dsla.DSLA_E4M3, pre_weight=w, post_weight=w)
    clean = e4m3_room(6, D, "e8m0")
    dsla.dsla_residual_norm(norm, x, y, None, clean[0], h_scale=clean[1])
    x[2, 5], y[4, 600] = float("inf"), float("nan")
    got = e4m3_room(6, D, "e8m0")
    dsla.dsla_residual_norm(norm, x, y, None, got[0], h_scale=got[1])
    rows = [0, 1, 3, 5]
    assert (stored(got[0])[rows] == stored(clean[0])[rows]).all() and (stored(got[1])[rows] == stored(clean[1])[rows]).all()
    assert torch.isnan(got[0][2, 5].float()) and torch.isnan(got[0][4].float()).all()
    assert (got[0][2, :5].float() == 0).all()   # finite over an infinite root mean square


# ---------------------------------------------------------------------------------------------------------------
# heads
@pytest.mark.parametrize("out, scale", [("bf16", "e8m0"), ("f32", "e8m0"), ("e4m3", "e8m0"), ("e4m3", "f32")])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows, H, d, gate, norm", [(1, 1, 64, "silu", True), (1, 1, 128, "none", True), (5, 3, 64, "sigmoid", True), (33, 32, 128, "silu", True), (7, 5, 64, "linear", False),
                                                    (3, 40, 128, "silu", True), (257, 12, 64, "none", False), (2, 9, 128, "sigmoid", False)])
def test_heads(rows, H, d, gate, norm, dtype, out, scale):
    o, g = values((rows, H, d), dtype, 1, 3.0), None if gate == "none" else values((rows, H, d), dtype, 2, 2.0)
    o *= torch.exp(values((1, H, 1), "f32", 5, 2.0)).to(o.dtype)
    w = 1 + 0.3 * values((d,), "f32", 3) if norm else None
    kind = "none" if gate == "linear" else gate
    heads = dsla.make_head_norm(H, d, io_dtype=CODE[dtype], out_dtype=CODE[out], scale_type=SCALE[scale], gate_act=ACT[kind], eps=EPS, weight=w)
    h, hs = e4m3_room(rows, H * d, scale) if out == "e4m3" else (torch.full((rows, H * d), float("nan"), device="cuda", dtype=TORCH[out]), None)
    dsla.dsla_head_norm(heads, o, h, gate=g, out_scale=hs)
    want = orc.head_norm(f64(o), f64(g), kind, f64(w), EPS).reshape(rows, H * d)
    off = np.abs(want) * (NORM + GATE[out])
    if out == "e4m3":
        assert_quantized("heads", h, hs, want, off)
        assert_scales_behind_untouched(hs, H * d)
    else:
        assert_within("heads", f64(h), want, off + HALF[out] * np.abs(want))


def test_heads_in_place_and_large_gates():
    """The result over o or over the gate; gates so large that their exponential overflows."""
    o, g = values((65, 6, 64), "bf16", 1), values((65, 6, 64), "bf16", 2, 300.0)
    heads = dsla.make_head_norm(6, 64, io_dtype=dsla.DSLA_BF16, out_dtype=dsla.DSLA_BF16, weight=torch.ones(64, device="cuda"))
    out = torch.empty(65, 384, device="cuda", dtype=torch.bfloat16)
    dsla.dsla_head_norm(heads, o, out, gate=g)
    with np.errstate(over="ignore"):
        want = orc.head_norm(f64(o), f64(g), "silu", np.ones(64), 1e-6).reshape(65, 384)
    # (below 2^-126 numbers have no 24 bits)
    assert_within("heads", f64(out), want, np.abs(want) * (NORM + GATE["bf16"] + HALF["bf16"]) + 2.0 ** -126)
    a, b = o.clone(), g.clone()
    dsla.dsla_head_norm(heads, a, a, gate=g)
    dsla.dsla_head_norm(heads, o, b, gate=b)
    assert torch.equal(a.view_as(out), out) and torch.equal(b.view_as(out), out)


def test_rows_past_two_gigabytes():
    """Offsets beyond 32 bits: the last rows of a tensor of 2^31 + 4096 elements."""
    rows, cols = 2 ** 19 + 1, 4096
    x = torch.zeros(rows, cols, device="cuda", dtype=torch.bfloat16)
    x[-2:] = values((2, cols), "bf16", 5)
    q, s = torch.empty(rows, cols, device="cuda", dtype=torch.float8_e4m3fn), torch.empty(rows, 32, device="cuda", dtype=torch.float8_e8m0fnu)
    dsla.dsla_quantize(x, q, s)
    want_q, want_s = orc.quantize(f64(x[-2:]), 1, True)
    assert (stored(q[-2:]) == want_q).all() and (stored(s[-2:]) == want_s).all() and not stored(q[-3]).any()
    heads = dsla.make_head_norm(32, 128, io_dtype=dsla.DSLA_BF16, out_dtype=dsla.DSLA_BF16, weight=torch.ones(128, device="cuda"))
    dsla.dsla_head_norm(heads, x, x)
    assert torch.isfinite(x[-2:]).all() and abs(float(x[-1].float().square().mean()) - 1) < 0.02 and not x[-3].any()
    norm = dsla.make_norm(cols, x_dtype=dsla.DSLA_BF16, y_dtype=dsla.DSLA_BF16, h_dtype=dsla.DSLA_BF16, pre_weight=torch.full((cols,), 2.0, device="cuda"))
    dsla.dsla_residual_norm(norm, x, None, None, x)
    assert abs(float(x[-1].float().square().mean()) - 4) < 0.08 and not x[-3].any()
