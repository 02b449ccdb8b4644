"""Heads and rows to be quantized from the number of blocks on at which 16 lanes take several: against the oracle, with a ragged last group."""
import numpy as np
import pytest
import torch

import paper_2506_09316_amd as dsla
from oracle import block as orc
from tests.block_common import GATE, HALF, NORM, TORCH, assert_quantized, assert_scales_behind_untouched, assert_within, e4m3_room, f64, stored, values

pytestmark = pytest.mark.gpu

CODE = {"f32": dsla.DSLA_F32, "bf16": dsla.DSLA_BF16, "e4m3": dsla.DSLA_E4M3}
SCALE = {"f32": dsla.DSLA_SCALE_F32, "e8m0": dsla.DSLA_SCALE_E8M0}
ACT = {"linear": dsla.DSLA_ACT_NONE, "sigmoid": dsla.DSLA_ACT_SIGMOID, "silu": dsla.DSLA_ACT_SILU}


@pytest.mark.parametrize("out, scale", [("bf16", "e8m0"), ("f32", "e8m0"), ("e4m3", "e8m0"), ("e4m3", "f32")])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows, H, d, gate", [(21850, 5, 64, "silu"), (21850, 3, 128, "silu"), (65537, 1, 64, "sigmoid"), (16389, 4, 128, "linear")])
def test_heads(rows, H, d, gate, dtype, out, scale):
    assert rows * -(-H * d // 128) > 65536 and rows * -(-H * d // 128) % 32
    o, g = values((rows, H, d), dtype, 1, 3.0), values((rows, H, d), dtype, 2, 2.0)
    o *= torch.exp(values((rows, 1, 1), "f32", 5, 2.0)).to(o.dtype)
    w = 1 + 0.3 * values((d,), "f32", 3)
    heads = dsla.make_head_norm(H, d, io_dtype=CODE[dtype], out_dtype=CODE[out], scale_type=SCALE[scale], gate_act=ACT[gate], eps=1e-6, weight=w)
    h, hs = e4m3_room(rows, H * d, scale) if out == "e4m3" else (torch.full((rows, H * d), float("nan"), device="cuda", dtype=TORCH[out]), None)
    dsla.dsla_head_norm(heads, o, h, gate=g, out_scale=hs)
    want = orc.head_norm(f64(o), f64(g), "none" if gate == "linear" else gate, f64(w), 1e-6).reshape(rows, H * d)
    off = np.abs(want) * (NORM + GATE[out])
    if out == "e4m3":
        assert_quantized("heads", h, hs, want, off)
        assert_scales_behind_untouched(hs, H * d)
    else:
        assert_within("heads", f64(h), want, off + HALF[out] * np.abs(want))


@pytest.mark.parametrize("scale", ["e8m0", "f32"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows, cols", [(32773, 400), (131075, 64)])
def test_quantize(rows, cols, dtype, scale):
    x = values((rows, cols), "f32", 3)
    x *= torch.exp(values((rows, 1), "f32", 4, 3.0))
    x[:, ::7] *= 1e-4
    x = x.to(TORCH[dtype])
    q, s = e4m3_room(rows, cols, scale)
    dsla.dsla_quantize(x, q, s)
    want_q, want_s = orc.quantize(f64(x), 1, scale == "e8m0")
    assert (stored(s)[:, :want_s.shape[1]] == want_s).all() and (stored(q) == want_q).all()
    assert_scales_behind_untouched(s, cols)
