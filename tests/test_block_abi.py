"""What the calls around a layer refuse, on the host: nothing is launched."""
import ctypes

import pytest

import paper_2506_09316_amd as dsla
from paper_2506_09316_amd import binding

OK, NULL, SHAPE, UNSUPPORTED = 0, 1, 2, 3
P = [ctypes.c_void_p(0x1000000 * (i + 1)) for i in range(12)]


@pytest.fixture(scope="module")
def lib():
    return binding.load_library()


def test_constants():
    assert (dsla.DSLA_F32, dsla.DSLA_BF16, dsla.DSLA_E4M3) == (0, 1, 2)
    assert [dsla.scale_pitch(c) for c in (16, 128, 512, 513, 4096, 11008)] == [4, 4, 4, 8, 32, 88]


def norm_of(**k):
    d = dict(D=256, x_dtype=1, y_dtype=1, h_dtype=1, scale_type=1, gate_act=0, eps=1e-6, residual_scale=1.0, post_weight=0x9000, pre_weight=0xa000)
    return binding.DslaNorm(**{**d, **k})


@pytest.mark.parametrize("change, call, want", [
    (dict(D=0), {}, SHAPE), (dict(D=-16), {}, SHAPE), (dict(D=24), {}, UNSUPPORTED), (dict(D=32784), {}, UNSUPPORTED), (dict(x_dtype=2), {}, UNSUPPORTED),
    (dict(y_dtype=2), {}, UNSUPPORTED), (dict(x_dtype=-1), {}, UNSUPPORTED), (dict(h_dtype=3), {}, UNSUPPORTED), (dict(gate_act=3), {}, UNSUPPORTED),
    (dict(gate_act=-1), dict(h=None), UNSUPPORTED), (dict(eps=0.0), {}, SHAPE), (dict(eps=-1.0), {}, SHAPE), (dict(eps=float("nan")), {}, SHAPE),
    (dict(eps=float("inf")), {}, SHAPE), (dict(residual_scale=float("inf")), {}, SHAPE), (dict(residual_scale=float("nan")), {}, SHAPE),
    ({}, dict(rows=0), SHAPE), ({}, dict(rows=-1), SHAPE), ({}, dict(rows=2 ** 31), SHAPE), ({}, dict(rows=2 ** 62), SHAPE), ({}, dict(x=None), NULL),
    ({}, dict(x_out=None, h=None), NULL), ({}, dict(y=None), NULL), (dict(post_weight=None), dict(y=None, gate=P[3]), NULL),
    ({}, dict(h_scale=P[5]), SHAPE), ({}, dict(h=None, h_scale=P[5]), SHAPE), (dict(h_dtype=2), {}, NULL), (dict(h_dtype=2, scale_type=2), dict(h_scale=P[5]), UNSUPPORTED),
    ({}, dict(x=ctypes.c_void_p(0x1008)), SHAPE), ({}, dict(y=ctypes.c_void_p(0x1008)), SHAPE), ({}, dict(gate=ctypes.c_void_p(0x1004)), SHAPE),
    ({}, dict(x_out=ctypes.c_void_p(0x1002)), SHAPE), ({}, dict(h=ctypes.c_void_p(0x1002)), SHAPE), (dict(post_weight=0x9004), {}, SHAPE),
    (dict(pre_weight=0x9004), {}, SHAPE), (dict(h_dtype=2), dict(h_scale=ctypes.c_void_p(0x1002)), SHAPE),
    ({}, dict(h=P[2]), SHAPE), (dict(h_dtype=2), dict(h=P[0], h_scale=P[5]), SHAPE), (dict(h_dtype=0), dict(h=P[1]), SHAPE), (dict(x_dtype=0), dict(x_out=P[1]), SHAPE),
    (dict(h_dtype=2), dict(h_scale=P[0]), SHAPE), (dict(h_dtype=2), dict(h_scale=P[4]), SHAPE)])
def test_residual_norm_refuses(lib, change, call, want):
    a = {**dict(rows=3, x=P[0], y=P[1], gate=None, x_out=P[2], h=P[4], h_scale=None), **call}
    assert lib.dsla_residual_norm(ctypes.byref(norm_of(**change)), a["rows"], a["x"], a["y"], a["gate"], a["x_out"], a["h"], a["h_scale"], None) == want


@pytest.mark.parametrize("change, call, want", [
    (dict(H=0), {}, SHAPE), (dict(H=65537), {}, SHAPE), (dict(d=96), {}, UNSUPPORTED), (dict(io_dtype=2), {}, UNSUPPORTED), (dict(out_dtype=3), {}, UNSUPPORTED),
    (dict(gate_act=4), {}, UNSUPPORTED), (dict(eps=0.0), {}, SHAPE), ({}, dict(rows=0), SHAPE), ({}, dict(rows=2 ** 31), SHAPE), ({}, dict(o=None), NULL), ({}, dict(out=None), NULL),
    ({}, dict(scale=P[5]), SHAPE), (dict(out_dtype=2), {}, NULL), (dict(out_dtype=2, scale_type=7), dict(scale=P[5]), UNSUPPORTED), (dict(weight=0x9008), {}, SHAPE),
    ({}, dict(o=ctypes.c_void_p(0x1008)), SHAPE), ({}, dict(gate=ctypes.c_void_p(0x1008)), SHAPE), ({}, dict(out=ctypes.c_void_p(0x1008)), SHAPE),
    (dict(out_dtype=0), dict(out=P[0]), SHAPE), (dict(out_dtype=2), dict(out=P[1], scale=P[5]), SHAPE), (dict(out_dtype=2), dict(scale=P[0]), SHAPE)])
def test_head_norm_refuses(lib, change, call, want):
    a = {**dict(rows=3, o=P[0], gate=P[1], out=P[2], scale=None), **call}
    d = binding.DslaHeads(**{**dict(H=4, d=64, io_dtype=1, out_dtype=1, scale_type=1, gate_act=2, eps=1e-6, weight=0x9000), **change})
    assert lib.dsla_head_norm(ctypes.byref(d), a["rows"], a["o"], a["gate"], a["out"], a["scale"], None) == want


def test_structures_are_required(lib):
    assert lib.dsla_residual_norm(None, 1, P[0], P[1], None, P[2], P[3], None, None) == NULL
    assert lib.dsla_head_norm(None, 1, P[0], None, P[2], None, None) == NULL


@pytest.mark.parametrize("call, want", [
    (dict(rows=0), SHAPE), (dict(cols=0), SHAPE), (dict(cols=24), UNSUPPORTED), (dict(cols=(1 << 21) + 16), UNSUPPORTED), (dict(dtype=2), UNSUPPORTED), (dict(block_rows=64), UNSUPPORTED),
    (dict(scale_type=2), UNSUPPORTED), (dict(rows=2 ** 31), SHAPE), (dict(x=None), NULL), (dict(q=None), NULL), (dict(scale=None), NULL), (dict(x=ctypes.c_void_p(8)), SHAPE),
    (dict(q=ctypes.c_void_p(8)), SHAPE), (dict(scale=ctypes.c_void_p(6)), SHAPE), (dict(q=P[0]), SHAPE), (dict(scale=P[0]), SHAPE), (dict(scale=P[1]), SHAPE)])
def test_quantize_refuses(lib, call, want):
    a = {**dict(rows=4, cols=256, dtype=1, block_rows=1, scale_type=1, x=P[0], q=P[1], scale=P[2]), **call}
    assert lib.dsla_quantize(a["rows"], a["cols"], a["dtype"], a["block_rows"], a["scale_type"], a["x"], a["q"], a["scale"], None) == want


@pytest.mark.parametrize("call, want", [
    (dict(M=0), SHAPE), (dict(M=-5), SHAPE), (dict(M=2 ** 63 - 1), SHAPE), (dict(M=2 ** 58, widths=[1 << 12]), SHAPE), (dict(K=0), SHAPE), (dict(K=72), UNSUPPORTED), (dict(K=(1 << 21) + 16), UNSUPPORTED), (dict(widths=[]), SHAPE),
    (dict(widths=[16] * 9), UNSUPPORTED), (dict(widths=[64, 0]), SHAPE), (dict(widths=[64, -16]), SHAPE), (dict(widths=[24]), UNSUPPORTED), (dict(widths=[1 << 24, 16]), SHAPE),
    (dict(widths=[(1 << 24) + 16]), SHAPE), (dict(M=2 ** 40, widths=[1 << 20]), SHAPE), (dict(scale_type=2), UNSUPPORTED), (dict(out=2), UNSUPPORTED), (dict(x=None), NULL), (dict(xs=None), NULL),
    (dict(w=None), NULL), (dict(ws=None), NULL), (dict(x=ctypes.c_void_p(8)), SHAPE), (dict(xs=ctypes.c_void_p(6)), SHAPE), (dict(w=ctypes.c_void_p(8)), SHAPE),
    (dict(ws=ctypes.c_void_p(6)), SHAPE), (dict(bias=ctypes.c_void_p(8)), SHAPE), (dict(outs=[None, 0x1000]), NULL), (dict(outs=[0x1000, 0x1008]), SHAPE), (dict(outs=[0x1000, 0x1000]), SHAPE),
    (dict(outs=[0x1000, P[0].value]), SHAPE), (dict(outs=[P[2].value, 0x1000]), SHAPE)])
def test_project_fp8_refuses(lib, call, want):
    a = {**dict(M=4, K=256, widths=[64, 128], scale_type=1, x=P[0], xs=P[1], w=P[2], ws=P[3], bias=None, out=1, outs=[0x100000, 0x200000]), **call}
    n = len(a["widths"])
    widths = (ctypes.c_int32 * max(1, n))(*a["widths"])
    outs = (ctypes.c_void_p * max(n, 2))(*(a["outs"] + [0x1000] * max(0, n - 2)))
    assert lib.dsla_project_fp8(a["M"], a["K"], n, widths, a["scale_type"], a["x"], a["xs"], a["w"], a["ws"], a["bias"], a["out"], outs, None) == want


def test_project_fp8_requires_its_arrays(lib):
    outs, widths = (ctypes.c_void_p * 1)(0x1000), (ctypes.c_int32 * 1)(64)
    assert lib.dsla_project_fp8(4, 256, 1, None, 1, P[0], P[1], P[2], P[3], None, 1, outs, None) == NULL
    assert lib.dsla_project_fp8(4, 256, 1, widths, 1, P[0], P[1], P[2], P[3], None, 1, None, None) == NULL
