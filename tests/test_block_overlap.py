"""Outputs of the norms given as one of the weights, or as an input whose elements have another size, are refused (launches stubbed out: an accepted
call is one)."""
from tests.launch_sizes import run_checked

BODY = r"""
F32, BF16, E4M3 = 0, 1, 2
X, Y, G, XO, H, S, POST, PRE = (ptr(n) for n in range(8))

def border(x_dtype=F32, y_dtype=F32, h_dtype=F32, rows=1, x=X, y=Y, gate=G, x_out=XO, h=H, s=None, post=POST, pre=PRE):
    stub.launch_stub_reset(-1)
    n = binding.DslaNorm(D=256, x_dtype=x_dtype, y_dtype=y_dtype, h_dtype=h_dtype, scale_type=0, gate_act=2, eps=1e-6, residual_scale=1.0, post_weight=post, pre_weight=pre)
    status = lib.dsla_residual_norm(ctypes.byref(n), i64(rows), x, y, gate, x_out, h, s, None)
    assert stub.launch_stub_count() == (status == OK)
    return status

assert border() == OK
for rows in (1, 5):
    assert [border(rows=rows, x_out=p) for p in (X, Y, G, POST, PRE, H)] == [OK, OK, OK, ERR_SHAPE, ERR_SHAPE, ERR_SHAPE]
    assert [border(rows=rows, h=p) for p in (X, Y, G, POST, PRE)] == [OK, OK, OK, ERR_SHAPE, ERR_SHAPE]
    assert [border(rows=rows, h_dtype=E4M3, s=p) for p in (S, X, Y, G, H, XO, POST, PRE)] == [OK] + 7 * [ERR_SHAPE]
# one buffer as both inputs, of different types: an output there has the size of one of them only
for x_dtype, y_dtype in ((F32, BF16), (BF16, F32)):
    for other in (dict(y=X), dict(gate=X)):
        assert border(x_dtype, y_dtype, **other) == OK
        assert border(x_dtype, y_dtype, x_out=X, **other) == ERR_SHAPE
        assert border(x_dtype, y_dtype, h_dtype=x_dtype, h=X, **other) == ERR_SHAPE
        assert border(x_dtype, x_dtype, h_dtype=x_dtype, h=X, **other) == OK

def heads(io=F32, out=F32, rows=1, o=X, gate=G, to=H, s=None, weight=POST):
    stub.launch_stub_reset(-1)
    n = binding.DslaHeads(H=1, d=128, io_dtype=io, out_dtype=out, scale_type=0, gate_act=2, eps=1e-6, weight=weight)
    status = lib.dsla_head_norm(ctypes.byref(n), i64(rows), o, gate, to, s, None)
    assert stub.launch_stub_count() == (status == OK)
    return status

assert [heads(to=p) for p in (H, X, G, POST)] == [OK, OK, OK, ERR_SHAPE]
assert [heads(out=E4M3, s=p) for p in (S, X, G, H, POST)] == [OK] + 4 * [ERR_SHAPE]
assert heads(to=POST, weight=None) == OK
"""


def test_what_an_output_may_be(tmp_path):
    run_checked(tmp_path, BODY)
