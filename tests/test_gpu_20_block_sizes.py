"""Calls around a layer with so many rows that a launch needs a second dimension: every row, some of them against the oracle."""
import numpy as np
import pytest
import torch

import paper_2506_09316_amd as dsla
from oracle import block as orc
from tests.block_common import HALF, NORM, TORCH, U, assert_within, f64, stored, values

pytestmark = pytest.mark.gpu

EPS = 1e-6


@pytest.fixture(autouse=True)
def room():
    torch.cuda.empty_cache()
    yield
    torch.cuda.empty_cache()


def taken(t, rows):
    return torch.stack([t[r] for r in rows])


def all_but(t, rows, want):
    """Every element but those of some rows is `want`.  (Those rows are lost.)"""
    for r in rows:
        t[r] = want
    return all(bool((c == want).all()) for c in t.view(-1).split(1 << 30))


def ones(rows, cols, some):
    x = torch.ones(rows, cols, device="cuda", dtype=torch.bfloat16)
    for r, v in zip(some, values((len(some), cols), "bf16", 5, 3.0)):
        x[r] = v
    return x, f64(taken(x, some))


@pytest.mark.parametrize("rows, D", [(2 ** 28 - 1, 16), (2 ** 28 + 5, 16), (2 ** 26 + 3, 144), (2 ** 24 + 77, 1040)])
def test_border_of_many_rows(rows, D):
    some = [0, 65536, rows // 2, 2 ** 24 - 1, rows - 2, rows - 1]
    x, start = ones(rows, D, some)
    w = torch.full((D,), 2.0, device="cuda")
    norm = dsla.make_norm(D, x_dtype=dsla.DSLA_BF16, y_dtype=dsla.DSLA_BF16, h_dtype=dsla.DSLA_BF16, pre_weight=w, eps=EPS)
    dsla.dsla_residual_norm(norm, x, None, None, x)
    want = orc.norm(start, f64(w), EPS)
    assert_within("rows", f64(taken(x, some)), want, np.abs(want) * (NORM + U + HALF["bf16"]))
    assert all_but(x, some, 2.0)


@pytest.mark.parametrize("rows, d", [(2 ** 29 + 9, 64), (2 ** 29 + 9, 128)])
def test_many_heads(rows, d):
    some = [0, 65536 * 32, rows // 2, rows - 2, rows - 1]
    o, start = ones(rows, d, some)
    w = torch.full((d,), 2.0, device="cuda")
    heads = dsla.make_head_norm(1, d, io_dtype=dsla.DSLA_BF16, out_dtype=dsla.DSLA_BF16, weight=w, eps=EPS)
    dsla.dsla_head_norm(heads, o.view(rows, 1, d), o)
    want = orc.norm(start, f64(w), EPS)
    assert_within("rows", f64(taken(o, some)), want, np.abs(want) * (NORM + HALF["bf16"]))
    assert all_but(o, some, 2.0)


@pytest.mark.parametrize("rows, block_rows", [(2 ** 30 + 70, 1), (2 ** 31 - 65, 128)])
def test_quantize_many_rows(rows, block_rows):
    """Ones are 256 times 2^-8."""
    some = [rows - 3, rows - 1] if block_rows == 1 else list(range(rows - rows % 128, rows))
    x, start = ones(rows, 16, some)
    q = torch.zeros(rows, 16, device="cuda", dtype=torch.uint8)
    s = torch.zeros(-(-rows // block_rows), 4, device="cuda", dtype=torch.uint8)
    dsla.dsla_quantize(x, q.view(torch.float8_e4m3fn), s.view(torch.float8_e8m0fnu), block_rows=block_rows)
    want_q, want_s = orc.quantize(start, block_rows, True)
    last = some if block_rows == 1 else [len(s) - 1]
    assert (stored(taken(q, some)) == want_q).all() and (stored(taken(s, last)[:, :1]) == want_s).all()
    assert all_but(q, some, 0x78)
    scales = s[:, :1].contiguous()
    assert all_but(scales, last, 119) and not any(bool(c.any()) for c in s[:, 1:].split(1 << 28))


@pytest.mark.parametrize("out", ["bf16", "f32"])
@pytest.mark.parametrize("extra", [-64, 71])
def test_product_of_many_rows(extra, out):
    """Rows of ones times a weight of ones, and a few others."""
    M, K, N = 2 ** 29 + extra, 16, 16
    some = [0, 65536 * 64, M // 2, M - 2, M - 1]
    x = torch.full((M, K), 0x38, device="cuda", dtype=torch.uint8)   # 1.0
    xs = torch.full((M, 4), 127, device="cuda", dtype=torch.uint8)
    wq, ws = torch.full((N, K), 0x38, device="cuda", dtype=torch.uint8), torch.full((1, 4), 127, device="cuda", dtype=torch.uint8)
    for i, r in enumerate(some):
        x[r, i] = 0x40 + 8 * i   # 2, 4, 8 ..
    y = torch.zeros(M, N, device="cuda", dtype=TORCH[out])
    dsla.dsla_project_fp8(x.view(torch.float8_e4m3fn), xs.view(torch.float8_e8m0fnu), wq.view(torch.float8_e4m3fn), ws.view(torch.float8_e8m0fnu), [y])
    assert f64(taken(y, some)).tolist() == [[15.0 + 2 ** (i + 1)] * N for i in range(len(some))]
    assert all_but(y, some, 16.0)
