"""Shared by the tests of what stands around a layer: tensors, and bounds derived from the arithmetic.

U = 2^-24 is half a step of fp32.  A sum of n squares in fp32, whatever its order, is off by at most (its depth + 1) U, relatively, since the terms
have one sign: a lane adds up to 32 of its own, 6 across the wavefront, up to 16 across wavefronts, so at most 57 U, half of that under the
square root, and 4 more for the quotient, eps, the root and the inverse: 33 U on 1 / rms.  Two more products: 35 U on a norm's result.  A
gate is at most 8 U off (the exponential 4, sum, quotient and product), so the part that is added to x at most 45 U, and the sum 1 U.

Where no result is in fp32 a gate's exponential is that of an exponent rounded once, |z| log2 e - 24 below 128 by 64 U (half a step from 64 on), so its power
is 64 U ln 2 = 45 U off, 2 U for the instruction, 2 U for the inverse's, 4 roundings: 53 U, and the part that is added 8 U less than 46 + 53.
"""
import numpy as np
import torch

from oracle import block as orc

U = 2.0 ** -24
HALF = {"bf16": 2.0 ** -8, "f32": U}
TORCH = {"bf16": torch.bfloat16, "f32": torch.float32, "e4m3": torch.float8_e4m3fn}
SCALES = {"f32": torch.float32, "e8m0": torch.float8_e8m0fnu}
NORM, PART = 35 * U, 46 * U
GATE = {"f32": 9 * U, "bf16": 54 * U, "e4m3": 54 * U}
PART_OF = {True: PART, False: PART + 45 * U}   # is a result in fp32?


def f64(t):
    return None if t is None else t.detach().double().cpu().numpy()


def stored(t):
    """Bytes of e4m3 or E8M0 tensors, fp32 scales as they are."""
    t = t.detach()
    return (t if t.dtype == torch.float32 else t.view(torch.uint8)).cpu().numpy()


def values(shape, dtype, seed, std=1.0, mean=0.0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return (torch.empty(*shape, device="cuda").normal_(0, 1, generator=g) * std + mean).to(TORCH[dtype])


def e4m3_room(rows, cols, scale, block_rows=1, fill=77):
    """Room for an e4m3 result and its scales, filled with a byte that is not zero."""
    q = torch.full((rows, cols), fill, device="cuda", dtype=torch.uint8).view(torch.float8_e4m3fn)
    n = -(-rows // block_rows)
    s = torch.full((n, orc.pitch(cols)), fill, device="cuda", dtype=torch.uint8) if scale == "e8m0" else torch.full((n, orc.pitch(cols)), float(fill), device="cuda")
    return q, s.view(SCALES[scale])


def assert_within(name, got, want, bound):
    bad = ~(np.abs(got - want) <= bound)
    assert got.shape == want.shape and not bad.any(), (
        f"{name}: {bad.sum()} of {bad.size} off, first at {np.argwhere(bad)[0]}: {got[bad][0]} for {want[bad][0]}, bound {np.broadcast_to(bound, want.shape)[bad][0]}")


def assert_scales_behind_untouched(s, cols, fill=77):
    behind = stored(s)[:, -(-cols // 128):]
    assert (behind == fill).all()


def assert_quantized(name, q, s, want, off):
    """An e4m3 result of values `want` that are known up to `off`: every scale that of a largest magnitude within that, every value
    within half a step of the type (2^-4 relative, 2^-10 scales below 2^-6 scales) and what the clamp at 448 cuts (4 U)."""
    q, s, cols = stored(q), stored(s), want.shape[1]
    nc = -(-cols // 128)
    s = s[:, :nc]
    amax, slack = orc.block_amax(want, 1), np.zeros((want.shape[0], nc))
    for b in range(nc):
        slack[:, b] = off[:, 128 * b:128 * b + 128].max(1)
    if s.dtype == np.uint8:
        low, high = orc.e8m0_of(np.maximum(amax - slack, orc.LEAST)), orc.e8m0_of(amax + slack)
        assert ((s >= low) & (s <= high)).all(), f"{name}: scales"
    else:
        assert_within(f"{name}: scales", s.astype(np.float64), amax / 448, (slack + 2 * U * amax) / 448)
    step = orc.spread(orc.scale_values(s), want.shape, 1)
    assert_within(name, orc.dequantize(q, s, 1), want, off * (1 + 2.0 ** -4) + np.maximum(2.0 ** -4 * np.abs(want), 2.0 ** -10 * step) + 4 * U * np.abs(want))
