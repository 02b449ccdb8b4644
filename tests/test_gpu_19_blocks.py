"""The calls around a layer together, as a program uses them: prompt and tokens through whole blocks, every step against the oracle on the
inputs that it had, the same from a graph, on another stream, and two calls at once."""
import json

import numpy as np
import pytest
import torch

import paper_2506_09316_amd as dsla
import serving_step
from oracle import block as orc
from oracle import dsla_oracle
from tests.block_common import GATE, HALF, NORM, PART, U, assert_quantized, assert_within, f64, stored

pytestmark = pytest.mark.gpu

EPS = 1e-5


def stack_of(L, K, H, d, seed=1):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return serving_step.Blocks(L, K, H, d, gen), gen


def layer_call(stack, B, T, S, decode=False, **more):
    desc = dsla.make_desc(B, stack.H, stack.d, stack.d, io_dtype=dsla.DSLA_BF16, gate_dtype=dsla.DSLA_BF16, gamma=0.3, scale=stack.d ** -0.5, gate_mode=1, **more)
    ws = torch.empty(max(256, 0 if decode else dsla.dsla_prefill_workspace_bytes(desc, T)), dtype=torch.uint8, device="cuda")
    if decode:
        return lambda l, *a: dsla.dsla_decode(desc, *a[:5], *S[l], a[5])
    return lambda l, *a: dsla.dsla_prefill(desc, T, *a[:5], *S[l], a[5], ws)


@pytest.mark.parametrize("B, T, K, H, d", [(2, 37, 208, 3, 64), (1, 300, 512, 4, 128)])
def test_a_block_step_by_step(B, T, K, H, d):
    """One block, every call's result against the oracle on what it read."""
    stack, gen = stack_of(1, K, H, d)
    x = torch.randn(B * T, K, device="cuda", generator=gen).to(torch.bfloat16)
    S = [[torch.zeros(B, H, d, d, device="cuda") for _ in range(2)]]
    room, start, width = stack.room(B * T), f64(x), H * d
    stack.run(x, room, layer_call(stack, B, T, S))
    # the first norm
    want = orc.norm(start, f64(stack.borders[0]._keep[1]), EPS)
    assert_quantized("h", *room["h"], want, np.abs(want) * (NORM + U))
    # the projections
    blocks = lambda t, n: stored(t)[:, :-(-n // 128)]
    outs, sizes = orc.project(stored(room["h"][0]), blocks(room["h"][1], K), stored(stack.inside[0][0]), blocks(stack.inside[0][1], K), [width] * 6, None)
    for got, want, size in zip(room["outs"], outs, sizes):
        assert_within("projection", f64(got), want, HALF["bf16"] * np.abs(want) + 2.0 ** -11 * size)
    # the layer, as its own tests hold it
    q, k, v, z1, z2 = (f64(t).reshape(B, T, H, d) for t in room["outs"][:5])
    log_gate = lambda z: -np.logaddexp(0, -z) / 16
    o, _, _ = dsla_oracle.recurrent(q, k, v, log_gate(z1), log_gate(z2), 0.3, d ** -0.5)
    got = f64(room["o"]).reshape(o.shape)
    assert np.abs(got - o).max() <= 2e-2 * np.abs(o).max()
    # norm and gate of its heads
    want = orc.head_norm(f64(room["o"]).reshape(-1, H, d), f64(room["outs"][5]).reshape(-1, H, d), "silu", f64(stack.heads[0]._keep[0]), EPS).reshape(-1, width)
    assert_quantized("heads", *room["o8"], want, np.abs(want) * (NORM + GATE["e4m3"]))
    # the output projection and the last border
    (want,), (size,) = orc.project(stored(room["o8"][0]), blocks(room["o8"][1], width), stored(stack.outside[0][0]), blocks(stack.outside[0][1], width), [K], None)
    assert_within("output projection", f64(room["y"]), want, HALF["bf16"] * np.abs(want) + 2.0 ** -11 * size)
    r, h, part = orc.residual_norm(start, f64(room["y"]), None, "none", 1.0, None, f64(stack.last._keep[1]), EPS)
    off = U * np.abs(r) + PART * np.abs(part)
    assert_within("x", f64(x), r, off + HALF["bf16"] * np.abs(r))
    inv = np.abs(h / np.where(r == 0, 1, r))
    assert_within("last norm", f64(room["final"]), h, inv * off + np.abs(h) * (NORM + np.linalg.norm(off, axis=-1, keepdims=True) / np.linalg.norm(r, axis=-1, keepdims=True) + HALF["bf16"]))


@pytest.mark.parametrize("B", [1, 5, 70, 300])
def test_tokens_from_a_graph(B):
    """Decode steps through two blocks from a captured graph, other work between the replays: as the eager ones, bit for bit."""
    stack, gen = stack_of(2, 384, 6, 64)
    token = torch.randn(B, 384, device="cuda", generator=gen).to(torch.bfloat16)
    begin = [[0.1 * torch.randn(B, 6, 64, 64, device="cuda", generator=gen) for _ in range(2)] for _ in range(2)]

    def fresh():
        return [[t.clone() for t in pair] for pair in begin]

    S, x, room = fresh(), token.clone(), stack.room(B)
    call = layer_call(stack, B, 1, S, decode=True)
    eager = []
    for _ in range(4):
        x.copy_(token)
        eager.append(stack.run(x, room, call).clone())
    states = [[t.clone() for t in pair] for pair in S]
    for pair, first in zip(S, begin):
        for t, f in zip(pair, first):
            t.copy_(f)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        x.copy_(token)
        out = stack.run(x, room, call)
    for want in eager:
        graph.replay()
        noise = torch.randn(1 << 18, device="cuda", generator=gen).sum()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.isfinite(noise)
    assert all(torch.equal(a, b) for p, q in zip(S, states) for a, b in zip(p, q))


@pytest.mark.parametrize("rows", [3, 130, 700])
def test_two_streams_and_repetition(rows):
    """Calls on two streams at once, on the same operands: no call keeps anything, results repeat bit for bit."""
    stack, gen = stack_of(1, 1024, 8, 128)
    x = torch.randn(rows, 1024, device="cuda", generator=gen).to(torch.bfloat16)
    rooms, streams = [stack.room(rows) for _ in range(3)], [torch.cuda.Stream() for _ in range(2)]
    identity = lambda l, q, k, v, g1, g2, o: o.copy_(q)
    want = stack.run(x.clone(), rooms[2], identity).clone()
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    for _ in range(3):
        copies = []
        for s, room in zip(streams, rooms):
            with torch.cuda.stream(s):
                copies.append(x.clone())
                stack.run(copies[-1], room, identity)
        torch.cuda.synchronize()
        assert all(torch.equal(room["final"], want) for room in rooms[:2])


def test_rows_do_not_depend_on_each_other():
    """A row's results are the same whatever stands in the other rows of its batch (batches of one size)."""
    stack, gen = stack_of(1, 640, 4, 128)
    a, b = (torch.randn(33, 640, device="cuda", generator=gen).to(torch.bfloat16) for _ in range(2))
    b[7] = a[7]
    b[9] = float("nan")
    identity = lambda l, q, k, v, g1, g2, o: o.copy_(q)
    first, second = (stack.run(t.clone(), stack.room(33), identity) for t in (a, b))
    assert torch.equal(first[7], second[7]) and torch.isnan(second[9]).all() and torch.isfinite(second[8]).all()


def test_the_command(capsys):
    serving_step.blocks(2, 3, 65, 256, 4, 64, 2)
    line = json.loads(capsys.readouterr().out.strip().splitlines()[-1])
    assert line["finite"] and line["prefill_us"] > 0 and line["decode_graph_us"] > 0 and line["prefill_kernels_us"]["project_fp8"] > 0


def test_arguments_the_binding_refuses():
    """Types, sizes and devices of tensors, with and without the native calls."""
    x, y = torch.zeros(4, 256, device="cuda", dtype=torch.bfloat16), torch.zeros(4, 256, device="cuda")
    q, s = torch.zeros(4, 256, device="cuda", dtype=torch.uint8).view(torch.float8_e4m3fn), torch.zeros(4, 4, device="cuda")
    w = torch.ones(256, device="cuda")
    norm = dsla.make_norm(256, x_dtype=dsla.DSLA_BF16, y_dtype=dsla.DSLA_BF16, h_dtype=dsla.DSLA_BF16, pre_weight=w)
    with pytest.raises(TypeError):
        dsla.dsla_residual_norm(norm, x, y, x, x.clone())
    with pytest.raises(ValueError):
        dsla.dsla_residual_norm(norm, x, x[:3], x, x.clone())
    with pytest.raises(ValueError):
        dsla.dsla_residual_norm(norm, x.view(-1)[:1000], None, None, x.clone())
    with pytest.raises((AssertionError, ValueError)):
        dsla.dsla_residual_norm(norm, x.cpu(), x, x, x.clone())
    with pytest.raises(AssertionError):
        dsla.dsla_residual_norm(norm, x.t().contiguous().t(), x, x.clone(), x.clone())
    with pytest.raises(TypeError):
        dsla.dsla_quantize(x, x.clone(), s)
    with pytest.raises(TypeError):
        dsla.dsla_quantize(x, q, s.to(torch.bfloat16))
    with pytest.raises(ValueError):
        dsla.dsla_quantize(x, q, s[:3])
    with pytest.raises((ValueError, dsla.DslaError)):   # (the scales are as many as for 4 rows)
        dsla.dsla_quantize(x, q, s, block_rows=64)
    W, ws = torch.zeros(48, 256, device="cuda", dtype=torch.uint8).view(torch.float8_e4m3fn), torch.zeros(1, 4, device="cuda")
    out = lambda n, rows=4, **k: torch.zeros(rows, n, device="cuda", **k)
    dsla.dsla_project_fp8(q, s, W, ws, [out(48)])
    for bad in ([out(32)], [out(48, 5)], [out(32), out(32)], []):
        with pytest.raises(ValueError):
            dsla.dsla_project_fp8(q, s, W, ws, bad)
    with pytest.raises(ValueError):
        dsla.dsla_project_fp8(q, s, W, ws, [out(16), out(32)])   # two outputs have two rows of scales
    with pytest.raises(TypeError):
        dsla.dsla_project_fp8(q, s, W, ws.to(torch.bfloat16), [out(48)])
    with pytest.raises(TypeError):
        dsla.dsla_project_fp8(q, s, W, ws, [out(48, dtype=torch.float16)])
    with pytest.raises(ValueError):
        dsla.dsla_project_fp8(q, s, W, ws, [out(48)], bias=torch.zeros(47, device="cuda"))
    with pytest.raises(dsla.DslaError):
        dsla.dsla_project_fp8(q[:0], s[:0], W, ws, [out(48, 0)])


def test_without_the_native_calls(monkeypatch):
    """Both ways of the binding give the same bits."""
    from paper_2506_09316_amd import binding
    stack, gen = stack_of(1, 512, 4, 64)
    x = torch.randn(9, 512, device="cuda", generator=gen).to(torch.bfloat16)
    identity = lambda l, q, k, v, g1, g2, o: o.copy_(v)
    want = stack.run(x.clone(), stack.room(9), identity).clone()
    monkeypatch.setattr(binding, "_native", binding._General)
    assert torch.equal(stack.run(x.clone(), stack.room(9), identity), want)
