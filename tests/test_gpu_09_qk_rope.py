"""Norm and rotation of q and k, keys and values into pages, against the oracle in fp64 (bounds: paged_common)."""
import numpy as np
import pytest
import torch

import paper_2506_09316_amd as dsla
from oracle import paged as orc
from tests.paged_common import GpuCache, TORCH, U, W, assert_within, bits, f64, gpu, values
from tests.util import code

pytestmark = pytest.mark.gpu


def frequencies(rot, theta=10000.0):
    return torch.tensor([theta ** (-2 * i / rot) for i in range(rot // 2)], dtype=torch.float32, device="cuda")


def bound(want, size, dtype):
    return 32 * U * size + (W * np.abs(want) if dtype == "bf16" else U * np.abs(want))


def compare(name, got, x, weight, position, freq, interleaved, dtype, eps=1e-6):
    want, size = orc.rotate(f64(x), None if weight is None else f64(weight), eps, position, f64(freq) if freq is not None else [], interleaved)
    assert_within(name, f64(got), want, bound(want, size, dtype))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("M, H, H_kv, d, rot, interleaved, norm", [
    (1, 32, 32, 128, 128, False, True), (7, 8, 2, 128, 64, True, False), (33, 5, 5, 64, 64, False, True), (3, 4, 1, 64, 16, True, True),
    (130, 12, 4, 64, 48, False, False), (5, 6, 3, 128, 0, False, True), (2, 1, 1, 128, 112, True, True), (4100, 3, 1, 64, 64, False, True)])
def test_without_a_cache(dtype, M, H, H_kv, d, rot, interleaved, norm):
    q, k = values((M, H, d), dtype, 1, 2.0), values((M, H_kv, d), dtype, 2)
    wq, wk = [1 + 0.3 * values((d,), "f32", 3 + i) for i in range(2)] if norm else (None, None)
    freq = frequencies(rot) if rot else None
    q_out, k_out = torch.full_like(q, float("nan")), torch.full_like(k, float("nan"))
    rope = dsla.make_rope(H, H_kv, d, io_dtype=code(dtype), inv_freq=freq, interleaved=interleaved, q_weight=wq, k_weight=wk)
    dsla.dsla_qk_rope(rope, q, k, None, q_out, k_out)
    compare("q", q_out, q, wq, np.arange(M), freq, interleaved, dtype)
    compare("k", k_out, k, wk, np.arange(M), freq, interleaved, dtype)
    # the same in place, at places of the caller's, far ones and ones before zero among them
    offsets = np.random.default_rng(5).integers(-1000, 2 ** 20, M).astype(np.int32)
    offsets[0] = 2 ** 31 - 1
    rope = dsla.make_rope(H, H_kv, d, io_dtype=code(dtype), inv_freq=freq, interleaved=interleaved, q_weight=wq, k_weight=wk, offsets=gpu(offsets))
    q2, k2 = q.clone(), k.clone()
    dsla.dsla_qk_rope(rope, q2, k2, None, q2, k2)
    compare("q in place", q2, q, wq, offsets, freq, interleaved, dtype)
    compare("k in place", k2, k, wk, offsets, freq, interleaved, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("counts, held, H, H_kv, d, page", [
    (None, [0, 5, 16, 100], 4, 4, 64, 16), ([3, 0, 40, 1], [0, 9, 30, 63], 6, 2, 128, 32), ([700, 2, 65], [1000, 0, 127], 8, 1, 64, 64),
    ([129, 128, 127, 1], [0, 1, 128, 4000], 4, 2, 128, 128)])
def test_into_the_pages(dtype, counts, held, H, H_kv, d, page):
    """Every token in its place; pages and rows of others, and rows of the tensors behind the last entry, as they were."""
    B = len(held)
    c = GpuCache(400, page, B + 2, 300, H_kv=H_kv, d=d, dtype=dtype)
    rows = [int(x) for x in np.random.default_rng(2).permutation(B + 2)[:B]]
    c.extend(c.batch(rows, held))
    n = counts or [1] * B
    total = sum(n) + (3 if counts else 0)
    x = c.batch(rows, None if counts is None else counts, total=total)
    start = c.extend(x)
    q, k, v = values((total, H, d), dtype, 1), values((total, H_kv, d), dtype, 2), values((total, H_kv, d), dtype, 3)
    w, freq = 1 + 0.3 * values((d,), "f32", 4), frequencies(d)
    for depth in (None, np.random.default_rng(3).integers(0, 9, total)):
        q_out, k_out = torch.full_like(q, 5.0), torch.full_like(k, 5.0)
        rope = dsla.make_rope(H, H_kv, d, io_dtype=code(dtype), inv_freq=freq, q_weight=w, k_weight=None, offsets=gpu(depth))
        dsla.dsla_qk_rope(rope, q, k, v, q_out, k_out, c.desc, x, c.pools[0], c.pools[1])
        places = [(b, j) for b in range(B) for j in range(n[b])]
        position = np.array([start[b] + (j if depth is None else depth[m]) for m, (b, j) in enumerate(places)])
        m = len(places)
        compare("q", q_out[:m], q[:m], w, position, freq, False, dtype)
        compare("k", k_out[:m], k[:m], None, position, freq, False, dtype)
        assert (q_out[m:] == 5).all() and (k_out[m:] == 5).all()
        want = [p.copy() for p in c.oracle.pools]
        k_bits, v_bits = bits(k_out), bits(v)
        for i, (b, j) in enumerate(places):
            t = int(start[b]) + j
            p = c.oracle.table[rows[b], t // page]
            want[0][p, :, t % page], want[1][p, :, t % page] = k_bits[i], v_bits[i]
        for got, x_ in zip(c.pools, want):
            assert np.array_equal(bits(got), x_)
        c.oracle.pools = want
    assert c.status.item() == 0


def test_what_takes_no_part():
    """Entries without a start, offsets and rows out of range, pages that are none, places past the table: nothing is written for them."""
    c = GpuCache(20, 16, 4, 3, H_kv=2, d=64, dtype="f32")
    c.extend(c.batch([0, 1, 2, 3], [20, 20, 20, 20]))
    q, k, v = values((8, 2, 64), "f32", 1), values((8, 2, 64), "f32", 2), values((8, 2, 64), "f32", 3)
    rope = dsla.make_rope(2, 2, 64, io_dtype=0, inv_freq=frequencies(64))
    q_out = torch.full_like(q, 5.0)
    x = c.batch([0, 1, 2, 7], [2, 2, 2, 2], start=[-1, 46, -2 ** 31, 0])
    dsla.dsla_qk_rope(rope, q, k, v, q_out, None, c.desc, x, c.pools[0], c.pools[1])
    assert c.status.item() == 4                                # row 7; and row 1 has room for 48 tokens but pages for 32
    assert (q_out[[0, 1, 4, 5, 6, 7]] == 5).all() and (q_out[2:4] != 5).any()
    c.status.zero_()
    c.same()
    x = c.batch([0, 1], [4, 4], start=[47, 2 ** 31 - 3])       # the first of these has a column, but no page
    dsla.dsla_qk_rope(rope, q, k, v, q_out, None, c.desc, x, c.pools[0], c.pools[1])
    assert c.status.item() == 4
    x = c.batch([0, 1, 2], cu=[5, 2, 9, 8], total=8, start=[0, 0, 0])
    dsla.dsla_qk_rope(rope, q, k, v, q_out, None, c.desc, x, c.pools[0], c.pools[1])
    c.status.zero_()
    c.same()
    dsla.dsla_qk_rope(rope, q[:0], k[:0], v[:0], q_out[:0])     # no tokens


def test_norm_of_extremes():
    """Rows of zeros, of the smallest and the largest values, with infinities and NaN: what the formula gives."""
    for dtype in ("bf16", "f32"):
        x = torch.zeros(6, 1, 64, dtype=TORCH[dtype], device="cuda")
        x[1], x[2], x[3, 0, 5], x[4, 0, 7], x[5] = 1e-30, 1e15, float("inf"), float("nan"), -1e-3
        out = torch.empty_like(x)
        w = torch.full((64,), 2.0, device="cuda")
        dsla.dsla_qk_rope(dsla.make_rope(1, 1, 64, io_dtype=code(dtype), q_weight=w, eps=1e-5), x, x, None, out)
        got = f64(out)[:, 0]
        with np.errstate(all="ignore"):
            want, size = orc.rotate(f64(x), f64(w), 1e-5, np.zeros(6), [], False)
        fine = [0, 1, 2, 5]
        # (the smallest: products of the norm may fall below the normal range of the type)
        assert (np.abs(got[fine] - want[fine, 0]) <= bound(want, size, dtype)[fine, 0] + 1e-37).all()
        assert np.isnan(got[3, 5]) and (got[3, :5] == 0).all() and np.isnan(got[4]).all()


def test_far_pages():
    """A pool of over 2^32 bytes: the last pages."""
    n_pages, H_kv, page, d = 33000, 8, 64, 128
    table, lens, refs = gpu([[n_pages - 1, 3, n_pages - 2]]), gpu([130]), torch.ones(n_pages, dtype=torch.int32, device="cuda")
    pools = [torch.zeros(n_pages, H_kv, page, d, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    cache = dsla.make_cache(table, lens, refs, page=page, H_kv=H_kv, d=d, dtype=1)
    q, k, v = (values((130, H_kv, d), "bf16", i) for i in range(3))
    batch = dsla.make_batch(gpu([0]), 130, cu=gpu([0, 130]), max_n=64)
    k_out = torch.empty_like(k)
    dsla.dsla_qk_rope(dsla.make_rope(H_kv, H_kv, d, io_dtype=1, inv_freq=frequencies(d)), q, k, v, q, k_out, cache, batch, pools[0], pools[1])
    for got, want in zip(pools, (k_out, v)):
        assert torch.equal(got[n_pages - 1].transpose(0, 1), want[:64]) and torch.equal(got[3].transpose(0, 1), want[64:128])
        assert torch.equal(got[n_pages - 2, :, :2].transpose(0, 1), want[128:])
        assert got.count_nonzero().item() == want.count_nonzero().item()
