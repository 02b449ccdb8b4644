"""Attention of the last tokens of every sequence over pages, against the oracle in fp64 (bounds: paged_common)."""
import numpy as np
import pytest
import torch

import paper_2506_09316_amd as dsla
from oracle import paged as orc
from tests.paged_common import GpuCache, attention_bound, assert_within, bits, f64, gpu, values

pytestmark = pytest.mark.gpu


def tree_of(counts, r):
    """A node sees its ancestors and itself."""
    masks = []
    for n in counts:
        own = []
        for j in range(n):
            own.append((own[int(r.integers(max(0, j - 6), j))] if j else 0) | 1 << j)
        masks += own
    return masks


def signed(masks):
    return gpu([m - (1 << 64) if m >> 63 else m for m in masks], torch.int64)


def held(lens, counts, *, H_kv, d, page, dtype, seed=0, spare=2, fill=float("nan")):
    """A cache whose rows hold lens[b] tokens in pages in a random order; rows past the ends, and all other pages, hold `fill`."""
    r = np.random.default_rng(seed)
    n = [-(-x // page) for x in lens]
    c = GpuCache(sum(n) + 3, page, len(lens) + spare, max(n + [1]) + 1, H_kv=H_kv, d=d, dtype=dtype, fill=fill)
    rows, order = [int(x) for x in r.permutation(len(lens) + spare)[: len(lens)]], r.permutation(sum(n) + 3)
    table, row_lens, at = np.full(c.table.shape, -1), np.zeros(len(lens) + spare, int), 0
    for b, row in enumerate(rows):
        table[row, : n[b]], row_lens[row] = order[at: at + n[b]], lens[b]
        at += n[b]
        if lens[b]:
            t = torch.arange(lens[b], device="cuda")
            pages = gpu(table[row], torch.int64)[t // page]
            for i, p in enumerate(c.pools):
                p[pages, :, t % page] = values((lens[b], H_kv, d), dtype, 1000 * seed + 10 * b + i)
    c.write_tables(table, row_lens)
    c.oracle.pools = [bits(p).copy() for p in c.pools]
    x = c.batch(rows, None if all(k == 1 for k in counts) else list(counts), start=[a - k for a, k in zip(lens, counts)], max_n=max(counts + [1]))
    return c, x


def attend(c, x, q, scale, max_len, tree=None, o=None):
    o = torch.full_like(q, 9.0) if o is None else o
    n = dsla.dsla_attention_paged_workspace_bytes(c.desc, x, q.shape[1], max_len)
    ws = torch.full((n,), 255, dtype=torch.uint8, device="cuda") if n else None
    dsla.dsla_attention_paged(c.desc, x, q, c.pools[0], c.pools[1], o, scale, max_len, tree=tree, workspace=ws)
    return o


def check(c, x, q, scale, max_len, tree=None, dtype="bf16"):
    got = f64(attend(c, x, q, scale, max_len, None if tree is None else signed(tree)))
    cu, rows, total = x.plain
    with np.errstate(all="ignore"):
        want, size, reach = orc.attention(c.oracle, f64(c.pools[0]), f64(c.pools[1]), cu, rows, c.start(x).tolist(), f64(q), float(np.float32(scale)), tree)
    n = sum(b - a for a, b in zip(cu, cu[1:])) if cu is not None else len(rows)
    assert (got[n:] == 9).all()
    assert_within("o", got[:n], want[:n], attention_bound(want, size, reach, int(c.lens.max().item()), c.d, dtype)[:n])
    return got, want


CASES = [   # lens, tokens, H, H_kv, d, page
    ([1], [1], 1, 1, 64, 16), ([2, 1, 17], [1, 1, 1], 4, 4, 128, 16), ([15, 16, 17, 31, 32, 33], [1] * 6, 8, 2, 64, 16),
    ([63, 64, 65, 127, 128, 129], [1] * 6, 4, 1, 128, 64), ([1000], [1], 32, 32, 128, 64), ([700, 3, 255, 257], [1] * 4, 16, 2, 128, 32),
    ([5000, 1, 1200], [1] * 3, 6, 2, 64, 128), ([9000], [1], 8, 1, 128, 16), ([40, 41], [2, 3], 4, 4, 64, 16), ([64, 500], [64, 33], 8, 2, 128, 64),
    ([300, 70, 64, 9], [5, 64, 17, 1], 12, 4, 64, 32), ([2500, 90], [16, 40], 10, 2, 128, 16), ([130, 64, 7], [4, 64, 7], 32, 1, 64, 128),
    ([129, 66, 48, 31], [9, 0, 3, 31], 3, 1, 128, 16), ([4100], [61], 16, 4, 128, 64)]


@pytest.mark.parametrize("tree", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_against_the_oracle(case, dtype, tree):
    lens, counts, H, H_kv, d, page = CASES[case]
    c, x = held(lens, counts, H_kv=H_kv, d=d, page=page, dtype=dtype, seed=case)
    q = values((sum(counts), H, d), dtype, 77, 1.5)
    masks = tree_of(counts, np.random.default_rng(case)) if tree else None
    check(c, x, q, d ** -0.5, max(lens), masks, dtype)
    assert c.status.item() == 0
    c.same()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_the_bound_of_the_lengths_only_plans(dtype):
    """Too small, zero and far too large a bound: the same results within the bounds."""
    c, x = held([3000, 100, 1], [3, 9, 1], H_kv=2, d=64, page=16, dtype=dtype)
    q = values((13, 4, 64), dtype, 5)
    for max_len in (0, 1, 100, 1500, 3000, 2 ** 20, 2 ** 31 - 1):
        check(c, x, q, 0.125, max_len, dtype=dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_that_see_nothing_and_masks_of_any_shape(dtype):
    """Masks that are no trees: none, all, every second, later tokens, bits past the entry's tokens; empty rows get zeros where there
    are no tokens before."""
    n = 40
    for lens in ([n, n + 1, 200], [n, 3 * n, n]):
        c, x = held(lens, [n] * 3, H_kv=2, d=64, page=16, dtype=dtype, seed=4)
        q = values((3 * n, 4, 64), dtype, 6)
        r = np.random.default_rng(7)
        masks = [[0, 2 ** 64 - 1, 0x5555555555555555, 1 << 63, 1 << (j % n), int(r.integers(0, 2 ** 63))][j % 6] for j in range(3 * n)]
        got, _ = check(c, x, q, 0.2, max(lens), masks, dtype)
        assert (got[0] == 0).all() and (got[3] == 0).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H, H_kv, n", [(4, 4, 5), (8, 1, 24), (8, 2, 64)])
def test_infinities_and_nan_where_a_query_does_not_look(dtype, H, H_kv, n):
    """Drafted tokens whose keys or values are infinite or NaN: only the queries that see them know."""
    c, x = held([n + 100, n], [n, n], H_kv=H_kv, d=64, page=16, dtype=dtype, seed=8)
    for i, bad in ((1, float("nan")), (2, float("inf")), (4, -float("inf"))):
        for row, at in zip(x.plain[1], (100, 0)):
            p = int(c.oracle.table[row, (at + i) // 16])
            c.pools[1][p, :, (at + i) % 16, 3 * i] = bad
            if i == 1:
                c.pools[0][p, :, (at + i) % 16] = bad
    q = values((2 * n, H, 64), dtype, 9)
    masks = [(1 << j | (1 if j else 0)) if j % 3 else 1 for j in range(n)] * 2
    masks[3] = masks[n + 3] = 0b10101                          # sees both infinities, of one sign each
    got, want = check(c, x, q, 0.125, n + 100, masks, dtype)
    assert np.isnan(want[1]).all() and np.isinf(want[2, :, 6]).all() and np.isfinite(want[5:n]).all() and np.isfinite(want[0]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_large_scores_and_plain_means(dtype):
    """Scores of hundreds (one key takes all), of equal keys (a mean), with a scale of zero and of minus one."""
    c, x = held([500, 33], [2, 1], H_kv=1, d=128, page=32, dtype=dtype, seed=11)
    q = values((3, 4, 128), dtype, 12, 8.0)
    for scale in (4.0, 0.0, -1.0, 0.05):
        check(c, x, q, scale, 500, dtype=dtype)


def test_what_takes_no_part():
    c, x = held([50, 60, 70, 80], [2, 3, 4, 5], H_kv=2, d=64, page=16, dtype="bf16", seed=13)
    q = values((14, 4, 64), "bf16", 14)
    c.start(x).copy_(gpu([-1, 57, -3, 75]))
    got, want = f64(attend(c, x, q, 0.125, 80)), None
    assert (got[0:2] == 9).all() and (got[5:9] == 9).all() and c.status.item() == 0
    y = c.batch(x.plain[1], [2, 3, 4, 5], start=[48, 57, 66, 75], max_n=4)          # five tokens where at most four were announced
    got = f64(attend(c, y, q, 0.125, 80))
    assert (got[9:] == 9).all() and (got[:9] != 9).any(axis=(1, 2)).all() and c.status.item() == 4
    c.status.zero_()
    y = c.batch([x.plain[1][0], 99, -1, x.plain[1][3]], [2, 3, 4, 5], start=[48, 57, 66, 2 ** 31 - 2])
    got = f64(attend(c, y, q, 0.125, 80))
    assert (got[2:] == 9).all() and (got[:2] != 9).any() and c.status.item() == 4
    # a page that is none: its tokens are not seen
    c.status.zero_()
    c.oracle.table[x.plain[1][3], 1] = 10 ** 6
    c.table.copy_(gpu(c.oracle.table))
    c.start(x).copy_(gpu([-1, -1, -1, 75]))
    got = f64(attend(c, x, q, 0.125, 80))[9:]
    want, size, reach = orc.attention(c.oracle, f64(c.pools[0]), f64(c.pools[1]), *x.plain[:2], [-1, -1, -1, 75], f64(q), 0.125)
    assert_within("o", got, want[9:], attention_bound(want, size, reach, 80, 64, "bf16")[9:])
    assert c.status.item() == 4


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B, n_hi, H, H_kv, d", [(70, 1, 4, 2, 64), (131, 3, 2, 1, 128), (66, 20, 8, 2, 64), (300, 1, 1, 1, 64)])
def test_many_entries(B, n_hi, H, H_kv, d, dtype):
    """More entries than a wavefront has lanes, some of no tokens, some that take no part, of short and long sequences."""
    r = np.random.default_rng(B)
    counts = [int(r.integers(0, n_hi + 1)) if n_hi > 1 else 1 for _ in range(B)]
    lens = [n + int(r.integers(0, [5, 60, 900][i % 3])) for i, n in enumerate(counts)]
    c, x = held(lens, counts, H_kv=H_kv, d=d, page=32, dtype=dtype, seed=B)
    start = [a - k if i % 7 else -1 for i, (a, k) in enumerate(zip(lens, counts))]
    c.start(x).copy_(gpu(start))
    q = values((sum(counts), H, d), dtype, 31)
    got = f64(attend(c, x, q, 0.1, max(lens)))
    cu, rows, total = x.plain
    want, size, reach = orc.attention(c.oracle, f64(c.pools[0]), f64(c.pools[1]), cu, rows, start, f64(q), float(np.float32(0.1)))
    part = ~np.isnan(want[:, 0, 0])
    assert (got[~part] == 9).all() and c.status.item() == 0
    assert_within("o", got[part], want[part], attention_bound(want, size, reach, max(lens), d, dtype)[part])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H, H_kv, n, page", [(8, 1, 24, 16), (4, 1, 64, 32), (2, 2, 3, 16), (16, 1, 1, 64)])
def test_pages_that_are_none(H, H_kv, n, page, dtype):
    """The first, the last and pages between: their tokens are not seen, whatever number the table has there."""
    c, x = held([400, n, 150], [n] * 3, H_kv=H_kv, d=128, page=page, dtype=dtype, seed=40)
    rows = x.plain[1]
    t = c.oracle.table
    t[rows[0], [0, 3, 399 // page]] = [-1, c.oracle.n_pages, 2 ** 31 - 1]
    t[rows[1], 0] = -2 ** 31                                   # all that it has, where one page holds it
    c.table.copy_(gpu(t))
    q = values((3 * n, H, 128), dtype, 41)
    tree = tree_of([n] * 3, np.random.default_rng(1)) if n > 1 else None
    got, _ = check(c, x, q, 0.1, 400, tree, dtype)
    assert c.status.item() == 4 and (page < n or (got[n:2 * n] == 0).all())


def test_the_same_again_and_on_another_stream():
    c, x = held([3000, 100, 700], [3, 9, 30], H_kv=2, d=128, page=16, dtype="bf16", seed=15)
    q = values((42, 8, 128), "bf16", 16)
    masks = signed(tree_of([3, 9, 30], np.random.default_rng(3)))
    want = attend(c, x, q, 0.1, 3000, masks)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    for _ in range(3):
        assert torch.equal(attend(c, x, q, 0.1, 3000, masks), want)
        with torch.cuda.stream(s):
            got = attend(c, x, q, 0.1, 3000, masks)
        s.synchronize()
        assert torch.equal(got, want)


def test_far_pages():
    """A pool of over 2^32 bytes: the same tokens in its last pages and in its first ones."""
    n_pages, H_kv, page, d, H = 33000, 8, 64, 128, 16
    pools = [torch.zeros(n_pages, H_kv, page, d, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    for i, p in enumerate(pools):
        p[:12] = values((12, H_kv, page, d), "bf16", 20 + i)
        p[-12:] = p[:12]
    refs, q = torch.ones(n_pages, dtype=torch.int32, device="cuda"), values((5, H, d), "bf16", 30)
    out = []
    for first in (0, n_pages - 12):
        cache = dsla.make_cache(gpu([range(first, first + 12)]), gpu([750]), refs, page=page, H_kv=H_kv, d=d, dtype=1)
        batch = dsla.make_batch(gpu([745]), 5, cu=gpu([0, 5]), max_n=5)
        n = dsla.dsla_attention_paged_workspace_bytes(cache, batch, H, 750)
        o = torch.empty_like(q)
        dsla.dsla_attention_paged(cache, batch, q, *pools, o, 0.1, 750, workspace=torch.empty(max(n, 16), dtype=torch.uint8, device="cuda"))
        out.append(o)
    assert torch.equal(*out) and out[0].isfinite().all() and out[0].abs().max() > 0
