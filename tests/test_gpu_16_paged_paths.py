"""The calls on a paged cache where their kernels take other paths: every size of tile with scales of every kind, far pages through LDS, refusals
among many entries and many pages, heads in several passes (bounds: paged_common)."""
import numpy as np
import pytest
import torch

import paper_2506_09316_amd as dsla
from tests.paged_common import GpuCache, bits, gpu, values
from tests.test_gpu_09_qk_rope import compare, frequencies
from tests.test_gpu_10_attention_paged import check, held, tree_of
from tests.util import code

pytestmark = pytest.mark.gpu


# heads, tokens of two entries: rows of a key/value head up to 16, 32, 48 and 64 (halves of a block to each pair of wavefronts), 128, several tiles
@pytest.mark.parametrize("H, H_kv, counts", [(4, 1, [4, 1]), (8, 1, [4, 3]), (4, 2, [16, 9]), (6, 1, [8, 2]), (2, 2, [64, 33]), (8, 1, [16, 5]), (7, 1, [64, 40])])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_scales_in_every_tile(dtype, d, H, H_kv, counts):
    """Scores of hundreds, whose references rise from block to block; of zero (plain means); of the other sign; with masks and without."""
    lens = [700, counts[1] + 30]
    c, x = held(lens, counts, H_kv=H_kv, d=d, page=32, dtype=dtype, seed=d + H)
    q = values((sum(counts), H, d), dtype, 12, 8.0)
    masks = tree_of(counts, np.random.default_rng(H))
    for scale, tree in ((4.0, None), (-4.0, masks), (0.0, None), (0.0, masks), (-1.0, None), (-0.02, masks), (0.05, None)):
        check(c, x, q, scale, 700, tree, dtype)
    assert c.status.item() == 0


@pytest.mark.parametrize("n", [17, 33, 64])
def test_far_pages_of_many_rows(n):
    """A pool of over 2^32 bytes: the same tokens in its last pages and in its first ones, 34 to 128 rows."""
    n_pages, H_kv, page, d, H = 33000, 8, 64, 128, 16
    pools = [torch.zeros(n_pages, H_kv, page, d, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    for i, p in enumerate(pools):
        p[:12] = values((12, H_kv, page, d), "bf16", 20 + i)
        p[-12:] = p[:12]
    refs, q = torch.ones(n_pages, dtype=torch.int32, device="cuda"), values((n, H, d), "bf16", 30)
    out = []
    for first in (0, n_pages - 12):
        cache = dsla.make_cache(gpu([range(first, first + 12)]), gpu([750]), refs, page=page, H_kv=H_kv, d=d, dtype=1)
        batch = dsla.make_batch(gpu([750 - n]), n, cu=gpu([0, n]), max_n=n)
        need = dsla.dsla_attention_paged_workspace_bytes(cache, batch, H, 750)
        o = torch.empty_like(q)
        dsla.dsla_attention_paged(cache, batch, q, *pools, o, 0.1, 750, workspace=torch.empty(max(need, 16), dtype=torch.uint8, device="cuda"))
        out.append(o)
    assert torch.equal(*out) and out[0].isfinite().all() and out[0].abs().max() > 0


def many(n_pages, n_seqs, max_pages=4):
    return GpuCache(n_pages, 16, n_seqs, max_pages, H_kv=1, n_pools=1)


@pytest.mark.parametrize("B", [257, 1024, 1100])
def test_many_entries_refused(B):
    """Rows named twice, the second time more than a planning workgroup behind; offsets and rows out of range; full rows; bad lengths and pages."""
    c = many(3 * B, B)
    held_ = [(7 * i) % 40 for i in range(B)]
    c.extend(c.batch(list(range(B)), held_))
    rows = [int(r) for r in np.random.default_rng(B).permutation(B)]
    rows[B - 1], rows[B // 2], rows[B // 3], rows[9] = rows[2], rows[3], B, -1          # twice, twice, out of range, out of range
    cu = np.concatenate([[0], np.cumsum([1 + i % 3 for i in range(B)])])
    cu[5], cu[B - 20] = -3, cu[B] + 5                                                    # two entries each cannot be
    table, lens = c.table.cpu().numpy().copy(), c.lens.tolist()
    bad = [s for s in range(B) if s in rows[20:60] and lens[s] % 16]
    table[bad[0], (lens[bad[0]] - 1) // 16], lens[bad[1]], lens[bad[2]] = 3 * B, 65, -1     # a last page that is none, lengths that cannot be
    full = bad[3]
    table[full], lens[full] = range(3 * B - 4, 3 * B), 64                                # no column left
    c.write_tables(table, lens, c.refs.cpu().numpy())
    start = c.extend(c.batch(rows, cu=cu, total=int(cu[B]), max_n=3))
    assert c.status.item() == 6 and (start < 0).sum() >= 10 and (start >= 0).sum() > B // 2


@pytest.mark.parametrize("B, spare", [(257, 0), (257, 100), (1100, 700), (1100, 870), (1100, 879), (1100, 880)])
def test_many_entries_short_of_pages(B, spare):
    """Pages for the first `spare` entries that need one; later ones are left out, those that need none are served."""
    c = many(B + spare, B)
    c.extend(c.batch(list(range(B)), [16 if s % 5 else 15 for s in range(B)]))
    rows = [int(r) for r in np.random.default_rng(B).permutation(B)]
    start = c.extend(c.batch(rows))
    served = int((start >= 0).sum())
    needy = sum(1 for r in rows if r % 5)
    assert served == B - needy + min(spare, needy) and (c.status.item() == 2) == (spare < needy)
    c.status.zero_()
    c.oracle.status = 0
    c.extend(c.batch(rows, [40] * B))                                                   # three pages each: fewer are served, in order


def test_many_entries_share_and_run_short():
    """Branches whose last page is shared: copies while pages last."""
    B = 300
    c = many(460, B)
    c.extend(c.batch(list(range(100)), [20] * 100))
    c.fork([-1] * 100 + [s % 100 for s in range(200)])
    start = c.extend(c.batch(list(range(B)), [1] * B))
    assert (start >= 0).sum() == 260 and c.status.item() == 2


def test_many_pages_short_and_refused():
    """More pages than the kernel for few entries takes, of which a handful are free, the last ones."""
    n_pages = 131072 + 128
    c = GpuCache(n_pages, 16, 9, 6, n_pools=0)
    table, lens, refs = np.full((9, 6), -1), np.zeros(9, int), np.ones(n_pages, int)
    table[0, :2], lens[0] = [7, 8], 32
    table[1, :2], lens[1] = [9, n_pages], 20                                            # its last page is none
    table[2, :1], lens[2] = [11], 16
    table[3, :1], lens[3] = [11], 5                                                     # shared, not full
    refs[11] = 2
    refs[[3, n_pages - 70, n_pages - 2, n_pages - 1]] = 0
    c.write_tables(table, lens, refs)
    assert c.extend(c.batch([0, 1, 3, 0, 12, 2, 4], [1, 1, 2, 1, 1, 17, 1])).tolist() == [32, -1, 5, -1, -1, 16, -1]
    assert c.status.item() == 6
    assert c.table[0, 2].item() == 3 and c.table[3, 0].item() == n_pages - 70 and c.table[2, 1:3].tolist() == [n_pages - 2, n_pages - 1]
    c.compact()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("M", [512, 513, 1400])
@pytest.mark.parametrize("H, H_kv, d, rot, interleaved", [(32, 8, 128, 128, False), (64, 8, 64, 32, True), (5, 40, 128, 64, True)])
def test_heads_in_several_passes(H, H_kv, d, rot, interleaved, M, dtype):
    """More heads than a workgroup holds at a time, on both sides of 512 tokens: with pages, with norms, in place."""
    c = GpuCache(100, 32, 3, 60, H_kv=H_kv, d=d, dtype=dtype)
    c.extend(c.batch([2, 0], [100, 33]))
    x = c.batch([2, 0], [M - 200, 200])
    start = c.extend(x)
    q, k, v = values((M, H, d), dtype, 1, 2.0), values((M, H_kv, d), dtype, 2), values((M, H_kv, d), dtype, 3)
    wq, wk, freq = *[1 + 0.3 * values((d,), "f32", 4 + i) for i in range(2)], frequencies(rot)
    rope = dsla.make_rope(H, H_kv, d, io_dtype=code(dtype), inv_freq=freq, interleaved=interleaved, q_weight=wq, k_weight=wk)
    q_out, k_out = q.clone(), k.clone()
    dsla.dsla_qk_rope(rope, q_out, k_out, v, q_out, k_out, c.desc, x, c.pools[0], c.pools[1])
    entry, j = np.repeat([0, 1], [M - 200, 200]), np.concatenate([np.arange(M - 200), np.arange(200)])
    position = np.asarray(start)[entry] + j
    compare("q", q_out, q, wq, position, freq, interleaved, dtype)
    compare("k", k_out, k, wk, position, freq, interleaved, dtype)
    pages = c.oracle.table[np.array([2, 0])[entry], position // 32]
    for pool, want in ((0, bits(k_out)), (1, bits(v))):
        c.oracle.pools[pool][pages, :, position % 32] = want
    c.same()
