"""The paged cache's book-keeping and moves against the oracle, call by call: whole numbers equal, pools equal as bits."""
import numpy as np
import pytest
import torch

import paper_2506_09316_amd as dsla
from tests.paged_common import GpuCache, gpu

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n_pages, page, n_seqs, max_pages", [(1, 16, 1, 1), (70, 16, 5, 20), (64, 128, 3, 40), (1025, 32, 40, 90), (5000, 64, 300, 17)])
def test_init_and_room(n_pages, page, n_seqs, max_pages):
    c = GpuCache(n_pages, page, n_seqs, max_pages, n_pools=1)
    c.same()
    rows = list(np.random.default_rng(1).permutation(n_seqs))
    c.extend(c.batch(rows))                                    # one token each
    c.extend(c.batch(rows[: max(1, n_seqs // 2)], [(7 * i) % 50 for i in range(max(1, n_seqs // 2))]))   # some of none
    c.extend(c.batch(list(range(n_seqs)), with_row=False))
    c.truncate([0] * n_seqs)
    assert c.refs.sum().item() == 0


@pytest.mark.parametrize("seed", range(6))
def test_random_programs(seed):
    """Requests that come, fork, grow, draft, shrink and end, in an order from the seed; pages run short now and then."""
    r = np.random.default_rng(seed)
    page, n_seqs = [16, 32, 64, 128][seed % 4], int(r.integers(3, 30))
    max_pages = int(r.integers(3, 9))
    n_pages = int(r.integers(n_seqs, n_seqs * max_pages))
    c = GpuCache(n_pages, page, n_seqs, max_pages, H_kv=[1, 2, 3][seed % 3], d=[64, 128][seed % 2], dtype=["bf16", "f32"][seed // 3], n_pools=1 + seed % 3, seed=seed)
    for step in range(40):
        what = r.choice(["extend", "extend", "fork", "truncate", "accept", "compact"])
        rows = [int(x) for x in r.permutation(n_seqs)[: r.integers(1, n_seqs + 1)]]
        if what == "extend":
            c.extend(c.batch(rows, [int(r.integers(0, page * 2)) for _ in rows]) if r.random() < 0.7 else c.batch(rows))
        elif what == "fork":
            parent = np.where(r.random(n_seqs) < 0.4, r.integers(0, n_seqs, n_seqs), -1)
            c.fork(parent)
        elif what == "truncate":
            c.truncate(np.where(r.random(n_seqs) < 0.3, r.integers(0, page * max_pages, n_seqs), -1) * (r.random(n_seqs) < 0.8))
        elif what == "accept":
            counts = [int(r.integers(0, 65)) for _ in rows]
            x = c.batch(rows, counts)
            c.extend(x)
            path, accepted = [], []
            for n in counts:
                k = int(r.integers(-1, n + 1)) if n else 0
                way = sorted(int(v) for v in r.choice(n, max(k, 0), replace=False)) if n else []
                path += way + [9999] * (n - len(way))
                accepted.append(k)
            c.accept(x, path, accepted)
        else:
            c.compact()


def test_a_copy_before_a_shared_page_is_written():
    """A parent of two and a half pages, forked three ways, then all four grow: three or four copies, and the original page is free
    where all have left it; pages that are full stay shared."""
    c = GpuCache(40, 16, 6, 8)
    c.extend(c.batch([0], [40]))
    c.fork([-1, 0, 0, 0, -1, -1])
    assert c.refs.max().item() == 4
    c.extend(c.batch([2], [0]))          # none: nothing is copied
    c.extend(c.batch([2], [1]))          # one copies
    c.extend(c.batch([3, 0, 1], [1, 30, 8]))   # all that share it copy: the page is free afterwards
    assert (c.refs.cpu().numpy() == 4).sum() == 2
    c.truncate([32, 33, 0, 0, 0, 0])     # a full shared page becomes the last one, and is copied when its sequence grows
    c.truncate([20, -1, -1, -1, -1, -1])
    c.extend(c.batch([0], [3]))


def test_pages_run_short():
    c = GpuCache(10, 16, 5, 4)
    assert c.extend(c.batch([0, 1, 2, 3], [64, 60, 48, 16])).tolist() == [0, 0, -1, -1]     # the third does not fit, the fourth comes after it
    assert c.status.item() == 2
    assert c.extend(c.batch([2, 1, 3], [48, 4, 16])).tolist() == [-1, 60, -1]               # one that needs no page is served
    assert c.extend(c.batch([0], [1])).tolist() == [-1]                                     # no column left
    assert c.extend(c.batch([2, 3], [32, 0])).tolist() == [0, 0]


def test_entries_that_are_not_valid():
    """Rows out of range, named twice, offsets that run backwards or past the tensors, lengths and pages that cannot be: left out and
    reported, the others served."""
    c = GpuCache(30, 16, 4, 5)
    assert c.extend(c.batch([3, 9, 3, 0], [5, 5, 6, 5])).tolist() == [0, -1, -1, 0]
    assert c.status.item() == 4
    assert c.extend(c.batch([0, 1, 2], cu=[0, 7, 3, 9], total=9, max_n=9)).tolist() == [5, -1, 0]
    assert c.extend(c.batch([0, 1, 2], cu=[-1, 7, 9, 12], total=11, max_n=9)).tolist() == [-1, 0, -1]
    lens, table = c.lens.tolist(), c.table.cpu().numpy().copy()
    lens[0], lens[1], table[2, 0] = 10 ** 6, -3, 30          # a length beyond the table, one below zero, a page that does not exist
    c.write_tables(table, lens, c.refs.cpu().numpy())
    assert c.extend(c.batch([0, 1, 2, 3])).tolist() == [-1, -1, -1, 5]
    c.truncate([0, 0, -1, -1])
    c.fork([-1, 0, 7, -1])
    c.truncate([-1, -1, 0, 0])
    c.status.zero_()
    c.oracle.status = 0
    c.fork([-1, -1, 3, -1])                                   # of an empty one: empty
    assert c.status.item() == 0
    c.fork([-1, -1, 2, 9])                                    # of itself; of none
    assert c.status.item() == 4


def test_accepted_paths():
    c = GpuCache(60, 16, 5, 12, H_kv=3)
    x = c.batch([4, 1, 0], [64, 10, 1])
    c.extend(c.batch([4, 1], [30, 16]))
    c.extend(x)
    path = list(range(0, 64, 2)) + [0] * 32 + [3, 5, 9] + [0] * 7 + [0]
    c.accept(x, path, [32, 3, 0])
    assert c.lens.tolist() == [0, 19, 0, 0, 62]
    c.accept(x, path, [32, 3, 1])                             # no longer the last tokens: nothing
    assert c.status.item() == 4
    y = c.batch([1, 2, 3, 0], [4, 4, 4, 4])
    c.extend(y)
    c.accept(y, [1, 1, 0, 0, 2, 1, 0, 0, 0, 1, 4, 0, 0, -1, 2, 0], [2, 2, 3, 2])    # not ascending (twice), out of range (twice)
    c.accept(y, [0, 1, 2, 3] * 4, [4, -1, 5, 4])              # all; as it is; more than there are; all
    c.fork([-1, -1, -1, -1, -1])
    c.truncate([-1, -1, -1, 0, -1])
    z = c.batch([1], [3])
    c.extend(z)
    c.fork([-1, -1, -1, 1, -1])                               # a fork between the draft and its acceptance: its pages stay as they are
    before = c.lens.tolist()
    c.accept(z, [1, 2, 0], [2])
    assert c.lens.tolist() == before


def test_one_row_named_twice():
    c = GpuCache(60, 16, 5, 12)   # (a batch has no more entries than the cache has rows)
    c.extend(c.batch([0, 1, 2], [20, 40, 5]))
    x = c.batch([1, 0, 1, 1, 2], [4, 4, 4, 9, 2])
    assert c.extend(x).tolist() == [40, 20, -1, -1, 5] and c.status.item() == 4
    y = c.batch([1, 0, 1, 1, 2], [4, 4, 4, 4, 2], start=[40, 20, 40, 40, 5])
    c.accept(y, [1, 3, 0, 0, 0, 0, 0, 0, 2, 0, 0, 0, 0, 0, 0, 0, 1, 0], [2, 0, 1, 0, 1])
    assert c.lens.tolist() == [20, 42, 6, 0, 0]


def test_many_entries():
    """More entries than a wavefront, than the kernel for few, and than the planning workgroup have lanes; more pages than that kernel takes."""
    for B, n_pages in ((257, 900), (1030, 4200), (65, 131200)):
        c = GpuCache(n_pages, 16, B + 3, 4, H_kv=1, n_pools=1)
        rows = [int(r) for r in np.random.default_rng(B).permutation(B + 3)[:B]]
        c.extend(c.batch(rows, [(11 * i) % 40 for i in range(B)]))
        c.fork([rows[0] if s not in rows else -1 for s in range(B + 3)])
        x = c.batch(rows, [1 + i % 5 for i in range(B)])
        c.extend(x)
        path = [j for i in range(B) for j in ([0] if i % 5 == 0 else [1] + [0] * (i % 5))]
        c.accept(x, path, [1 if i % 3 else 0 for i in range(B)])
        c.truncate([0 if s % 2 else -1 for s in range(B + 3)])
        c.compact()
        c.extend(c.batch(rows))


def test_to_the_front():
    c = GpuCache(600, 16, 9, 80, n_pools=3)
    c.extend(c.batch(list(range(9)), [16 * 7 * (i + 1) for i in range(9)]))
    c.fork([-1] * 9)
    c.truncate([0, -1, 0, -1, 40, -1, 0, -1, 0])
    c.fork([1, -1, 3, -1, -1, -1, -1, -1, -1])
    L = c.compact()
    assert (c.refs[:L] > 0).all() and (c.refs[L:] == 0).all()
    assert c.compact() == L                                   # nothing more to do
    c.truncate([0] * 9)
    assert c.compact() == 0


def test_no_pools_and_many():
    """The tables alone (a program that moves nothing), and as many pools as a call takes."""
    c = GpuCache(20, 16, 3, 6, n_pools=0)
    c.extend(c.batch([0, 1], [20, 20]))
    c.fork([-1, -1, 0])
    c.extend(c.batch([0, 2], [1, 1]))
    c.truncate([0, -1, -1])
    c.compact()
    c = GpuCache(12, 16, 3, 6, n_pools=256, H_kv=1)
    c.extend(c.batch([0, 1], [20, 20]))
    c.fork([-1, -1, 0])
    c.extend(c.batch([2], [1]))
    c.truncate([0, -1, -1])
    c.compact()


def test_what_the_binding_refuses():
    c = GpuCache(20, 16, 3, 6)
    x = c.batch([0, 1])
    with pytest.raises(dsla.DslaError) as e:
        dsla.dsla_cache_extend(c.desc, x, c.handles, c.ws[:16])
    assert e.value.status == 4
    with pytest.raises(ValueError):                           # pools of another cache
        dsla.dsla_cache_extend(c.desc, x, dsla.make_pools([c.pools[0][:5]]), c.ws)
    with pytest.raises(dsla.DslaError):                       # one pool twice
        dsla.dsla_cache_extend(c.desc, x, dsla.make_pools([c.pools[0], c.pools[0]]), c.ws)
    with pytest.raises(ValueError):
        dsla.dsla_cache_truncate(c.desc, gpu([0, 0]))
    with pytest.raises(TypeError):
        dsla.dsla_cache_fork(c.desc, gpu([0, 0, 0], torch.int64))
    with pytest.raises(AssertionError):
        dsla.make_cache(c.table.t(), c.lens, c.refs, page=16, H_kv=2, d=64, dtype=1)
    with pytest.raises(ValueError):
        dsla.make_batch(gpu([0, 0]), 2, cu=gpu([0, 1]))
    torch.cuda.synchronize()
    c.same()
