"""CPU side of the calls on a paged cache: what they refuse (nothing is launched), errors of launches, and the oracle by hand."""
import ctypes
import os

import numpy as np
import pytest

import paper_2506_09316_amd as dsla
from oracle import paged as orc
from paper_2506_09316_amd.binding import DslaBatch, DslaCache, DslaRope
from tests.test_launch_stub import run_stubbed

OK, NULL, SHAPE, UNSUPPORTED, WORKSPACE = range(5)
P = ctypes.c_void_p(4096)


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(dsla.library_path()):
        from paper_2506_09316_amd import build
        build.build()
    return dsla.load_library()


def cache(**change):
    return DslaCache(**dict(dict(n_pages=100, page=64, H_kv=8, d=128, dtype=1, n_seqs=9, max_pages=50, table=4096, lens=4096, refs=4096, status=None), **change))


def batch(**change):
    return DslaBatch(**dict(dict(B=4, max_n=8, total=20, cu=4096, row=None, start=4096), **change))


def rope(**change):
    return DslaRope(**dict(dict(H=32, H_kv=8, d=128, io_dtype=1, rot_dim=128, interleaved=0, eps=1e-6, inv_freq=4096, q_weight=None, k_weight=None,
                                offsets=None), **change))


BAD_CACHES = [(dict(n_pages=0), SHAPE), (dict(n_pages=(1 << 30) + 1), SHAPE), (dict(H_kv=0), SHAPE), (dict(H_kv=70000), SHAPE), (dict(n_seqs=0), SHAPE), (dict(n_seqs=(1 << 23) + 1), SHAPE),
              (dict(max_pages=0), SHAPE), (dict(max_pages=1 << 25), SHAPE), (dict(page=48), UNSUPPORTED), (dict(page=0), UNSUPPORTED), (dict(page=256), UNSUPPORTED),
              (dict(d=96), UNSUPPORTED), (dict(dtype=2), UNSUPPORTED), (dict(table=None), NULL), (dict(lens=None), NULL), (dict(refs=None), NULL),
              (dict(table=4098), SHAPE), (dict(status=4097), SHAPE)]
BAD_BATCHES = [(dict(B=0), SHAPE), (dict(B=10), SHAPE), (dict(total=-1), SHAPE), (dict(total=1 << 31), SHAPE), (dict(cu=None), SHAPE), (dict(start=None), NULL),
               (dict(cu=4098), SHAPE), (dict(row=4098), SHAPE), (dict(start=4098), SHAPE)]


def calls(lib, c, x, n_pools=2, pools=(4096, 8192), ws=P, n=1 << 30):
    """Every call of the cache with these descriptors: {name: status}."""
    c, x = (ctypes.byref(v) if v is not None else None for v in (c, x))
    pools = (ctypes.c_void_p * max(1, len(pools)))(*pools) if pools is not None else None
    return dict(extend=lambda: lib.dsla_cache_extend(c, x, n_pools, pools, ws, n, None), accept=lambda: lib.dsla_cache_accept(c, x, P, P, n_pools, pools, ws, n, None),
                compact=lambda: lib.dsla_cache_compact(c, P, n_pools, pools, ws, n, None), init=lambda: lib.dsla_cache_init(c, None),
                fork=lambda: lib.dsla_cache_fork(c, P, None), truncate=lambda: lib.dsla_cache_truncate(c, P, None),
                attention=lambda: lib.dsla_attention_paged(c, x, 32, 1000, 1.0, P, P, ctypes.c_void_p(8192), None, P, ws, n, None),
                rope=lambda: lib.dsla_qk_rope(ctypes.byref(rope()), 20, P, P, P, P, None, c, x, P, ctypes.c_void_p(8192), None))


@pytest.mark.parametrize("change, status", BAD_CACHES)
def test_bad_caches(lib, change, status):
    for name, call in calls(lib, cache(**change), batch()).items():
        want = status
        assert call() == want, name
    assert lib.dsla_cache_workspace_bytes(ctypes.byref(cache(**change)), 4) == 0
    assert lib.dsla_attention_paged_workspace_bytes(ctypes.byref(cache(**change)), ctypes.byref(batch()), 32, 1000) == 0


@pytest.mark.parametrize("change, status", BAD_BATCHES)
def test_bad_batches(lib, change, status):
    for name, call in calls(lib, cache(), batch(**change)).items():
        if name in ("extend", "accept", "attention", "rope"):
            assert call() == status, name


def test_missing_descriptors(lib):
    for name, call in calls(lib, None, batch()).items():
        assert call() == NULL, name
    for name, call in calls(lib, cache(), None).items():
        if name in ("extend", "accept", "attention", "rope"):
            assert call() == NULL, name


def test_pools_and_workspaces(lib):
    need = lib.dsla_cache_workspace_bytes(ctypes.byref(cache()), 4)
    assert need > 0 and lib.dsla_cache_workspace_bytes(ctypes.byref(cache()), 10) == lib.dsla_cache_workspace_bytes(ctypes.byref(cache()), 0) == 0
    for name in ("extend", "accept", "compact"):
        try_ = lambda **kw: calls(lib, cache(), batch(), **kw)[name]()
        assert try_(n_pools=-1) == SHAPE and try_(n_pools=257, pools=[16 * i for i in range(1, 258)]) == UNSUPPORTED
        assert try_(pools=None) == NULL and try_(pools=(4096, None)) == NULL and try_(pools=(4096, 4104)) == SHAPE and try_(pools=(4096, 4096)) == SHAPE
        assert try_(ws=None) == WORKSPACE and try_(n=16) == WORKSPACE and try_(ws=ctypes.c_void_p(4104)) == SHAPE
    c = ctypes.byref(cache())
    assert lib.dsla_cache_fork(c, None, None) == lib.dsla_cache_truncate(c, None, None) == lib.dsla_cache_compact(c, None, 0, None, P, 1 << 30, None) == NULL
    assert lib.dsla_cache_accept(c, ctypes.byref(batch()), None, P, 0, None, P, 1 << 30, None) == NULL
    assert lib.dsla_cache_accept(c, ctypes.byref(batch()), P, ctypes.c_void_p(4098), 0, None, P, 1 << 30, None) == SHAPE
    big = cache(n_seqs=1 << 20, H_kv=1 << 6)
    assert lib.dsla_cache_accept(ctypes.byref(big), ctypes.byref(batch(B=(1 << 19) + 1)), P, P, 1, (ctypes.c_void_p * 1)(4096), P, 1 << 62, None) == SHAPE


def test_rope_arguments(lib):
    def call(r=None, total=20, q=P, k=P, v=P, q_out=P, k_out=None, c=None, x=None, kp=None, vp=None, **change):
        return lib.dsla_qk_rope(ctypes.byref(rope(**change)) if r is None else r, total, q, k, v, q_out, k_out, c, x, kp, vp, None)

    odd = ctypes.c_void_p(4104)
    for change, status in ((dict(H=0), SHAPE), (dict(H_kv=-1), SHAPE), (dict(H=70000), SHAPE), (dict(d=80), UNSUPPORTED), (dict(io_dtype=3), UNSUPPORTED),
                           (dict(rot_dim=-16), SHAPE), (dict(rot_dim=144), SHAPE), (dict(rot_dim=24), UNSUPPORTED), (dict(inv_freq=None), NULL),
                           (dict(q_weight=4096, eps=0.0), SHAPE), (dict(k_weight=4096, eps=float("nan")), SHAPE), (dict(k_weight=4096, eps=float("inf")), SHAPE),
                           (dict(inv_freq=4100), SHAPE), (dict(q_weight=4100), SHAPE), (dict(offsets=4098), SHAPE)):
        assert call(**change) == status, change
    assert call(total=-1) == call(total=1 << 31) == SHAPE
    assert call(q=None) == call(k=None) == call(q_out=None) == NULL and call(q=odd) == call(k_out=odd) == call(q_out=odd) == SHAPE
    assert call(total=0, q=None) == OK
    c, x, vp = ctypes.byref(cache()), ctypes.byref(batch()), ctypes.c_void_p(8192)
    assert call(c=c) == call(x=x) == call(kp=P) == call(vp=P) == call(c=c, x=x) == call(c=c, x=x, kp=P) == NULL      # all of the cache, or nothing
    assert call(c=c, x=x, kp=P, vp=P) == call(c=c, x=x, kp=odd, vp=vp) == call(c=c, x=x, kp=P, vp=vp, total=21) == SHAPE
    assert call(c=c, x=x, kp=P, vp=vp, H_kv=4) == call(c=c, x=x, kp=P, vp=vp, d=64, rot_dim=64) == SHAPE
    assert call(c=c, x=x, kp=P, vp=vp, io_dtype=0) == UNSUPPORTED and call(c=c, x=x, kp=P, vp=vp, v=None) == NULL
    assert lib.dsla_qk_rope(None, 20, P, P, P, P, None, None, None, None, None, None) == NULL


def test_attention_arguments(lib):
    def call(H=32, max_len=1000, q=P, kp=P, vp=P, tree=None, o=P, ws=P, n=1 << 40, c=None, **change):
        return lib.dsla_attention_paged(ctypes.byref(c or cache()), ctypes.byref(batch(**change)), H, max_len, 1.0, q, kp, vp, tree, o, ws, n, None)

    odd = ctypes.c_void_p(4104)
    assert call(H=0) == call(H=12) == call(H=-8) == call(max_len=-1) == call(max_n=0) == SHAPE and call(max_n=65) == UNSUPPORTED
    assert call(q=None) == call(kp=None) == call(vp=None) == call(o=None) == NULL
    assert call(q=odd) == call(kp=odd) == call(vp=odd) == call(o=odd) == call(tree=ctypes.c_void_p(4100)) == SHAPE
    assert call(total=0, q=None) == OK
    assert call(c=cache(n_seqs=1 << 20), H=1 << 15, B=1 << 16) == SHAPE and call(H=8 * 4097) == UNSUPPORTED
    assert call(c=cache(max_pages=(1 << 24) + 3), B=8, max_n=64) == SHAPE      # places of 64 x 32 rows of up to 2^30 tokens on 8 heads


LAUNCHES = r"""
from paper_2506_09316_amd.binding import DslaBatch, DslaCache, DslaRope
for n in ("dsla_cache_workspace_bytes", "dsla_attention_paged_workspace_bytes"):
    getattr(lib, n).restype = ctypes.c_size_t

def each_launch(name, launches, call):
    stub.launch_stub_reset(-1)
    assert call() == OK and stub.launch_stub_count() == launches, (name, stub.launch_stub_count())
    for n in range(launches):
        stub.launch_stub_reset(n)
        assert call() == ERR_HIP and stub.launch_stub_count() == n + 1, (name, n)

pools = (ctypes.c_void_p * 2)(4096, 8192)
for dtype in (0, 1):
    for d in (64, 128):
        c = ctypes.byref(DslaCache(100, 64, 8, d, dtype, 9, 1000, 4096, 4096, 4096, None))
        x = ctypes.byref(DslaBatch(4, 8, 20, 4096, None, 4096))
        n = size(lib.dsla_cache_workspace_bytes(c, 9))
        each_launch("init", 1, lambda: lib.dsla_cache_init(c, None))
        for k in (0, 2):
            each_launch("extend", 1 + (k > 0), lambda: lib.dsla_cache_extend(c, x, k, pools, fake, n, None))
            each_launch("accept", 2, lambda: lib.dsla_cache_accept(c, x, fake, fake, k, pools, fake, n, None))
            each_launch("compact", 2 + (k > 0), lambda: lib.dsla_cache_compact(c, fake, k, pools, fake, n, None))
        each_launch("fork", 1, lambda: lib.dsla_cache_fork(c, fake, None))
        each_launch("truncate", 1, lambda: lib.dsla_cache_truncate(c, fake, None))
        r = ctypes.byref(DslaRope(32, 8, d, dtype, d, 0, 1e-6, 4096, None, None, None))
        for total in (20, 9000):
            y = ctypes.byref(DslaBatch(4, 8, total, 4096, None, 4096))
            each_launch("rope", 1, lambda: lib.dsla_qk_rope(r, i64(total), fake, fake, fake, fake, None, c, y, fake, ctypes.c_void_p(8192), None))
            each_launch("rope", 1, lambda: lib.dsla_qk_rope(r, i64(total), fake, fake, None, fake, fake, None, None, None, None, None))
        for B, max_n, length in ((1, 1, 100), (1, 1, 50000), (9, 64, 100), (9, 64, 60000)):
            y = ctypes.byref(DslaBatch(B, max_n, 9 * 64, 4096, None, 4096))
            n = lib.dsla_attention_paged_workspace_bytes(c, y, 32, i64(length))
            call = lambda: lib.dsla_attention_paged(c, y, 32, i64(length), f32(1), fake, fake, fake, None, fake, fake, size(n), None)
            each_launch(("attention", B, max_n, length), 2 if n else 1, call)
            if n:
                assert lib.dsla_attention_paged(c, y, 32, i64(length), f32(1), fake, fake, fake, None, fake, fake, size(n - 1), None) == ERR_WORKSPACE
                assert lib.dsla_attention_paged(c, y, 32, i64(length), f32(1), fake, fake, fake, None, fake, ctypes.c_void_p(4104), size(n), None) == ERR_SHAPE
"""


def test_launch_errors_reach_the_caller(tmp_path):
    run_stubbed(tmp_path, LAUNCHES)


def test_the_oracle_by_hand():
    pool = np.arange(6 * 16).reshape(6, 1, 16, 1).astype(float)
    c = orc.Cache(6, 16, 3, 3, [pool])
    assert c.extend([0, 20, 36], [2, 0], 36).tolist() == [0, 0]
    assert c.table.tolist() == [[2, -1, -1], [-1, -1, -1], [0, 1, -1]] and c.refs.tolist() == [1, 1, 1, 0, 0, 0]
    c.fork([-1, 2, -1])
    assert c.refs.tolist() == [2, 2, 1, 0, 0, 0] and c.lens.tolist() == [16, 20, 20]
    assert c.extend(None, [1, 0], 2).tolist() == [20, 16]        # a copy of page 1 for the branch; a second page for the other
    assert c.table.tolist() == [[2, 4, -1], [0, 3, -1], [0, 1, -1]] and c.refs.tolist() == [2, 1, 1, 1, 1, 0]
    assert pool[3, 0, :5, 0].tolist() == [16, 17, 18, 19, 52]
    c.truncate([0, -1, 16])
    assert c.refs.tolist() == [2, 0, 0, 1, 0, 0] and c.table[2].tolist() == [0, -1, -1]
    assert c.compact() == 2 and c.table[1].tolist() == [0, 1, -1] and c.refs.tolist() == [2, 1, 0, 0, 0, 0] and pool[1, 0, 0, 0] == 16
    start = c.extend([0, 4], [1], 4)
    c.accept([0, 4], [1], 4, start, [1, 3, 0, 0], [2])
    assert c.lens.tolist() == [0, 23, 16] and pool[1, 0, 5:9, 0].tolist() == [54, 56, 55, 56] and c.status == 0
    # rotation: a quarter turn of (1, 0), and a norm of (3, 4): root mean square sqrt(12.5)
    y, _ = orc.rotate(np.array([[[1.0, 0.0]]]), None, 0, [1], [np.pi / 2], False)
    assert np.allclose(y, [[[0, 1]]])
    y, _ = orc.rotate(np.array([[[3.0, 4.0]]]), [1, 2], 0, [0], [1.0], True)
    assert np.allclose(y, np.array([[[3, 8]]]) / np.sqrt(12.5))
    # attention: two keys of equal score, a mask that leaves the second one
    c = orc.Cache(1, 16, 1, 1)
    c.table[0, 0] = 0
    k, v = np.zeros((1, 1, 16, 2)), np.zeros((1, 1, 16, 2))
    v[0, 0, 0], v[0, 0, 1] = [1, 2], [3, 6]
    o, _, _ = orc.attention(c, k, v, [0, 2], [0], [0], np.ones((2, 1, 2)), 1.0)
    assert o[:, 0].tolist() == [[1, 2], [2, 4]]
    o, _, _ = orc.attention(c, k, v, [0, 2], [0], [0], np.ones((2, 1, 2)), 1.0, [0, 2])
    assert o[:, 0].tolist() == [[0, 0], [3, 6]]
