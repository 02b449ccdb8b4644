"""Where the sizes that attention over a paged cache takes end: both sides of the limit that the header states, on the CPU."""
import ctypes

import pytest

from tests.test_paged_abi import P, SHAPE, WORKSPACE, batch, cache, lib  # noqa: F401


def tiles(rows, dtype):
    """Tiles of a key/value head's rows (tokens times heads of its group), as include/dsla.h counts them."""
    size = 16 if rows <= 16 else 32 if rows <= 32 else 128 if dtype == 1 else 64
    return -(-rows // size)


def sizes(lib, B, H, H_kv, max_n, max_pages, page, dtype):
    """(workspace bytes, status of the call without a workspace)"""
    c = ctypes.byref(cache(H_kv=H_kv, max_pages=max_pages, page=page, dtype=dtype, n_seqs=1 << 23))
    x = ctypes.byref(batch(B=B, max_n=max_n, total=B * max_n))
    n = lib.dsla_attention_paged_workspace_bytes(c, x, H, 1000)
    return n, lib.dsla_attention_paged(c, x, H, 1000, 1.0, P, P, ctypes.c_void_p(8192), None, P, None, 0, None)


@pytest.mark.parametrize("B, H, H_kv, max_n, max_pages", [(511, 64, 8, 64, 64), (512, 64, 8, 64, 64), (256, 128, 8, 64, 128), (1024, 128, 8, 16, 128),
                                                          (4096, 32, 8, 32, 512), (1 << 16, 32, 32, 1, 16), (64, 4096, 1, 64, 16)])
@pytest.mark.parametrize("dtype", [0, 1])
def test_many_requests_with_many_rows(lib, dtype, B, H, H_kv, max_n, max_pages):
    """What the stated limit allows is not refused for another one."""
    assert B * H_kv * tiles(max_n * H // H_kv, dtype) * (max_pages * 64 // 128 + 3) < 10 ** 9
    need, status = sizes(lib, B, H, H_kv, max_n, max_pages, 64, dtype)
    assert need > 0 and status == WORKSPACE


@pytest.mark.parametrize("H, H_kv, max_n", [(1, 1, 1), (16, 1, 1), (17, 1, 1), (8, 2, 8), (33, 1, 1), (64, 1, 1), (65, 1, 1), (8, 1, 16), (129, 1, 1),
                                            (64, 8, 64), (4096, 1, 64)])
@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("max_pages, page", [(1, 16), (9, 16), (1000, 64), (1 << 20, 128)])
def test_both_sides_of_the_limit(lib, max_pages, page, dtype, H, H_kv, max_n):
    one = H_kv * tiles(max_n * H // H_kv, dtype) * (max_pages * page // 128 + 3)
    B = (10 ** 9 - 1) // one   # the most entries that are allowed
    if 1 <= B <= 1 << 23:
        need, status = sizes(lib, B, H, H_kv, max_n, max_pages, page, dtype)
        assert need > 0 and status == WORKSPACE
    if B + 1 <= 1 << 23:
        assert sizes(lib, B + 1, H, H_kv, max_n, max_pages, page, dtype) == (0, SHAPE)
