"""Shared by the tests of the paged cache: a cache on the GPU beside the oracle's, and the bounds of the results.

Bounds, for one element, before any was run.  u = 2^-24 (half a step of fp32), w = 2^-8 (of bf16), both relative.
  rotation: the root mean square sums 2 x 8 squares in a lane and doubles at most three times more: 19 u, halved by the root; root,
    division and the two products of the norm 4 u: below 14 u of a feature.  Cosine and sine: the fraction of a turn is rounded
    to 32 bits, pi u, and the functions are within 2 u: below 6 u.  Two products and a sum: 3 u.  Together 23 u, held to 32 u, of the
    two features' absolute values, and the rounding to the type.
  attention: a score is a sum of d products in any order, scaled: (d + 4) u of sum |q||k| scale, and the weight exp(score - top) is off
    by twice that and the exponential's 4 u; the sums over L keys, taken in any order and rescaled, by (L + 64) u; all of the weighted
    mean of |v|.  In bf16 the weights are rounded for the second product, w; at the end w of the result.
"""
import numpy as np
import torch

import paper_2506_09316_amd as dsla
from oracle import paged as orc
from tests.util import code

U, W = 2.0 ** -24, 2.0 ** -8
TORCH = {"bf16": torch.bfloat16, "f32": torch.float32}


def gpu(x, dtype=torch.int32):
    return None if x is None else torch.tensor(np.asarray(x), dtype=dtype, device="cuda")


def values(shape, dtype, seed, std=1.0):
    g = torch.Generator()
    g.manual_seed(seed)
    return (torch.randn(*shape, generator=g) * std).to(TORCH[dtype]).cuda()


def f64(t):
    return t.detach().double().cpu().numpy()


def bits(t):
    return t.view(torch.int16 if t.dtype == torch.bfloat16 else torch.int32).cpu().numpy()


class GpuCache:
    """A cache on the GPU and the oracle's, kept alike; pools are compared as bits."""

    def __init__(self, n_pages, page, n_seqs, max_pages, *, H_kv=2, d=64, dtype="bf16", n_pools=2, seed=0, fill=None):
        self.dtype, self.H_kv, self.d = dtype, H_kv, d
        self.table, self.lens, self.refs = (torch.full(s, 77, dtype=torch.int32, device="cuda") for s in ((n_seqs, max_pages), (n_seqs,), (n_pages,)))
        self.status = torch.zeros(1, dtype=torch.int32, device="cuda")
        if fill is None:
            self.pools = [values((n_pages, H_kv, page, d), dtype, 100 * seed + i) for i in range(n_pools)]
        else:
            self.pools = [torch.full((n_pages, H_kv, page, d), fill, dtype=TORCH[dtype], device="cuda") for i in range(n_pools)]
        self.desc = dsla.make_cache(self.table, self.lens, self.refs, page=page, H_kv=H_kv, d=d, dtype=code(dtype), status=self.status)
        self.handles = dsla.make_pools(self.pools)
        self.oracle = orc.Cache(n_pages, page, n_seqs, max_pages, [bits(p).copy() for p in self.pools])
        self.ws = torch.full((dsla.dsla_cache_workspace_bytes(self.desc, n_seqs),), 255, dtype=torch.uint8, device="cuda")
        dsla.dsla_cache_init(self.desc)

    def batch(self, rows, counts=None, *, total=None, start=None, max_n=None, cu=None, with_row=True):
        """An entry for each of rows, of counts[b] tokens (one each: no offsets)."""
        cu = cu if cu is not None else None if counts is None else np.concatenate([[0], np.cumsum(counts)])
        total = total if total is not None else len(rows) if cu is None else int(cu[-1])
        x = dsla.make_batch(gpu(start if start is not None else [-7] * len(rows)), total, cu=gpu(cu), row=gpu(rows) if with_row else None,
                            max_n=max_n or max(counts or [1]))
        x.plain = (cu, list(rows), total)
        return x

    def start(self, x):
        return x._keep[0]

    def extend(self, x):
        dsla.dsla_cache_extend(self.desc, x, self.handles, self.ws)
        want = self.oracle.extend(*x.plain)
        self.same()
        assert self.start(x).tolist() == want.tolist()
        return want

    def truncate(self, new_lens):
        dsla.dsla_cache_truncate(self.desc, gpu(new_lens))
        self.oracle.truncate(new_lens)
        self.same()

    def fork(self, parent):
        dsla.dsla_cache_fork(self.desc, gpu(parent))
        self.oracle.fork(parent)
        self.same()

    def accept(self, x, path, n_accepted):
        dsla.dsla_cache_accept(self.desc, x, gpu(path), gpu(n_accepted), self.handles, self.ws)
        cu, rows, total = x.plain
        self.oracle.accept(cu, rows, total, self.start(x).tolist(), path, n_accepted)
        self.same()

    def compact(self):
        live = torch.full((1,), -5, dtype=torch.int32, device="cuda")
        dsla.dsla_cache_compact(self.desc, live, self.handles, self.ws)
        want = self.oracle.compact()
        self.same()
        assert live.item() == want
        return want

    def same(self):
        o = self.oracle
        assert np.array_equal(self.lens.cpu().numpy(), o.lens) and np.array_equal(self.refs.cpu().numpy(), o.refs)
        assert np.array_equal(self.table.cpu().numpy(), o.table)
        assert self.status.item() == o.status
        for got, want in zip(self.pools, o.pools):
            assert np.array_equal(bits(got), want)

    def write_tables(self, table, lens, refs=None):
        """A program's own tables, in the place of the library's."""
        refs = np.bincount(np.asarray(table)[np.asarray(table) >= 0].ravel(), minlength=self.oracle.n_pages) if refs is None else refs
        for t, x in ((self.table, table), (self.lens, lens), (self.refs, refs)):
            t.copy_(gpu(x))
        self.oracle.table, self.oracle.lens, self.oracle.refs = (np.asarray(x, np.int32).copy() for x in (table, lens, refs))


def attention_bound(o, size, reach, L, d, dtype):
    b = size * ((2 * (d + 4) * U * reach[..., None]) + (4 + 64 + L) * U)
    return b if dtype == "f32" else b + W * size + W * np.abs(o)


def assert_within(name, got, want, bound):
    """Element by element; infinities and NaN in the same places."""
    fine = np.isfinite(want)
    assert np.array_equal(np.isnan(got), np.isnan(want)), f"{name}: NaN in other places"
    other = ~fine & ~np.isnan(want)
    assert np.array_equal(got[other], want[other]), f"{name}: infinities in other places"
    off = np.abs(got[fine] - want[fine])
    share = off / np.maximum(bound[fine], 1e-300)
    print(f"    {name}: largest error {off.max() if off.size else 0:.3e}, {share.max() if off.size else 0:.3f} of its bound", flush=True)
    assert not off.size or share.max() <= 1, f"{name}: {share.max()} of the bound"
