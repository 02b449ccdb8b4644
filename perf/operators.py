"""Cases of the paged cache, of the attention that reads it and of the rotation that fills it.

A softmax layer of a partly converted model keeps its keys and values in pages: pools [n_pages][H_kv][page][d], a table
[n_seqs][max_pages] of the pages of every request, its length, and how often each page is named (0 = free).  One batch
description (B entries, token offsets, cache rows, where each entry's tokens start) goes through all calls of a step.

The kinds of cases:
  rope     norm and rotation of q and k for every head, keys and values written into their pages (dsla_qk_rope)
  attn     the last tokens of every request, one or a tree of drafted ones, over the pages (dsla_attention_paged)
  step     room for the next tokens, after those of the last attempt were given up (dsla_cache_truncate, dsla_cache_extend)
  fork     requests forked into branches, each with its first token of its own (dsla_cache_fork, dsla_cache_extend)
  compact  requests that end and come, pages moved to the front of the pools between (dsla_cache_compact)
  turn     a turn of drafting on one layer: all of the above that take part in it, and dsla_cache_accept

Plain forms are elementary torch operations in 32 bits, angles in 64.
"""
import math

import numpy as np
import torch

own = False

THETA = 10000.0   # base of the rotation frequencies
EPS = 1e-6        # of the norms


def listed():
    return [
        # an interactive user's next token: q and k of one token, latency
        dict(name="rope_b1", kind="rope", B=1, lo=1, hi=1, H=32, Hkv=32, d=128, io="bf16", norm=0, rot=128, pairs="halves", page=64, past=1000),
        # a mixed batch of prompts, 16000 tokens in all, some of them far into long conversations
        dict(name="rope_16k", kind="rope", B=6, lo=700, hi=6050, H=32, Hkv=8, d=128, io="bf16", norm=1, rot=128, pairs="halves", page=64, past=40000),
        # the fp32 arithmetic of a reference run: half of each head rotated, neighbours paired, small pages
        dict(name="rope_f32", kind="rope", B=3, lo=33, hi=400, H=4, Hkv=4, d=64, io="f32", norm=1, rot=32, pairs="neighbours", page=16, past=50),
        # an interactive user: one token over a short conversation, every head its own keys; latency
        dict(name="attn_b1", kind="attn", B=1, lo=1000, hi=1000, n_lo=1, n_hi=1, H=32, Hkv=32, d=128, io="bf16", page=64, tree=0),
        # a full batch of decoding requests at different context lengths, grouped heads
        dict(name="attn_b64", kind="attn", B=64, lo=100, hi=8192, n_lo=1, n_hi=1, H=32, Hkv=8, d=128, io="bf16", page=64, tree=0),
        # one long document
        dict(name="attn_128k", kind="attn", B=1, lo=131072, hi=131072, n_lo=1, n_hi=1, H=32, Hkv=8, d=128, io="bf16", page=16, tree=0),
        # trees of 17 to 64 drafted tokens over long contexts
        dict(name="attn_tree", kind="attn", B=8, lo=4000, hi=8192, n_lo=17, n_hi=64, H=32, Hkv=8, d=128, io="bf16", page=64, tree=1),
        # chains of up to five drafted tokens in fp32, narrow heads, short contexts
        dict(name="attn_f32", kind="attn", B=5, lo=7, hi=1300, n_lo=1, n_hi=5, H=8, Hkv=2, d=64, io="f32", page=32, tree=0),
        # the book-keeping of a decode step of 64 requests over 20000 small pages
        dict(name="step_b64", kind="step", B=64, lo=100, hi=8192, n_lo=1, n_hi=1, Hkv=1, d=64, io="bf16", page=16, pools=2),
        # eight requests sampled seven ways each, 16 layers: branches share the full pages and copy the last one
        dict(name="fork_8x7", kind="fork", B=8, ways=7, lo=300, hi=1500, Hkv=8, d=128, io="bf16", page=64, pools=32),
        # half of the requests end and others of the same lengths come, twice; 16 layers
        dict(name="compact_16", kind="compact", B=16, lo=200, hi=900, Hkv=8, d=128, io="bf16", page=64, pools=32),
        # a whole turn of drafting on one layer
        dict(name="turn_b8", kind="turn", B=8, lo=2000, hi=8000, n_lo=17, n_hi=64, H=32, Hkv=8, d=128, io="bf16", page=64),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["rope", "rope", "attn", "attn", "attn", "attn", "step", "fork", "compact", "turn"])
    H, Hkv, d = rng.choice([(32, 8, 128), (32, 32, 128), (32, 8, 128), (8, 1, 128), (32, 4, 64), (12, 4, 64)])
    io = "f32" if rng.random() < 0.2 else "bf16"
    page = rng.choice([16, 32, 64, 64, 128])
    if kind == "rope":
        B = _log_int(rng, 1, 64)
        hi = _log_int(rng, 1, 8000 // B)
        return dict(kind=kind, B=B, lo=_log_int(rng, 1, hi), hi=hi, H=H, Hkv=Hkv, d=d, io=io, norm=rng.randrange(2),
                    rot=rng.choice([d, d, d // 2]), pairs=rng.choice(["halves", "halves", "neighbours"]), page=page, past=_log_int(rng, 1, 100000 // B))
    if kind == "attn":
        B = _log_int(rng, 1, 64)
        hi = _log_int(rng, 70, min(131072, 524288 // B // (4 if Hkv == 32 else 1)))
        n_hi = _log_int(rng, 1, max(1, min(64, 8 * 8192 * 64 // (B * hi))))
        return dict(kind=kind, B=B, lo=_log_int(rng, n_hi, hi), hi=hi, n_lo=rng.randrange(1, n_hi + 1), n_hi=n_hi, H=H, Hkv=Hkv, d=d, io=io, page=page,
                    tree=rng.randrange(2))
    if kind == "turn":
        B, n_hi = _log_int(rng, 1, 8), _log_int(rng, 2, 64)
        hi = _log_int(rng, 100, 8000)
        return dict(kind=kind, B=B, lo=_log_int(rng, 10, hi), hi=hi, n_lo=rng.randrange(1, n_hi + 1), n_hi=n_hi, H=H, Hkv=Hkv, d=d, io=io, page=page)
    if kind == "step":
        n_hi, hi = _log_int(rng, 1, 100), _log_int(rng, 100, 8192)
        return dict(kind=kind, B=_log_int(rng, 1, 64), lo=_log_int(rng, 1, hi), hi=hi, n_lo=1, n_hi=n_hi, Hkv=1, d=64, io="bf16", page=page, pools=2)
    pools, hi = rng.choice([2, 8, 32]), _log_int(rng, 20, 900)
    c = dict(kind=kind, B=rng.randrange(1, 9), lo=_log_int(rng, 1, hi), hi=hi, Hkv=min(Hkv, 8), d=d, io=io, page=page, pools=pools)
    return dict(c, ways=rng.randrange(1, 8)) if kind == "fork" else dict(c, B=2 * c["B"])


# ---------------------------------------------------------------------------------------------------------------
def _type(io):
    return torch.bfloat16 if io == "bf16" else torch.float32


def _size(io):
    return 2 if io == "bf16" else 4


def _spread(n, lo, hi):
    """n lengths from lo to hi, evenly over their logarithm."""
    return [hi if n == 1 else int(round(lo * (hi / lo) ** (i / (n - 1)))) for i in range(n)]


def _counts(c):
    """Tokens of every entry: between n_lo and n_hi."""
    return [c["n_lo"] + (i * 37) % (c["n_hi"] - c["n_lo"] + 1) for i in range(c["B"])]


class _Draw:
    """Values on the GPU and choices on the host, from one seed."""

    def __init__(self, seed):
        self.gen = torch.Generator(device="cuda")
        self.gen.manual_seed(1000003 * int(seed) + 29)
        self.host = np.random.default_rng(1000003 * int(seed) + 29)

    def normal(self, *shape, std=1.0, dtype=torch.float32):
        return torch.empty(*shape, device="cuda", dtype=dtype).normal_(0.0, std, generator=self.gen)


def _gpu(x, dtype=np.int32):
    return torch.from_numpy(np.ascontiguousarray(np.asarray(x, dtype=dtype))).cuda()


def _cache(r, c, held, room, *, rows=None, n_pools=2, spare=None, ordered=False):
    """A cache with held[b] tokens in row rows[b], space for room[b], pages in a random order (or in the order of the entries)."""
    page, B = c["page"], len(held)
    rows = list(range(B)) if rows is None else rows
    pages = [-(-x // page) for x in held]
    n_seqs = max(rows) + 1 if spare is None else spare
    n_pages = sum(-(-x // page) for x in room) + 5
    table = np.full((n_seqs, max(-(-x // page) for x in room) + 1), -1, np.int32)
    order = np.arange(n_pages) if ordered else r.host.permutation(n_pages)
    refs, lens, at = np.zeros(n_pages, np.int32), np.zeros(n_seqs, np.int32), 0
    for b in range(B):
        table[rows[b], :pages[b]] = order[at:at + pages[b]]
        refs[order[at:at + pages[b]]] = 1
        lens[rows[b]] = held[b]
        at += pages[b]
    return dict(table=_gpu(table), lens=_gpu(lens), refs=_gpu(refs), n_pages=n_pages,
                pools=r.normal(n_pools, n_pages, c["Hkv"], page, c["d"], dtype=_type(c["io"])))


def _batch(r, counts, starts, rows):
    """Tokens packed back to back; one token each: no offsets."""
    cu = None if all(n == 1 for n in counts) else _gpu(np.concatenate([[0], np.cumsum(counts)]))
    return dict(total=sum(counts), cu=cu, rows=_gpu(rows), start=_gpu(starts), longest=max(counts))


def _trees(r, counts):
    """For every node the set of nodes on its way from the root, itself included, as 64 bits, and its depth; a path of accepted nodes."""
    masks, depths, path, accepted = [], [], [], []
    for n in counts:
        mask, depth, parent = [], [], []
        for j in range(n):
            p = int(r.host.integers(max(0, j - 8), j)) if j else -1
            parent.append(p)
            mask.append((mask[p] if j else 0) | 1 << j)
            depth.append(depth[p] + 1 if j else 0)
        leaf, way = int(r.host.integers(n)), []
        while leaf >= 0:
            way.insert(0, leaf)
            leaf = parent[leaf]
        masks += [m - (1 << 64) if m >> 63 else m for m in mask]
        depths += depth
        path += way + [0] * (n - len(way))
        accepted.append(len(way))
    return _gpu(masks, np.int64), _gpu(depths), _gpu(path), _gpu(accepted)


def prepare(case, seed):
    c, r, s = case, _Draw(seed), dict(case)
    kind, B = c["kind"], c["B"]
    dt = _type(c["io"])
    if kind == "rope":
        counts = _spread(B, c["lo"], c["hi"])
        starts = [(c["past"] * (b + 1)) // B for b in range(B)]
        rows = [int(x) for x in r.host.permutation(B + 2)[:B]]
        s["cache"] = _cache(r, c, [a + n for a, n in zip(starts, counts)], [a + n for a, n in zip(starts, counts)], rows=rows, spare=B + 2)
        s["batch"] = _batch(r, counts, starts, rows)
    elif kind in ("attn", "turn"):
        counts = _counts(c)
        held = _spread(B, c["lo"], c["hi"])
        rows = [int(x) for x in r.host.permutation(B + 3)[:B]]
        starts = [x - n for x, n in zip(held, counts)] if kind == "attn" else held
        s["cache"] = _cache(r, c, held, held if kind == "attn" else [x + n for x, n in zip(held, counts)], rows=rows, spare=B + 3)
        s["batch"] = _batch(r, counts, starts, rows)
        s["mask"], s["depth"], s["path"], s["accepted"] = _trees(r, counts)
        if kind == "attn" and not c["tree"]:
            s["mask"] = None
        s["o"] = torch.zeros(sum(counts), c["H"], c["d"], device="cuda", dtype=dt)
        if kind == "turn":
            keep = np.full(B + 3, -1, np.int32)
            keep[rows] = held
            s["keep"] = _gpu(keep)
    elif kind == "step":
        counts, held = _counts(c), _spread(B, c["lo"], c["hi"])
        rows = [int(x) for x in r.host.permutation(B)]
        s["cache"] = _cache(r, c, held, [x + n for x, n in zip(held, counts)], rows=rows, n_pools=c["pools"])
        s["batch"] = _batch(r, counts, [0] * B, rows)
        keep = np.zeros(B, np.int32)
        keep[rows] = held
        s["keep"] = _gpu(keep)
    elif kind == "fork":
        # row b: a request; rows B + ways b ..: its branches, which share its pages and then take one token each
        held, branches = _spread(B, c["lo"], c["hi"]), B * c["ways"]
        s["cache"] = _cache(r, c, held, held + [c["page"]] * 2 * branches, rows=list(range(B)), n_pools=c["pools"], spare=B + branches)
        s["batch"] = _batch(r, [1] * branches, [0] * branches, [B + i for i in range(branches)])
        s["keep"] = _gpu([-1] * B + [0] * branches)
        s["parent"] = _gpu([-1] * B + [i // c["ways"] for i in range(branches)])
    else:
        # the first half of the requests holds the front of the pools, the second, of the same lengths, what is behind
        half = _spread(B // 2, c["lo"], c["hi"])
        s["cache"] = _cache(r, c, half + half, half + half, n_pools=c["pools"], ordered=True)
        s["batch"] = [_batch(r, half, [0] * (B // 2), list(range(i * (B // 2), (i + 1) * (B // 2)))) for i in range(2)]
        s["keep"] = [_gpu([0 if (b < B // 2) == (i == 0) else -1 for b in range(B)]) for i in range(2)]
        s["live"] = torch.zeros(1, device="cuda", dtype=torch.int32)
    if kind in ("rope", "turn", "attn"):
        total = s["batch"]["total"]
        s["q"] = r.normal(total, c["H"], c["d"], std=1.5, dtype=dt)
    if kind in ("rope", "turn"):
        s["k"], s["v"] = (r.normal(total, c["Hkv"], c["d"], dtype=dt) for _ in range(2))
        s["q_out"] = torch.zeros_like(s["q"])
        s["rot"] = c.get("rot", c["d"])
        s["freq"] = torch.tensor([THETA ** (-2 * i / s["rot"]) for i in range(s["rot"] // 2)], dtype=torch.float32, device="cuda")
        s["weights"] = [1 + 0.2 * r.normal(c["d"]) for _ in range(2)] if c.get("norm", 1) else [None, None]
    if own:
        _handles(s)
    return s


def _handles(s):
    """What a program keeps for the library's calls: descriptors and workspaces."""
    import paper_2506_09316_amd as dsla
    from paper_2506_09316_amd.binding import DSLA_BF16, DSLA_F32
    c, io = s["cache"], DSLA_BF16 if s["io"] == "bf16" else DSLA_F32
    s["h_cache"] = dsla.make_cache(c["table"], c["lens"], c["refs"], page=s["page"], H_kv=s["Hkv"], d=s["d"], dtype=io)
    s["h_pools"] = dsla.make_pools(list(c["pools"]))
    batches = s["batch"] if isinstance(s["batch"], list) else [s["batch"]]
    s["h_batch"] = [dsla.make_batch(x["start"], x["total"], cu=x["cu"], row=x["rows"], max_n=x["longest"]) for x in batches]
    nbytes = dsla.dsla_cache_workspace_bytes(s["h_cache"], s["h_batch"][0].B)
    if s["kind"] in ("attn", "turn"):
        s["longest"] = max(_spread(s["B"], s["lo"], s["hi"])) + (s["n_hi"] if s["kind"] == "turn" else 0)
        nbytes = max(nbytes, dsla.dsla_attention_paged_workspace_bytes(s["h_cache"], s["h_batch"][0], s["H"], s["longest"]))
    s["ws"] = torch.empty(nbytes, dtype=torch.uint8, device="cuda")
    if s["kind"] in ("rope", "turn"):
        s["h_rope"] = dsla.make_rope(s["H"], s["Hkv"], s["d"], io_dtype=io, inv_freq=s["freq"], interleaved=s.get("pairs") == "neighbours",
                                     q_weight=s["weights"][0], k_weight=s["weights"][1], eps=EPS, offsets=s.get("depth"))


# ---------------------------------------------------------------------------------------------------------------
# the plain forms
def _entries(batch):
    """Entry of every token and its place in it."""
    m = torch.arange(batch["total"], device="cuda")
    if batch["cu"] is None:
        return m, torch.zeros_like(m)
    e = torch.searchsorted(batch["cu"][1:].long(), m, right=True)
    return e, m - batch["cu"].long()[e]


def _rotated(x, weight, position, freq, pairs, norm):
    y = x.float()
    if norm:
        y = y * torch.rsqrt((y * y).mean(-1, keepdim=True) + EPS) * weight
    angle = position.double()[:, None] * freq.double()
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
    rot = 2 * freq.numel()
    a, b = (y[..., :rot // 2], y[..., rot // 2:rot]) if pairs == "halves" else (y[..., 0:rot:2], y[..., 1:rot:2])
    u, w = a * cos - b * sin, a * sin + b * cos
    turned = torch.cat([u, w], -1) if pairs == "halves" else torch.stack([u, w], -1).flatten(-2)
    return torch.cat([turned, y[..., rot:]], -1).to(x.dtype)


def _plain_rope(s):
    c, batch = s["cache"], s["batch"]
    e, j = _entries(batch)
    at = batch["start"].long()[e]
    position = at + (s["depth"].long() if "depth" in s else j)
    pairs, norm = s.get("pairs", "halves"), s["weights"][0] is not None
    s["q_out"].copy_(_rotated(s["q"], s["weights"][0], position, s["freq"], pairs, norm))
    where = at + j
    pages = c["table"][batch["rows"].long()[e], where // s["page"]].long()
    c["pools"][0][pages, :, where % s["page"]] = _rotated(s["k"], s["weights"][1], position, s["freq"], pairs, norm)
    c["pools"][1][pages, :, where % s["page"]] = s["v"]


def _plain_attention(s, q):
    c, batch, d, G = s["cache"], s["batch"], s["d"], s["H"] // s["Hkv"]
    B, n = batch["start"].numel(), batch["longest"]
    cu = torch.arange(B + 1, device="cuda") if batch["cu"] is None else batch["cu"].long()
    start, count = batch["start"].long(), cu[1:] - cu[:-1]
    table = c["table"][batch["rows"].long()].long()
    L = table.shape[1] * s["page"]
    keys, values = (p[table.clamp_min(0)].permute(0, 2, 1, 3, 4).reshape(B, s["Hkv"], L, d).float() for p in c["pools"])
    i, j = torch.arange(L, device="cuda"), torch.arange(n, device="cuda")
    token = (cu[:-1, None] + j).clamp_max(batch["total"] - 1)                                    # [B][n]
    drafted = i[None] - start[:, None]                                                           # [B][L]
    if s["mask"] is None:
        seen = drafted[:, None] <= j[None, :, None]
    else:
        bit = s["mask"][token][:, :, None] >> drafted.clamp(0, 63)[:, None] & 1
        seen = (drafted < 0)[:, None] | ((bit == 1) & (drafted < count[:, None])[:, None])
    values = torch.where((drafted < count[:, None])[:, None, :, None], values, 0.0)
    x = q[token].float().reshape(B, n, s["Hkv"], G, d).permute(0, 2, 3, 1, 4).reshape(B, s["Hkv"], G * n, d)
    score = (torch.matmul(x, keys.transpose(-1, -2).contiguous()) * d ** -0.5).reshape(B, s["Hkv"], G, n, L)
    score = torch.where(seen[:, None, None], score, -math.inf)
    top = score.amax(-1, keepdim=True)
    p = torch.exp(score - torch.where(top == -math.inf, 0.0, top))
    out = torch.matmul(p.reshape(B, s["Hkv"], G * n, L), values).reshape(B, s["Hkv"], G, n, d)
    z = p.sum(-1)[..., None]
    out = torch.where(z > 0, out / z, 0.0).permute(0, 3, 1, 2, 4).reshape(B, n, s["H"], d)
    e, j = _entries(batch)
    s["o"].copy_(out[e, j])


def _plain_truncate(s, keep):
    c, page = s["cache"], s["page"]
    left = torch.where(keep < 0, c["lens"], torch.minimum(c["lens"], keep))
    col = torch.arange(c["table"].shape[1], device="cuda")
    drop = (col >= ((left + page - 1) // page)[:, None]) & (col < ((c["lens"] + page - 1) // page)[:, None])
    c["refs"].scatter_add_(0, c["table"].clamp_min(0).long().flatten(), -drop.int().flatten())
    c["table"].masked_fill_(drop, -1)
    c["lens"].copy_(left)


def _plain_extend(s, batch):
    c, page, rows = s["cache"], s["page"], batch["rows"].long()
    count = torch.ones_like(rows) if batch["cu"] is None else (batch["cu"][1:] - batch["cu"][:-1]).long()
    start = c["lens"][rows].long()
    have, want = (start + page - 1) // page, (start + count + page - 1) // page
    last = c["table"][rows, (have - 1).clamp_min(0)].clamp_min(0).long()
    shared = (start % page > 0) & (c["refs"][last] > 1) & (count > 0)   # a shared page that is not full is copied
    first = have - shared.long()
    need = want - first
    before = need.cumsum(0) - need
    free = torch.argsort(c["refs"] != 0, stable=True)                    # free pages first, in ascending order
    col = torch.arange(c["table"].shape[1], device="cuda")
    new = (col >= first[:, None]) & (col < want[:, None])
    pages = free[(before[:, None] + col - first[:, None]).clamp(0, free.numel() - 1)]
    c["table"][rows] = torch.where(new, pages.int(), c["table"][rows])
    c["refs"].scatter_add_(0, pages.flatten(), new.int().flatten())
    c["refs"].scatter_add_(0, last, -shared.int())
    c["lens"][rows] = (start + count).int()
    batch["start"].copy_(start)
    copied = shared.nonzero()[:, 0]
    if copied.numel():
        fresh, kept = pages[copied, first[copied]], torch.arange(page, device="cuda") < (start[copied] % page)[:, None]
        c["pools"][:, fresh] = torch.where(kept[None, :, None, :, None], c["pools"][:, last[copied]], c["pools"][:, fresh])


def _plain_fork(s):
    c, parent = s["cache"], s["parent"].long()
    new = (parent >= 0)[:, None]
    c["table"].copy_(torch.where(new, c["table"][parent.clamp_min(0)], c["table"]))
    c["lens"].copy_(torch.where(new[:, 0], c["lens"][parent.clamp_min(0)], c["lens"]))
    c["refs"].scatter_add_(0, c["table"].clamp_min(0).long().flatten(), (new & (c["table"] >= 0)).int().flatten())


def _plain_compact(s):
    c = s["cache"]
    live, index = c["refs"] > 0, torch.arange(c["n_pages"], device="cuda")
    n = live.sum()
    src, dst = (live & (index >= n)).nonzero()[:, 0], (~live & (index < n)).nonzero()[:, 0]
    index[src] = dst
    c["pools"][:, dst] = c["pools"][:, src]
    c["refs"][dst] = c["refs"][src]
    c["refs"][src] = 0
    c["table"].copy_(torch.where(c["table"] >= 0, index[c["table"].clamp_min(0).long()].int(), -1))
    s["live"].copy_(n)


def _plain_accept(s):
    c, batch, page = s["cache"], s["batch"], s["page"]
    e, j = _entries(batch)
    moved = (j < s["accepted"].long()[e]).nonzero()[:, 0]
    e, j = e[moved], j[moved]
    at = batch["start"].long()[e]
    src, dst = at + s["path"].long()[moved], at + j
    row = batch["rows"].long()[e]
    rows = c["pools"][:, c["table"][row, src // page].long(), :, src % page]
    c["pools"][:, c["table"][row, dst // page].long(), :, dst % page] = rows
    keep = torch.full_like(c["lens"], -1)
    keep[batch["rows"].long()] = batch["start"] + s["accepted"]
    _plain_truncate(s, keep)


def _plain(s):
    kind = s["kind"]
    if kind == "rope":
        _plain_rope(s)
    elif kind == "attn":
        _plain_attention(s, s["q"])
    elif kind == "turn":
        _plain_truncate(s, s["keep"])
        _plain_extend(s, s["batch"])
        _plain_rope(s)
        _plain_attention(s, s["q_out"])
        _plain_accept(s)
    elif kind == "step":
        _plain_truncate(s, s["keep"])
        _plain_extend(s, s["batch"])
    elif kind == "fork":
        _plain_truncate(s, s["keep"])
        _plain_fork(s)
        _plain_extend(s, s["batch"])
    else:
        _plain_truncate(s, s["keep"][0])
        _plain_compact(s)
        _plain_extend(s, s["batch"][0])
        _plain_truncate(s, s["keep"][1])
        _plain_compact(s)
        _plain_extend(s, s["batch"][1])


def _own(s):
    import paper_2506_09316_amd as dsla
    kind, cache, batch, pools, ws = s["kind"], s["h_cache"], s["h_batch"], s["h_pools"], s["ws"]
    k_pages, v_pages = s["cache"]["pools"][0], s["cache"]["pools"][1]
    if kind == "rope":
        dsla.dsla_qk_rope(s["h_rope"], s["q"], s["k"], s["v"], s["q_out"], None, cache, batch[0], k_pages, v_pages)
    elif kind == "attn":
        dsla.dsla_attention_paged(cache, batch[0], s["q"], k_pages, v_pages, s["o"], s["d"] ** -0.5, s["longest"], tree=s["mask"], workspace=ws)
    elif kind == "turn":
        dsla.dsla_cache_truncate(cache, s["keep"])
        dsla.dsla_cache_extend(cache, batch[0], pools, ws)
        dsla.dsla_qk_rope(s["h_rope"], s["q"], s["k"], s["v"], s["q_out"], None, cache, batch[0], k_pages, v_pages)
        dsla.dsla_attention_paged(cache, batch[0], s["q_out"], k_pages, v_pages, s["o"], s["d"] ** -0.5, s["longest"], tree=s["mask"], workspace=ws)
        dsla.dsla_cache_accept(cache, batch[0], s["path"], s["accepted"], pools, ws)
    elif kind == "step":
        dsla.dsla_cache_truncate(cache, s["keep"])
        dsla.dsla_cache_extend(cache, batch[0], pools, ws)
    elif kind == "fork":
        dsla.dsla_cache_truncate(cache, s["keep"])
        dsla.dsla_cache_fork(cache, s["parent"])
        dsla.dsla_cache_extend(cache, batch[0], pools, ws)
    else:
        for i in range(2):
            dsla.dsla_cache_truncate(cache, s["keep"][i])
            dsla.dsla_cache_compact(cache, s["live"], pools, ws)
            dsla.dsla_cache_extend(cache, batch[i], pools, ws)


def run(s):
    if own:
        _own(s)
    else:
        _plain(s)
    c, kind = s["cache"], s["kind"]
    if kind == "rope":
        return {"q": s["q_out"], "k_pages": c["pools"][0], "v_pages": c["pools"][1]}
    if kind == "attn":
        return {"o": s["o"]}
    out = {"table": c["table"], "lens": c["lens"], "refs": c["refs"]}
    if kind == "turn":
        return dict(out, start=s["batch"]["start"], q=s["q_out"], o=s["o"], k_pages=c["pools"][0], v_pages=c["pools"][1])
    if kind == "step":
        return dict(out, start=s["batch"]["start"])
    if kind == "fork":
        return dict(out, start=s["batch"]["start"], pools=c["pools"])
    return dict(out, start=[x["start"] for x in s["batch"]], live=s["live"], pools=c["pools"])


def work(case):
    """Every input read once and every output written once; what a call leaves alone is neither."""
    c, e, B = case, _size(case["io"]), case["B"]
    kind, row = c["kind"], case["Hkv"] * case["d"] * _size(case["io"])
    if kind == "rope":
        tokens = sum(_spread(B, c["lo"], c["hi"]))
        return {"bytes": tokens * (2 * c["H"] * c["d"] * e + 4 * row), "flops": tokens * (c["H"] + c["Hkv"]) * (3 * c["rot"] + 4 * c["d"] * c["norm"])}
    if kind in ("attn", "turn"):
        counts, held = _counts(c), _spread(B, c["lo"], c["hi"])
        if kind == "turn":
            held = [x + n for x, n in zip(held, counts)]
        w = {"bytes": 2 * sum(held) * row + 2 * sum(counts) * c["H"] * c["d"] * e,
             "flops": sum(4 * n * c["H"] * c["d"] * (x - n) + 2 * n * (n + 1) * c["H"] * c["d"] for x, n in zip(held, counts))}
        if kind == "turn":   # and the rotation: q once more, keys and values in and out
            w["bytes"] += sum(counts) * (2 * c["H"] * c["d"] * e + 4 * row)
            w["flops"] += sum(counts) * (c["H"] + c["Hkv"]) * 7 * c["d"]
        return w
    if kind == "step":
        # lengths, starts and counts of the entries, and the table entries, references and lengths that change, twice
        pages = sum(-(-(x + n) // c["page"]) - -(-x // c["page"]) for x, n in zip(_spread(B, c["lo"], c["hi"]), _counts(c)))
        return {"bytes": 28 * B + 24 * pages, "flops": 0}
    if kind == "fork":
        held = _spread(B, c["lo"], c["hi"])
        return {"bytes": c["ways"] * sum(2 * (x % c["page"]) * row * c["pools"] + 16 * -(-x // c["page"]) for x in held), "flops": 0}
    pages = sum(-(-x // c["page"]) for x in _spread(B // 2, c["lo"], c["hi"]))
    return {"bytes": 2 * pages * (2 * c["page"] * row * c["pools"] + 32), "flops": 0}


# ---------------------------------------------------------------------------------------------------------------
def exact(case, seed):
    """The same from the definitions in 64 bits, entry by entry; whole numbers and moved pages have no such value."""
    kind = case["kind"]
    if kind not in ("rope", "attn", "turn"):
        return None
    s = prepare(case, seed)
    c, batch, page = s["cache"], s["batch"], s["page"]
    B, rows = case["B"], batch["rows"].tolist()
    cu = list(range(B + 1)) if batch["cu"] is None else batch["cu"].tolist()
    starts, table = batch["start"].tolist(), c["table"].cpu().numpy()
    k_pages, v_pages = c["pools"][0].double(), c["pools"][1].double()
    if kind != "attn":
        def turned(x, weight, depth, at):
            y = x.double()
            if weight is not None:
                y = y / (y.square().mean(-1, keepdim=True) + EPS).sqrt() * weight.double()
            angle = torch.tensor([at + p for p in depth], dtype=torch.float64, device="cuda")[:, None, None] * s["freq"].double()
            n, out = s["freq"].numel(), y.clone()
            first, second = (slice(0, n), slice(n, 2 * n)) if s.get("pairs", "halves") == "halves" else (slice(0, 2 * n, 2), slice(1, 2 * n, 2))
            out[..., first] = y[..., first] * angle.cos() - y[..., second] * angle.sin()
            out[..., second] = y[..., first] * angle.sin() + y[..., second] * angle.cos()
            return out

        depth = s["depth"].tolist() if "depth" in s else None
        q = torch.empty(s["q"].shape, dtype=torch.float64, device="cuda")
        new = []
        for b in range(B):
            t = slice(cu[b], cu[b + 1])
            way = depth[t] if depth else range(cu[b + 1] - cu[b])
            q[t] = turned(s["q"][t], s["weights"][0], way, starts[b])
            new.append((turned(s["k"][t], s["weights"][1], way, starts[b]), s["v"][t].double()))
            if kind == "rope":
                for i in range(cu[b + 1] - cu[b]) if cu[b + 1] - cu[b] < 4 else ():
                    w = starts[b] + i
                    k_pages[int(table[rows[b], w // page]), :, w % page], v_pages[int(table[rows[b], w // page]), :, w % page] = new[b][0][i], new[b][1][i]
                if cu[b + 1] - cu[b] >= 4:
                    w = np.arange(starts[b], starts[b] + cu[b + 1] - cu[b])
                    at, off = _gpu(table[rows[b]][w // page], np.int64), _gpu(w % page, np.int64)
                    k_pages[at, :, off], v_pages[at, :, off] = new[b]
        if kind == "rope":
            return {"q": q, "k_pages": k_pages, "v_pages": v_pages}
    o = torch.zeros(s["o"].shape, dtype=torch.float64, device="cuda")
    G = case["H"] // case["Hkv"]
    for b in range(B):
        t, at = slice(cu[b], cu[b + 1]), starts[b]
        n = cu[b + 1] - cu[b]
        total = at + n
        at_pages = [int(x) for x in table[rows[b]][:-(-(at if kind == "turn" else total) // page)]]
        keys, values = (p[at_pages].transpose(1, 2).reshape(-1, case["Hkv"], case["d"])[:at if kind == "turn" else total] for p in (k_pages, v_pages))
        # (queries that are rounded before the attention reads them have the values they were rounded to)
        x = s["q"][t].double() if kind == "attn" else q[t].to(s["q"].dtype).double()
        if kind == "turn":
            keys, values = torch.cat([keys, new[b][0].to(s["k"].dtype).double()]), torch.cat([values, new[b][1]])
        seen = torch.ones(n, total, dtype=torch.bool, device="cuda")
        if s["mask"] is None:
            seen[:, at:] = torch.ones(n, n, device="cuda").tril() > 0
        else:
            bits = np.array([[m >> i & 1 for i in range(n)] for m in s["mask"][t].tolist()], dtype=bool)
            seen[:, at:] = torch.from_numpy(bits).cuda()
        for h in range(case["Hkv"]):
            score = torch.einsum("ngd,ld->ngl", x[:, h * G:(h + 1) * G], keys[:, h]) * case["d"] ** -0.5
            weight = torch.softmax(score.masked_fill(~seen[:, None], -math.inf), -1)
            o[t, h * G:(h + 1) * G] = torch.einsum("ngl,ld->ngd", weight, values[:, h])
    if kind == "attn":
        return {"o": o}
    return {"table": None, "lens": None, "refs": None, "start": None, "q": q, "o": o, "k_pages": None, "v_pages": None}
