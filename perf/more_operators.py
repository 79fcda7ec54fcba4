"""Operators of the drafter's cache: what a draft model's block does between its
projections, over a paged key-value cache.

New queries and keys are rotated by positions of one axis or several
(``rotary_axes``; with ``inverse`` it is its own gradient), keys and values are
stored in pages (``cache_append``, which rotates on the way), the rows of one
new token or of a draft tree attend to them (``paged_attention``), the accepted
nodes of a tree are kept (``cache_keep``), and sequences are forked, cut and
dropped by their pages (``cache_fork``).

``run`` computes each of them with elementary torch operations in 32 bits, or
(``own``) through the framework's binding.  Head counts follow the widths of
this repository's workloads in heads of 128 (3584: 28 heads over 4 of keys;
4096: 32; 5120: 40), trees are of up to 64 draft states, memories of 256 to
8192 visual entries; drawn cases spread around them.
"""

import math
import random

import torch

own = False

E4M3_MAX = 448.0


def _rotary(name, dtype, tokens, heads, kv_heads, **more):
    # rot: rotated dims of a head; axes: pairs of each axis' share are even;
    # adjacent: pairs (2j, 2j + 1), else (j, j + rot / 2); fused: q and k are
    # views of one projection's output; far: the first position
    return dict(dict(name=name, kind="rotary", dtype=dtype, tokens=tokens, heads=heads, kv_heads=kv_heads, dim=128,
                     rot=128, axes=1, adjacent=False, inverse=False, fused=True, far=0), **more)


def _append(name, cache, batch, new, heads, kv_heads, **more):
    # new: tokens per sequence (ragged: down to none, the batch padded);
    # start: entries that the sequences hold already, at most; cache: type of the
    # pages; rotate: q and k are rotated on the way, else k is stored as it is
    return dict(dict(name=name, kind="append", cache=cache, batch=batch, new=new, heads=heads, kv_heads=kv_heads,
                     dim=128, page=64, start=64, ragged=False, rotate=True, axes=1, adjacent=False), **more)


def _attention(name, cache, batch, nodes, heads, kv_heads, longest, **more):
    # nodes: new tokens per sequence, which are the last entries; masked: a
    # draft tree's ancestors, else each sees the ones before it; ragged: lengths
    # spread from a few entries to the longest; idle: share of sequences without any
    return dict(dict(name=name, kind="attention", cache=cache, batch=batch, nodes=nodes, heads=heads,
                     kv_heads=kv_heads, dim=128, page=64, longest=longest, ragged=False, masked=False, idle=0.0), **more)


def _keep(name, cache, batch, nodes, kv_heads, **more):
    # path: accepted nodes, at most
    return dict(dict(name=name, kind="keep", cache=cache, batch=batch, nodes=nodes, kv_heads=kv_heads, dim=128,
                     page=64, path=6, longest=256), **more)


def _fork(name, cache, batch, width, kv_heads, longest, **more):
    # width: continuations of each sequence that goes on (as many in all as there were, at least `width`)
    return dict(dict(name=name, kind="fork", cache=cache, batch=batch, width=width, kv_heads=kv_heads, dim=128,
                     page=64, longest=longest, room=64), **more)


def listed():
    return [
        # Prompts of images: time, height and width.
        _rotary("rotary-image-prompts", "bf16", 8 * 2880, 28, 4, axes=3, far=1000),
        # The gradient of a training batch of images, two axes in adjacent pairs.
        _rotary("rotary-training-gradient", "fp32", 16 * 576, 40, 40, axes=2, adjacent=True, inverse=True, fused=False),
        # One new token of each sequence stored, its query rotated on the way.
        _append("append-step", "bf16", 32, 1, 28, 4, page=16, axes=3, start=1024),
        # Prompts of uneven length stored in 8 bits.
        _append("append-prompts", "e4m3", 4, 8192, 32, 8, ragged=True),
        # One sequence decodes behind an image: latency.
        _attention("attention-one-state", "bf16", 1, 1, 32, 32, 576 + 64),
        # A served batch of uneven lengths, small pages, a few idle sequences.
        _attention("attention-batch", "bf16", 64, 1, 28, 4, 8192, page=16, ragged=True, idle=0.05),
        # Long caches in 8 bits.
        _attention("attention-long", "e4m3", 4, 1, 32, 8, 131072, page=128),
        # The draft trees of a batch, each node with its ancestors.
        _attention("attention-trees", "bf16", 8, 32, 28, 4, 2880 + 32, ragged=True, masked=True),
        # A draft tree stored and its accepted path kept, one sequence.
        _keep("keep-one-tree", "fp32", 1, 64, 32),
        # The same for a batch.
        _keep("keep-trees", "bf16", 16, 64, 40, page=16),
        # One sequence goes on as six: its last page is copied five times.
        _fork("fork-one", "bf16", 1, 6, 32, 700, page=16),
        # A batch's sequences replaced by the continuations of the best quarter.
        _fork("fork-batch", "bf16", 128, 4, 4, 8192),
    ]


def draw(rng):
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    heads, kv = rng.choice([(32, 32), (28, 4), (40, 40), (32, 8), (16, 2), (6, 2), (12, 1), (5, 5)])
    dim, page = rng.choice([64, 128, 128, 128, 256]), rng.choice([16, 32, 48, 64, 128])
    cache = rng.choice(["bf16", "bf16", "e4m3", "fp32"])
    size = {"bf16": 2, "e4m3": 1, "fp32": 4}[cache]
    kind = rng.choice(["rotary", "append", "attention", "attention", "attention", "keep", "fork"])
    if kind == "rotary":
        dtype = rng.choice(["bf16", "bf16", "fp32"])
        most = (8 * 2880 * 32 * 128) // ((heads + kv) * dim)
        return dict(kind=kind, dtype=dtype, tokens=log_int(1, most), heads=heads, kv_heads=kv, dim=dim,
                    rot=rng.choice([dim, dim, dim // 2, dim - 16]), axes=rng.choice([1, 2, 3, 4]),
                    adjacent=rng.random() < 0.4, inverse=rng.random() < 0.4, fused=rng.random() < 0.6,
                    far=rng.choice([0, log_int(10, 10_000_000)]))
    if kind == "append":
        batch, rotate = log_int(1, 64), rng.random() < 0.7
        most = max(1, 32768 * 48 * 128 // (batch * (heads + 2 * kv) * dim * size))
        return dict(kind=kind, cache=cache, batch=batch, new=log_int(1, min(8192, most)), heads=heads, kv_heads=kv,
                    dim=dim, page=page, start=log_int(1, 1024), ragged=rng.random() < 0.5, rotate=rotate,
                    axes=rng.choice([1, 3]), adjacent=rng.random() < 0.3)
    if kind == "attention":
        batch, nodes = log_int(1, 64), rng.choice([1, 1, 1, 2, 7, log_int(1, 64)])
        # entries: by the cache's bytes, and by the products of many rows
        most = min(400_000_000 // (batch * kv * dim * size * 2), 10_000_000_000 // (batch * heads * nodes * dim * 4))
        longest = nodes + log_int(1, max(2, min(131072, most)))
        return dict(kind=kind, cache=cache, batch=batch, nodes=nodes, heads=heads, kv_heads=kv, dim=dim, page=page,
                    longest=longest, ragged=rng.random() < 0.5, masked=nodes > 1 and rng.random() < 0.7,
                    idle=rng.choice([0.0, 0.0, 0.2]))
    if kind == "keep":
        nodes = rng.choice([7, 16, 64, log_int(2, 64)])
        return dict(kind=kind, cache=cache, batch=log_int(1, 64), nodes=nodes, kv_heads=kv, dim=dim, page=page,
                    path=rng.choice([1, 6, min(nodes, 10)]), longest=log_int(nodes, 512))
    batch = log_int(1, 128)
    most = max(2, 400_000_000 // (batch * kv * dim * size * 2))
    return dict(kind=kind, cache=cache, batch=batch, width=rng.choice([1, 2, 4, 6]), kv_heads=kv, dim=dim, page=page,
                longest=log_int(1, min(8192, most)), room=rng.choice([0, 1, 64]))


# ---------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------

def _dtype(name):
    return {"bf16": torch.bfloat16, "fp32": torch.float32, "e4m3": torch.float8_e4m3fn}[name]


def _rows_type(case):
    """Type of queries, new keys and values beside a cache of this type."""
    return torch.float32 if case["cache"] == "fp32" else torch.bfloat16


def _ceil(n, m):
    return -(-n // m)


def _lengths(case, lowest):
    """The sequences' lengths in descending order: from the longest to a few
    entries by equal factors (ragged), or within a quarter of the longest."""
    n, top = case["batch"], case["longest"]
    low = lowest if case.get("ragged", True) else max(lowest, top - top // 4)
    lens = [max(low, int(round(top * (low / top) ** (i / max(1, n - 1))))) for i in range(n)]
    idle = int(n * case.get("idle", 0.0))
    return lens[:n - idle] + [0] * idle


def _frequencies(rot, axes, base=1e6):
    """Radians per position of each pair of dims in 64 bits, and each pair's axis: equal shares in blocks."""
    j = torch.arange(rot // 2, dtype=torch.float64)
    return (base ** (-2.0 * j / rot)).cuda(), (j.long() * axes // (rot // 2)).to(torch.int32).cuda()


def _positions(axes, tokens, far):
    """Time, and coordinates on a grid of 24 columns behind it."""
    n = torch.arange(tokens, dtype=torch.int32, device="cuda")
    rows = [far + n // 576, far + n % 576 // 24, far + n % 24, far + n % 7]
    return torch.stack([far + n] if axes == 1 else rows[:axes])


def _tables(counts, width, spare, g):
    """Pages for so many of each sequence, in random order, -1 behind; and the number of pages, some of them spare."""
    total = sum(counts)
    n_pages = total + total // 8 + spare
    order = torch.randperm(n_pages, generator=g, device="cuda").to(torch.int32)
    table = torch.full((len(counts), width), -1, dtype=torch.int32, device="cuda")
    at = 0
    for b, c in enumerate(counts):
        table[b, :c] = order[at:at + c]
        at += c
    return table, n_pages


def _pages(case, n_pages, g):
    """A pool of normal entries; in 8 bits they stand for about that."""
    shape = (n_pages, case["kv_heads"], case["page"], case["dim"])
    pool = torch.empty(shape, dtype=_dtype(case["cache"]), device="cuda")
    step = max(1, (1 << 27) // (shape[1] * shape[2] * shape[3]))
    for p in range(0, n_pages, step):
        x = torch.randn((min(step, n_pages - p),) + shape[1:], generator=g, device="cuda")
        pool[p:p + step] = (64.0 * x if case["cache"] == "e4m3" else x).to(pool.dtype)
    return pool


def _scales(case, g):
    if case["cache"] != "e4m3":
        return None, None
    s = (1.0 + 0.2 * torch.rand((2, case["kv_heads"]), generator=g, device="cuda")) / 64.0
    return s[0], s[1]


def _tree_bits(batch, nodes, g):
    """Ancestors (and itself) of each node of random trees, the root first, as words of 32 bits."""
    seen = torch.zeros((batch, nodes, _ceil(nodes, 32) * 32), dtype=torch.bool, device="cuda")
    rows = torch.arange(batch, device="cuda")
    for j in range(nodes):
        if j:
            parent = torch.randint(0, max(1, (j + 1) // 2), (batch,), generator=g, device="cuda")
            seen[:, j] = seen[rows, parent]
        seen[:, j, j] = True
    words = (seen.view(batch, nodes, -1, 32).long() << torch.arange(32, device="cuda")).sum(-1)
    return torch.where(words >= 1 << 31, words - (1 << 32), words).to(torch.int32)


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    pick = random.Random(int(seed))

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda")

    def whole(values):
        return torch.tensor(values, dtype=torch.int32, device="cuda")

    kind, s = case["kind"], dict(case=case)
    dim, kv = case["dim"], case["kv_heads"]
    if kind == "rotary":
        n, h, dt = case["tokens"], case["heads"], _dtype(case["dtype"])
        if case["fused"]:
            x = normal(n, h + 2 * kv, dim).to(dt)
            s["q"], s["k"] = x[:, :h], x[:, h:h + kv]
        else:
            s["q"], s["k"] = normal(n, h, dim).to(dt), normal(n, kv, dim).to(dt)
        s["frequencies"], s["axis"] = _frequencies(case["rot"], case["axes"])
        s["positions"] = _positions(case["axes"], n, case["far"] + pick.randrange(1000))
        return s
    s["k_scale"], s["v_scale"] = _scales(case, g)
    dt, page = _rows_type(case), case["page"]
    if kind == "append":
        batch, new, h = case["batch"], case["new"], case["heads"]
        counts = [new - (new * b // batch if case["ragged"] else 0) for b in range(batch)]
        starts = [case["start"] - case["start"] * b // batch for b in range(batch)]
        pick.shuffle(starts)
        pages = [_ceil(c + t, page) for c, t in zip(counts, starts)]
        s["table"], n_pages = _tables(pages, max(pages) + 1, 2, g)
        n = batch * new
        x = normal(n, h + 2 * kv, dim).to(dt)
        s["q"], s["k"], s["v"] = x[:, :h], x[:, h:h + kv], x[:, h + kv:]
        j = torch.arange(new, dtype=torch.int32, device="cuda")[None]
        rows = torch.arange(batch, dtype=torch.int32, device="cuda")[:, None]
        # rows of the padded batch that hold no token belong to no sequence
        s["sequence"] = torch.where(j < whole(counts)[:, None], rows, -1).reshape(n)
        s["entry"] = (whole(starts)[:, None] + j).reshape(n).contiguous()
        s["frequencies"], s["axis"] = _frequencies(dim, case["axes"])
        s["positions"] = _positions(case["axes"], n, pick.randrange(1000))
    elif kind == "attention":
        lens = _lengths(case, case["nodes"])
        pick.shuffle(lens)
        pages = [_ceil(c, page) for c in lens]
        s["table"], n_pages = _tables(pages, max(pages), 2, g)
        s["lens"] = whole(lens)
        s["q"] = (2.0 * normal(case["batch"] * case["nodes"], case["heads"], dim)).to(dt)
        s["tree"] = _tree_bits(case["batch"], case["nodes"], g) if case["masked"] else None
    elif kind == "keep":
        batch, nodes = case["batch"], case["nodes"]
        lens = _lengths(case, nodes)
        pick.shuffle(lens)
        pages = [_ceil(c, page) for c in lens]
        s["table"], n_pages = _tables(pages, max(pages), 2, g)
        s["lens"] = whole(lens)
        n = batch * nodes
        s["k"], s["v"] = normal(n, kv, dim).to(dt), normal(n, kv, dim).to(dt)
        s["sequence"] = torch.arange(batch, dtype=torch.int32, device="cuda").repeat_interleave(nodes)
        j = torch.arange(nodes, dtype=torch.int32, device="cuda")[None]
        s["entry"] = (s["lens"][:, None] - nodes + j).reshape(n).contiguous()
        most = min(case["path"], nodes)
        paths = [[0] + sorted(pick.sample(range(1, nodes), pick.randint(0, most - 1))) for _ in range(batch)]
        s["nodes"] = whole([p + [-1] * (most - len(p)) for p in paths])
    else:
        batch = case["batch"]
        lens = _lengths(case, 1)
        pick.shuffle(lens)
        pages = [_ceil(c, page) for c in lens]
        c, grown = max(batch, case["width"]), _ceil(case["room"], page)
        # enough pages for a copy of a last page and the room of each
        s["table"], n_pages = _tables(pages, max(pages) + grown, c * (1 + grown), g)
        s["lens"] = whole(lens)
        alive = pick.sample(range(batch), _ceil(c, case["width"]))
        parents = [alive[i // case["width"]] for i in range(c)]
        parents = [p if pick.random() < 0.97 or c < 8 else -1 for p in parents]
        s["parents"] = whole(parents)
        s["keep"] = whole([max(0, lens[p] - (pick.randrange(8) if pick.random() < 0.1 else 0)) if p >= 0 else 0
                           for p in parents])
        s["room"] = whole([case["room"] if p >= 0 else 0 for p in parents])
    s["k_pages"], s["v_pages"] = _pages(case, n_pages, g), _pages(case, n_pages, g)
    return s


# ---------------------------------------------------------------------------
# Plain forms: elementary operations in 32 bits (angles in 64)
# ---------------------------------------------------------------------------

def _plain_rotate(x, positions, frequencies, axis, adjacent, inverse):
    """x [N, heads, D] in 32 bits, its first dims rotated."""
    x = x.float()
    r = 2 * frequencies.numel()
    angle = positions[axis.long()].T.double() * frequencies
    cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
    if inverse:
        sin = -sin
    a, b = (x[..., 0:r:2], x[..., 1:r:2]) if adjacent else (x[..., :r // 2], x[..., r // 2:r])
    c, d = a * cos - b * sin, a * sin + b * cos
    turned = torch.stack((c, d), -1).flatten(-2) if adjacent else torch.cat((c, d), -1)
    return torch.cat((turned, x[..., r:]), -1)


def _stored(x, scale, dtype):
    """Entries in the cache's type."""
    x = x.float()
    if scale is not None:
        x = (x / scale[:, None]).clamp(-E4M3_MAX, E4M3_MAX)
    return x.to(dtype)


def _bytes(pool):
    """8-bit floats are indexed as bytes."""
    return pool.view(torch.uint8) if pool.dtype == torch.float8_e4m3fn else pool


def _plain_store(pool, x, table, sequence, entry):
    page = pool.shape[2]
    at = torch.nonzero(sequence >= 0)[:, 0]
    e = entry[at].long()
    p = table[sequence[at].long(), e // page].long()
    _bytes(pool)[p, :, e % page] = _bytes(x)[at]


def _plain_append(s, q, rotate, adjacent=False):
    k = s["k"]
    if rotate:
        k = _plain_rotate(k, s["positions"], s["frequencies"], s["axis"], adjacent, False)
        q = _plain_rotate(q, s["positions"], s["frequencies"], s["axis"], adjacent, False).to(q.dtype)
    dtype = s["k_pages"].dtype
    _plain_store(s["k_pages"], _stored(k, s["k_scale"], dtype), s["table"], s["sequence"], s["entry"])
    _plain_store(s["v_pages"], _stored(s["v"], s["v_scale"], dtype), s["table"], s["sequence"], s["entry"])
    return q


def _gathered(pool, table):
    """[B, kv_heads, width * page, D] in 32 bits."""
    x = _bytes(pool)[table.long().clamp(min=0)].view(pool.dtype).float()
    return x.transpose(1, 2).flatten(2, 3)


def _plain_attention(s):
    case, q, lens = s["case"], s["q"], s["lens"].long()
    batch, nodes, kv = case["batch"], case["nodes"], case["kv_heads"]
    group = case["heads"] // kv
    scale = case["dim"] ** -0.5
    q = q.float().view(batch, nodes, kv, group, -1).permute(0, 2, 1, 3, 4).flatten(2, 3)
    k = _gathered(s["k_pages"], s["table"])
    z = q @ k.transpose(2, 3) * scale
    del k
    if s["k_scale"] is not None:
        z = z * s["k_scale"][:, None, None]
    at = torch.arange(z.shape[3], device=z.device)
    node = at - (lens[:, None] - nodes)                         # which of the new ones, negative: before them
    if s["tree"] is None:
        seen = node[:, None] <= torch.arange(nodes, device=z.device)[:, None]
    else:
        j = node.clamp(0, nodes - 1)
        word = s["tree"].gather(2, (j // 32)[:, None].expand(-1, nodes, -1))
        seen = (node < 0)[:, None] | ((word >> (j % 32)[:, None]) & 1 != 0)
    seen = seen & (at < lens[:, None])[:, None]
    z = z.view(batch, kv, nodes, group, -1).masked_fill(~seen[:, None, :, None], -math.inf)
    m = z.amax(-1, keepdim=True)
    m = torch.where(m == -math.inf, 0.0, m)
    e = torch.exp(z - m)
    total = e.sum(-1, keepdim=True)
    lse = m + torch.log(total)
    e = e / torch.where(total > 0, total, 1.0)
    out = e.flatten(2, 3) @ _gathered(s["v_pages"], s["table"])
    if s["v_scale"] is not None:
        out = out * s["v_scale"][:, None, None]
    out = out.view(batch, kv, nodes, group, -1).permute(0, 2, 1, 3, 4)
    lse = lse[..., 0].permute(0, 2, 1, 3)
    return dict(out=out.reshape(s["q"].shape).to(s["q"].dtype), lse=lse.reshape(batch * nodes, -1))


def _plain_keep(s):
    table, lens, nodes, page = s["table"], s["lens"].long(), s["nodes"].long(), s["case"]["page"]
    count = (nodes >= 0).sum(1)
    b, i = torch.nonzero(nodes >= 0, as_tuple=True)
    base = lens[b] - s["case"]["nodes"]
    src, dst = base + nodes[b, i], base + i
    for pool in (_bytes(s["k_pages"]), _bytes(s["v_pages"])):
        pool[table[b, dst // page].long(), :, dst % page] = pool[table[b, src // page].long(), :, src % page]
    return (lens - s["case"]["nodes"] + count).to(torch.int32)


def _plain_fork(s):
    table, page, n_pages = s["table"], s["case"]["page"], s["k_pages"].shape[0]
    parents, width = s["parents"].long(), table.shape[1]
    held = torch.where(parents >= 0, s["lens"].long()[parents.clamp(min=0)], 0)
    n = torch.minimum(s["keep"].long(), held)
    pages = table[parents.clamp(min=0)].long()
    i = torch.arange(width, device=table.device)[None]
    child = torch.arange(n.numel(), device=table.device)
    whole, rest = n // page, n % page
    full = i < whole[:, None]
    # pages that some child holds whole, and the first child that holds each in part
    by_whole = torch.zeros(n_pages + 1, dtype=torch.bool, device=table.device)
    by_whole[torch.where(full, pages, n_pages)] = True
    last = torch.where(rest > 0, pages.gather(1, whole.clamp(max=width - 1)[:, None])[:, 0], n_pages)
    first = torch.full((n_pages + 1,), n.numel(), device=table.device).scatter_reduce(0, last, child, "amin")
    stays = (rest > 0) & ~by_whole[last] & (first[last] == child)
    held_pages = by_whole.clone()
    held_pages[last] = True
    held_pages = held_pages[:n_pages]
    order = torch.argsort(held_pages.int(), stable=True)        # free pages first, the lowest first
    have = whole + stays
    need = torch.minimum((n + s["room"].long() + page - 1) // page, torch.full_like(n, width))
    fresh = need - have
    begin = torch.cumsum(fresh, 0) - fresh
    rank = begin[:, None] + i - have[:, None]
    new = torch.where(i < have[:, None], pages, torch.where(i < need[:, None], order[rank.clamp(0, n_pages - 1)], -1))
    c = torch.nonzero((rest > 0) & ~stays)[:, 0]
    src, dst = last[c], new[c, whole[c]]
    inside = (torch.arange(page, device=table.device) < rest[c, None])[:, None, :, None]
    for pool in (_bytes(s["k_pages"]), _bytes(s["v_pages"])):
        pool[dst] = torch.where(inside, pool[src], pool[dst])
    free = n_pages - held_pages.sum() - fresh.sum()
    return dict(table=new.to(torch.int32), lens=n.to(torch.int32), free=free.to(torch.int32).view(1))


# ---------------------------------------------------------------------------
# One pass
# ---------------------------------------------------------------------------

def run(s):
    case = s["case"]
    kind = case["kind"]
    if own:
        from paper_2608_22883_gb300 import fovea
        if kind == "rotary":
            return fovea.rotary_axes(s["q"], s["k"], s["positions"], s["frequencies"], s["axis"],
                                     adjacent=case["adjacent"], inverse=case["inverse"])
        pools = (s["k_pages"], s["v_pages"])
        scales = dict(k_scale=s["k_scale"], v_scale=s["v_scale"])
        if kind == "append":
            more = dict(q=s["q"], positions=s["positions"], frequencies=s["frequencies"], axis=s["axis"],
                        adjacent=case["adjacent"]) if case["rotate"] else {}
            q = fovea.cache_append(s["k"], s["v"], *pools, s["table"], s["sequence"], s["entry"], **scales, **more)
            return dict(q=q if case["rotate"] else s["q"], k_pages=pools[0], v_pages=pools[1])
        if kind == "attention":
            return fovea.paged_attention(s["q"], *pools, s["table"], s["lens"], tree=s["tree"], want_lse=True, **scales)
        if kind == "keep":
            fovea.cache_append(s["k"], s["v"], *pools, s["table"], s["sequence"], s["entry"], **scales)
            lens = fovea.cache_keep(*pools, s["table"], s["lens"], s["nodes"], case["nodes"])
            return dict(lens=lens, k_pages=pools[0], v_pages=pools[1])
        r = fovea.cache_fork(*pools, s["table"], s["lens"], s["parents"], s["keep"], s["room"])
        return dict(r, k_pages=pools[0], v_pages=pools[1])
    if kind == "rotary":
        return tuple(_plain_rotate(x, s["positions"], s["frequencies"], s["axis"], case["adjacent"],
                                   case["inverse"]).to(x.dtype) for x in (s["q"], s["k"]))
    if kind == "attention":
        return _plain_attention(s)
    if kind == "append":
        r = dict(q=_plain_append(s, s["q"], case["rotate"], case["adjacent"]))
    elif kind == "keep":
        # a tree's entries are stored before it is verified
        _plain_append(s, None, False)
        r = dict(lens=_plain_keep(s))
    else:
        r = _plain_fork(s)
    return dict(r, k_pages=s["k_pages"], v_pages=s["v_pages"])


# ---------------------------------------------------------------------------
# The same from the definitions in 64 bits, one sequence or head at a time
# ---------------------------------------------------------------------------

def _exact_rotate(x, s, adjacent, inverse):
    y = x.double()
    half = s["frequencies"].numel()
    pair = torch.arange(half, device="cuda")
    first, second = (2 * pair, 2 * pair + 1) if adjacent else (pair, pair + half)
    turn = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"),
                       s["positions"].double()[s["axis"].long(), :].T * s["frequencies"] * (-1 if inverse else 1))
    z = torch.complex(y[..., first], y[..., second]) * turn[:, None]
    y[..., first], y[..., second] = z.real, z.imag
    return y


def _exact_stored(s, k, v):
    """Both pools in 64 bits with the new entries in their places, unrounded."""
    pools, page = [], s["case"]["page"]
    for name, x, scale in (("k_pages", k, s["k_scale"]), ("v_pages", v, s["v_scale"])):
        pool = s[name].to(torch.float32 if s["case"]["cache"] != "fp32" else torch.float64)
        x = x.double() if scale is None else x.double() / scale.double()[:, None]
        if scale is not None:
            x = x.clamp(-E4M3_MAX, E4M3_MAX)
        n_pages, kv, _, dim = pool.shape
        flat = pool.transpose(1, 2).reshape(-1, kv, dim)
        use = s["sequence"] >= 0
        entry = s["entry"][use].long()
        slot = s["table"][s["sequence"][use].long(), entry.div(page, rounding_mode="floor")].long() * page
        flat[slot + entry.remainder(page)] = x[use].to(flat.dtype)
        pools.append(flat.view(n_pages, page, kv, dim).transpose(1, 2))
    return pools


def _exact_attention(s, case):
    nodes, kv, page = case["nodes"], case["kv_heads"], case["page"]
    group = case["heads"] // kv
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.full(s["q"].shape[:2], -math.inf, dtype=torch.float64, device="cuda")
    for b, n in enumerate(s["lens"].tolist()):
        if n == 0:
            continue
        t = s["table"][b, :_ceil(n, page)].long()
        seen = torch.ones((nodes, n), dtype=torch.bool, device="cuda")
        if s["tree"] is None:
            seen[:, n - nodes:] = torch.ones((nodes, nodes), device="cuda").tril().bool()
        else:
            words = s["tree"][b].long() & 0xFFFFFFFF
            j = torch.arange(nodes, device="cuda")
            seen[:, n - nodes:] = (words[:, j // 32] >> (j % 32)) % 2 == 1
        for h in range(kv):
            k = _bytes(s["k_pages"])[t, h].view(s["k_pages"].dtype).flatten(0, 1)[:n].double()
            v = _bytes(s["v_pages"])[t, h].view(s["v_pages"].dtype).flatten(0, 1)[:n].double()
            if s["k_scale"] is not None:
                k, v = k * s["k_scale"][h].double(), v * s["v_scale"][h].double()
            rows = s["q"][b * nodes:(b + 1) * nodes, h * group:(h + 1) * group].double()
            z = (rows.flatten(0, 1) @ k.T / math.sqrt(case["dim"])).unflatten(0, (nodes, group))
            z = z.masked_fill(~seen[:, None], -math.inf)
            total = torch.logsumexp(z, 2)
            p = torch.exp(z - total.nan_to_num(neginf=0.0)[..., None])
            out[b * nodes:(b + 1) * nodes, h * group:(h + 1) * group] = p @ v
            lse[b * nodes:(b + 1) * nodes, h * group:(h + 1) * group] = total
    return dict(out=out, lse=lse)


def _exact_keep(s, case):
    pools = _exact_stored(s, s["k"], s["v"])
    lens = []
    for b, (n, path) in enumerate(zip(s["lens"].tolist(), s["nodes"].tolist())):
        path = [j for j in path if j >= 0]
        src = torch.tensor([n - case["nodes"] + j for j in path], device="cuda")
        dst = torch.arange(len(path), device="cuda") + n - case["nodes"]
        for pool in pools:
            moved = pool[s["table"][b].long()[src // case["page"]], :, src % case["page"]]
            pool[s["table"][b].long()[dst // case["page"]], :, dst % case["page"]] = moved
        lens.append(n - case["nodes"] + len(path))
    return dict(lens=torch.tensor(lens, dtype=torch.int32, device="cuda"), k_pages=pools[0], v_pages=pools[1])


def _exact_fork(s, case):
    page, n_pages = case["page"], s["k_pages"].shape[0]
    old, lens = s["table"].tolist(), s["lens"].tolist()
    width = len(old[0])
    kept = [(p, min(k, lens[p]) if p >= 0 else 0) for p, k in zip(s["parents"].tolist(), s["keep"].tolist())]
    whole, part = set(), {}
    for c, (p, n) in enumerate(kept):
        whole.update(old[p][:n // page] if n else [])
        if n % page:
            part.setdefault(old[p][n // page], c)
    free = [p for p in range(n_pages) if p not in whole and p not in part]
    used, table, copies = 0, [], []
    for c, ((p, n), room) in enumerate(zip(kept, s["room"].tolist())):
        row = old[p][:n // page] if n else []
        moves = False
        if n % page:
            last = old[p][n // page]
            moves = last in whole or part[last] != c
            row = row if moves else row + [last]
        more = min(_ceil(n + room, page), width) - len(row)
        if moves:
            copies.append((last, free[used], n % page))
        row = row + free[used:used + more]
        used += more
        table.append(row + [-1] * (width - len(row)))
    pools = [s[name].to(torch.float32) for name in ("k_pages", "v_pages")]
    for src, dst, n in copies:
        for pool in pools:
            pool[dst, :, :n] = pool[src, :, :n]
    whole32 = dict(dtype=torch.int32, device="cuda")
    return dict(table=torch.tensor(table, **whole32), lens=torch.tensor([n for _, n in kept], **whole32),
                free=torch.tensor([len(free) - used], **whole32), k_pages=pools[0], v_pages=pools[1])


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "rotary":
        return tuple(_exact_rotate(s[x], s, case["adjacent"], case["inverse"]) for x in ("q", "k"))
    if kind == "append":
        k, q = s["k"], s["q"]
        if case["rotate"]:
            k, q = (_exact_rotate(x, s, case["adjacent"], False) for x in (k, q))
        pools = _exact_stored(s, k, s["v"])
        return dict(q=q.double(), k_pages=pools[0], v_pages=pools[1])
    return {"attention": _exact_attention, "keep": _exact_keep, "fork": _exact_fork}[kind](s, case)


# ---------------------------------------------------------------------------
# What a pass cannot do without
# ---------------------------------------------------------------------------

def work(case):
    kind, dim, kv = case["kind"], case["dim"], case["kv_heads"]
    if kind == "rotary":
        n, size = case["tokens"], 2 if case["dtype"] == "bf16" else 4
        values = n * (case["heads"] + kv) * dim
        return dict(bytes=2 * values * size + n * case["axes"] * 4 + case["rot"] // 2 * 12, flops=3 * values)
    size, rows = {"bf16": 2, "e4m3": 1, "fp32": 4}[case["cache"]], 4 if case["cache"] == "fp32" else 2
    entry = 2 * kv * dim                                     # values of a key and a value in all heads
    if kind == "append":
        counts = [case["new"] - (case["new"] * b // case["batch"] if case["ragged"] else 0) for b in range(case["batch"])]
        n, turned = sum(counts), case["batch"] * case["new"] * case["heads"] * dim if case["rotate"] else 0
        return dict(bytes=n * entry * (rows + size) + 2 * turned * rows + 8 * n, flops=3 * (turned + n * entry // 2))
    page = case["page"]
    if kind == "attention":
        lens = _lengths(case, case["nodes"])
        q = case["batch"] * case["nodes"] * case["heads"]
        return dict(bytes=sum(lens) * entry * size + 2 * q * dim * rows + 4 * q + 4 * sum(_ceil(n, page) for n in lens),
                    flops=4 * sum(lens) * case["nodes"] * case["heads"] * dim)
    if kind == "keep":
        n, moved = case["batch"] * case["nodes"], case["batch"] * (min(case["path"], case["nodes"]) - 1) // 2
        return dict(bytes=n * entry * (rows + size) + 2 * moved * entry * size, flops=n * entry)
    lens = _lengths(case, 1)
    c = max(case["batch"], case["width"])
    pages = sum(_ceil(n, page) for n in lens) // len(lens) * c
    copied = (c - _ceil(c, case["width"])) * page // 2       # entries of the last pages, half full
    return dict(bytes=2 * copied * entry * size + 8 * pages + 16 * c, flops=copied * entry + pages)
