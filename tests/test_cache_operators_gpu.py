"""The operators of the drafter's cache (rotary_axes, cache_append, paged_attention,
cache_keep, cache_fork) against their definitions in 64 bits.

Bounds count roundings (u = 2^-24 each of fp32) of the operations on one element, of the
sums, and of the last rounding to the stored type."""

import math

import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
BF16, FP32, E4M3 = torch.bfloat16, torch.float32, torch.float8_e4m3fn
HALF_ULP = {BF16: 2.0 ** -8, FP32: U}
I32 = dict(dtype=torch.int32, device="cuda")


@pytest.fixture(scope="module")
def fovea():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    from paper_2608_22883_gb300 import fovea as f
    f.lib()
    return f


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def normal(g, *shape):
    return torch.randn(shape, generator=g, device="cuda")


def ints(values):
    return torch.tensor(values, **I32)


def within(got, want, bound, what=""):
    """|got - want| <= bound element by element; equal where want is not finite."""
    got, want = got.double(), want.double()
    fine = torch.isfinite(want)
    assert torch.equal(torch.isnan(got), torch.isnan(want)), what
    assert torch.equal(got[~fine & ~torch.isnan(want)], want[~fine & ~torch.isnan(want)]), what
    err, b = (got - want).abs()[fine], torch.broadcast_to(bound, want.shape)[fine]
    assert bool((err <= b).all()), f"{what}: {float((err / b.clamp(min=1e-300)).max()):.3g} of the bound"


def same(a, b):
    """Equal bit for bit."""
    kind = {1: torch.uint8, 2: torch.int16, 4: torch.int32}[a.element_size()]
    return torch.equal(a.contiguous().view(kind), b.contiguous().view(kind))


# ---------------------------------------------------------------------------
# rotary_axes
# ---------------------------------------------------------------------------

def rotated(x, positions, frequencies, axis, adjacent, inverse=False):
    """(the rotated rows, the sums of magnitudes) in 64 bits."""
    x, half = x.double(), frequencies.numel()
    axis = torch.zeros(half, **I32) if axis is None else axis
    phi = (positions.double()[axis.long()].T * frequencies)[:, None]
    if inverse:
        phi = -phi
    first = torch.arange(half, device="cuda") * (2 if adjacent else 1)
    second = first + (1 if adjacent else half)
    a, b = x[..., first], x[..., second]
    y, size = x.clone(), torch.zeros_like(x)
    y[..., first] = a * torch.cos(phi) - b * torch.sin(phi)
    y[..., second] = a * torch.sin(phi) + b * torch.cos(phi)
    size[..., first] = size[..., second] = a.abs() + b.abs()
    return y, size


# Of an angle in half turns: its 32 bits (2^-31), rounded to fp32 (u), by pi; sincospif two
# roundings of values up to 1; a product and its sum two more: seven, with the 64-bit
# angle's own error at far positions beside them.
ROTARY = 8 * U


def check_rotary(fovea, q, k, positions, frequencies, axis, adjacent=False, inverse=False, stream=None):
    got = fovea.rotary_axes(q, k, positions, frequencies, axis, adjacent=adjacent, inverse=inverse, stream=stream)
    torch.cuda.synchronize()
    for x, y in zip((q, k), got):
        if x is None:
            assert y is None
            continue
        assert y.dtype == x.dtype and y.shape == x.shape and y.is_contiguous()
        want, size = rotated(x, positions, frequencies, axis, adjacent, inverse)
        within(y, want, want.abs() * HALF_ULP[x.dtype] + size * ROTARY + 1e-40, "rotated")
        rest = 2 * frequencies.numel()
        assert same(y[..., rest:], x[..., rest:])
    return got


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("adjacent", [False, True])
@pytest.mark.parametrize("n,heads,kv,dim,rot,axes", [
    (1, 32, 32, 128, 128, 1), (3, 28, 4, 128, 128, 3), (77, 5, 1, 64, 32, 2), (200, 40, 40, 128, 112, 4),
    (19, 2, 2, 256, 256, 3), (33, 3, 1, 80, 48, 2), (10, 3, 2, 81, 34, 3), (5, 1, 0, 2, 2, 1), (4, 7, 3, 512, 512, 8),
    (700, 12, 1, 96, 96, 3), (2, 1, 1, 17, 10, 1)])
def test_rotary(fovea, dtype, adjacent, n, heads, kv, dim, rot, axes):
    g = gen(n + dim)
    share = [rot // 2 // axes + (i < rot // 2 % axes) for i in range(axes)]
    f, axis = fovea.rotary_frequencies(rot, share, base=1e4, interleaved=bool(n % 2))
    q = normal(g, n, heads, dim).to(dtype)
    k = normal(g, n, kv, dim).to(dtype) if kv else None
    positions = torch.randint(-1000, 200000, (axes, n), generator=g, **I32)
    check_rotary(fovea, q, k, positions, f, axis, adjacent, inverse=bool(dim % 3))


@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_rotary_strides(fovea, dtype):
    g = gen(1)
    f, axis = fovea.rotary_frequencies(128, [16, 24, 24], base=1e6)
    positions = torch.randint(0, 5000, (3, 40), generator=g, **I32)
    x = normal(g, 40, 36 * 128 + 8).to(dtype)                    # one projection's output, padded rows
    heads = x[:, :36 * 128].unflatten(1, (36, 128))
    assert not heads.is_contiguous()
    check_rotary(fovea, heads[:, :28], heads[:, 28:32], positions, f, axis)
    odd = normal(g, 40, 12 * 128 + 3).to(dtype)[:, 3:].unflatten(1, (12, 128))     # off the vectors' boundary
    check_rotary(fovea, odd[:, :8], odd[:, 8:], positions, f, axis, adjacent=True)
    by_head = normal(g, 6, 40, 128).to(dtype).transpose(0, 1)    # heads outside tokens
    check_rotary(fovea, by_head[:, :4], by_head[:, 4:], positions, f, axis)
    one = normal(g, 1, 1, 128).to(dtype).expand(40, 4, 128)      # one head for all
    check_rotary(fovea, one, None, positions, f, axis)
    wide = torch.zeros(3, 64, **I32)
    wide[:, :40] = positions
    check_rotary(fovea, heads[:, :28], None, wide[:, :40], f, axis)
    check_rotary(fovea, heads[:, :28], None, positions[:1].expand(3, 40), f, axis)       # one position for all axes


def test_rotary_far_positions(fovea):
    """Angles are right at every 32-bit position: whole turns go in exact arithmetic."""
    f = torch.tensor([1.0, 0.5, 2 * math.pi / 3, 1e-3, 1e-7, 2.5, math.pi, 0.0], dtype=torch.float64, device="cuda")
    at = [0, 1, -1, 999999937, 2 ** 31 - 1, -2 ** 31, 123456789, 10 ** 6]
    positions = ints([at])
    q = torch.zeros(len(at), 1, 16, device="cuda")
    q[..., :8] = 1.0                                             # gives cos and sin themselves
    got, _ = fovea.rotary_axes(q, None, positions, f)
    # frequencies as the exact rationals that they are, reduced by 2 pi with 60 digits
    from fractions import Fraction
    turn = Fraction(int("6283185307179586476925286766559005768394338798750211641949889"), 10 ** 60)
    for n, p in enumerate(at):
        for j, w in enumerate(f.tolist()):
            phi = Fraction(w) * p / turn
            phi = 2 * math.pi * float(phi - math.floor(phi))
            # one rounding of f / 2 pi to 53 bits, times the position
            tol = ROTARY + abs(p * w) * 2.0 ** -52
            assert abs(float(got[n, 0, j]) - math.cos(phi)) <= tol, (p, w)
            assert abs(float(got[n, 0, 8 + j]) - math.sin(phi)) <= tol, (p, w)


@pytest.mark.parametrize("adjacent", [False, True])
def test_rotary_gradient(fovea, adjacent):
    """inverse=True is the gradient: against the formula's and against differences."""
    g = gen(4)
    n, h, dim = 6, 3, 32
    f, axis = fovea.rotary_frequencies(24, [4, 4, 4], base=100.0)
    positions = torch.randint(0, 100, (3, n), generator=g, **I32)
    x, dy = normal(g, n, h, dim), normal(g, n, h, dim)
    dx, _ = check_rotary(fovea, dy, None, positions, f, axis, adjacent, inverse=True)
    leaf = x.double().requires_grad_()
    a = leaf[..., 0:24:2] if adjacent else leaf[..., :12]
    b = leaf[..., 1:24:2] if adjacent else leaf[..., 12:24]
    phi = (positions.double()[axis.long()].T * f)[:, None]
    c, d = a * phi.cos() - b * phi.sin(), a * phi.sin() + b * phi.cos()
    y = torch.cat((torch.stack((c, d), -1).flatten(-2) if adjacent else torch.cat((c, d), -1), leaf[..., 24:]), -1)
    y.backward(dy.double())
    within(dx, leaf.grad, (dy.double().abs().amax() * 2 * ROTARY).expand_as(leaf), "gradient")
    # the operator is linear: its difference along v is its value at v, to both values' errors
    v = normal(g, n, h, dim)
    up, _ = fovea.rotary_axes(x + v, None, positions, f, axis, adjacent=adjacent)
    at, _ = fovea.rotary_axes(x, None, positions, f, axis, adjacent=adjacent)
    step = ((up.double() - at.double()) * dy.double()).sum()
    want = (dx.double() * ((x + v).double() - x.double())).sum()
    size = ((x.abs() + v.abs()) * dy.abs()).double().sum()
    assert abs(float(step - want)) <= float(size) * 6 * ROTARY


def test_rotary_bad_frequencies(fovea):
    f = torch.tensor([1.0, float("nan"), float("inf"), 2.0], dtype=torch.float64, device="cuda")
    axis = ints([0, 0, 1, 2])
    x = torch.ones(3, 2, 8, device="cuda")
    y, _ = fovea.rotary_axes(x, None, ints([[1, 2, 3], [4, 5, 6]]), f, axis)
    bad = torch.isnan(y)
    assert bad[..., [1, 2, 3, 5, 6, 7]].all() and not bad[..., [0, 4]].any()


# ---------------------------------------------------------------------------
# A cache and its plain reading
# ---------------------------------------------------------------------------

def make_cache(g, cache, lens, kv, dim, page, spare=3, shuffle=True, width=None):
    """Pools with pages for these lengths in random order, and their table."""
    counts = [-(-n // page) for n in lens]
    n_pages = sum(counts) + spare
    order = torch.randperm(n_pages, generator=g, device="cuda") if shuffle else torch.arange(n_pages, device="cuda")
    table = torch.full((len(lens), width or max(counts + [1])), -1, **I32)
    at = 0
    for b, c in enumerate(counts):
        table[b, :c] = order[at:at + c].to(torch.int32)
        at += c
    shape = (n_pages, kv, page, dim)
    if cache is E4M3:
        k, v = ((100 * normal(g, *shape)).clamp(-448, 448).to(E4M3) for _ in range(2))
        scales = dict(k_scale=(0.5 + torch.rand(kv, generator=g, device="cuda")) / 100,
                      v_scale=(0.5 + torch.rand(kv, generator=g, device="cuda")) / 100)
    else:
        k, v = (normal(g, *shape).to(cache) for _ in range(2))
        scales = dict()
    return k, v, table, scales


def entries(pool, table, b, n):
    """[n, kv, dim] of a sequence, as stored."""
    page = pool.shape[2]
    at = torch.arange(n, device="cuda")
    raw = pool.view(torch.uint8) if pool.dtype is E4M3 else pool
    x = raw[table[b].long()[at // page], :, at % page]
    return x.view(E4M3) if pool.dtype is E4M3 else x


def seen_of(tree, b, nodes, n):
    """[nodes, n] truth values."""
    at = torch.arange(n, device="cuda")
    j = at - (n - nodes)
    if tree is None:
        bits = torch.ones(nodes, nodes, device="cuda").tril().bool()
    else:
        words = tree[b if tree.shape[0] > 1 else 0].long()
        i = torch.arange(nodes, device="cuda")
        bits = (words[:, i // 32] >> (i % 32)) & 1 == 1
    return (j < 0)[None] | bits[:, j.clamp(0, nodes - 1)]


def check_attention(fovea, q, k_pages, v_pages, table, lens, tree=None, scale=None, scales={}, **kw):
    got = fovea.paged_attention(q, k_pages, v_pages, table, lens, tree=tree, scale=scale, want_lse=True, **scales, **kw)
    torch.cuda.synchronize()
    out, lse = got["out"], got["lse"]
    B, heads, dim = table.shape[0], q.shape[1], q.shape[2]
    kv = k_pages.shape[1]
    nodes, group = q.shape[0] // B, heads // kv
    scale = dim ** -0.5 if scale is None else scale
    assert out.shape == q.shape and out.dtype == q.dtype and lse.shape == q.shape[:2]
    got["bounds"] = []
    p_error = {BF16: 2.0 ** -16, E4M3: 2.0 ** -11, FP32: 2.0 ** -21}[k_pages.dtype]
    for b, n in enumerate(lens.tolist()):
        rows = slice(b * nodes, (b + 1) * nodes)
        if n <= 0:
            assert not out[rows].any() and bool((lse[rows] == -math.inf).all())
            got["bounds"].append(None)
            continue
        k, v = (entries(x, table, b, n).double() for x in (k_pages, v_pages))
        if scales:
            k, v = k * scales["k_scale"].double()[:, None], v * scales["v_scale"].double()[:, None]
        x = q[rows].double().view(nodes, kv, group, dim)
        seen = seen_of(tree, b, nodes, n)[:, None, None]
        # masked places may hold anything: taken out before the sums
        z = torch.where(seen, torch.einsum("tkgd,nkd->tkgn", x, k) * scale, -math.inf)
        top = z.amax(-1, keepdim=True).nan_to_num(neginf=0.0)
        e = torch.exp(z - top)
        total = e.sum(-1, keepdim=True)
        p = e / torch.where(total > 0, total, 1.0)
        want_lse = (top + total.log())[..., 0]
        want = torch.zeros(nodes, kv, group, dim, dtype=torch.float64, device="cuda")
        size = torch.zeros_like(want)
        for t in range(nodes):
            use = seen[t, 0, 0]
            want[t] = torch.einsum("kgn,nkd->kgd", p[t][..., use], v[use])
            size[t] = torch.einsum("kgn,nkd->kgd", p[t][..., use], v[use].nan_to_num(0, 0, 0).abs())
        # Scores: products exact (bf16) or to 2^-21 (three tf32 products, fp16's smallest
        # step), and dim / 8 additions that truncate, each to 2^-23 of the sum of
        # magnitudes; two roundings of the scaled score; 2^-22 of the exponential.
        sizes = torch.einsum("tkgd,nkd->tkgn", x.abs(), k.nan_to_num(0, 0, 0).abs()) * abs(scale)
        sizes = torch.where(seen, sizes, 0.0).amax(-1)
        delta = sizes * (dim / 8 + 8) * 2.0 ** -22 + 2.0 ** -21
        # Sums: a truncated addition a block of 16 and part of p, the joins of warps and runs.
        sums = (n / 8 + 64) * 2.0 ** -23
        bound = want.abs() * HALF_ULP[q.dtype] + size * (2 * delta[..., None] + sums + p_error) + 1e-38
        got["bounds"].append(bound)
        within(out[rows].view_as(want), want, bound, f"out of sequence {b}")
        within(lse[rows].view_as(want_lse), want_lse, delta + sums + want_lse.abs().nan_to_num(0, 0, 0) * 2 * U, f"lse {b}")
    return got


def tree_bits(g, batch, nodes, empty=False):
    """Random trees' ancestors as words; with `empty`, one node that sees none of the tree."""
    seen = torch.zeros(batch, nodes, -(-nodes // 32) * 32, dtype=torch.bool, device="cuda")
    rows = torch.arange(batch, device="cuda")
    for j in range(nodes):
        if j:
            seen[:, j] = seen[rows, torch.randint(0, j, (batch,), generator=g, device="cuda")]
        seen[:, j, j] = True
    if empty:
        seen[:, nodes // 2] = False
    words = (seen.view(batch, nodes, -1, 32).long() << torch.arange(32, device="cuda")).sum(-1)
    return torch.where(words >= 1 << 31, words - (1 << 32), words).to(torch.int32)


CASES = [
    # lens, nodes, heads, kv, dim, page
    ([1], 1, 1, 1, 64, 16),
    ([2, 17, 16, 15], 1, 2, 1, 128, 16),
    ([640], 1, 32, 32, 128, 64),
    ([0, 5, 33, 0], 1, 7, 1, 128, 32),
    ([1000, 1, 63, 64, 65, 128, 300], 1, 28, 4, 128, 48),
    ([5000, 12], 1, 12, 1, 256, 64),
    ([3000, 2999], 1, 32, 4, 64, 128),
    ([7, 70, 700], 7, 5, 5, 128, 16),
    ([64, 65, 333], 64, 28, 4, 128, 64),
    ([40, 33], 33, 3, 1, 64, 16),
    ([300], 256, 2, 1, 128, 1024),
    ([20, 3, 0, 9], 9, 4, 2, 64, 16),             # a sequence shorter than its rows
    ([50, 49], 3, 6, 2, 256, 16),
    ([129] * 40, 1, 40, 40, 64, 64),
]


@pytest.mark.parametrize("cache", [BF16, E4M3, FP32])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_attention(fovea, cache, case):
    lens, nodes, heads, kv, dim, page = CASES[case]
    g = gen(case)
    k, v, table, scales = make_cache(g, cache, lens, kv, dim, page)
    q = (2 * normal(g, len(lens) * nodes, heads, dim)).to(FP32 if cache is FP32 else BF16)
    check_attention(fovea, q, k, v, table, ints(lens), scales=scales)
    if nodes > 1:
        for batch in (len(lens), 1):
            check_attention(fovea, q, k, v, table, ints(lens), tree_bits(g, batch, nodes, True), scales=scales)


@pytest.mark.parametrize("cache", [BF16, E4M3])
@pytest.mark.parametrize("lens,nodes,heads,kv,dim", [
    ([2912, 1531, 805, 423, 222, 117, 61, 32], 32, 28, 4, 128), ([64, 65, 333], 64, 28, 4, 128), ([700], 64, 32, 32, 128),
    ([600] * 16, 64, 40, 40, 128), ([900, 30, 64, 1500], 12, 16, 2, 64), ([1000, 900], 7, 8, 2, 256)])
def test_attention_repeats(fovea, cache, lens, nodes, heads, kv, dim):
    """Trees through every kernel of many rows give the same bits in every run, with the
    machine to themselves and behind other work."""
    g = gen(17)
    k, v, table, scales = make_cache(g, cache, lens, kv, dim, 16)
    q = (2 * normal(g, len(lens) * nodes, heads, dim)).to(BF16)
    tree = tree_bits(g, len(lens), nodes)
    want = check_attention(fovea, q, k, v, table, ints(lens), tree, scales=scales)
    for _ in range(5):
        got = [fovea.paged_attention(q, k, v, table, ints(lens), tree=tree, want_lse=True, **scales) for _ in range(20)]
        torch.cuda.synchronize()
        assert all(same(r["out"], want["out"]) and same(r["lse"], want["lse"]) for r in got)


@pytest.mark.parametrize("cache", [BF16, E4M3, FP32])
def test_attention_long(fovea, cache):
    g = gen(9)
    lens = [60000, 0, 123, 31000]
    k, v, table, scales = make_cache(g, cache, lens, 2, 128, 64)
    q = (3 * normal(g, 4, 8, 128)).to(FP32 if cache is FP32 else BF16)
    a = check_attention(fovea, q, k, v, table, ints(lens), scales=scales)
    b = fovea.paged_attention(q, k, v, table, ints(lens), want_lse=True, **scales)
    assert same(a["out"], b["out"]) and same(a["lse"], b["lse"])             # repeats bit for bit


def test_attention_rows_that_see_nothing(fovea):
    g = gen(2)
    lens, nodes = [4, 30], 4                       # the first sequence holds its new entries alone
    k, v, table, _ = make_cache(g, BF16, lens, 2, 64, 16)
    q = normal(g, 8, 4, 64).to(BF16)
    tree = ints([[[0], [2], [0], [15]], [[0], [0], [0], [0]]])
    got = check_attention(fovea, q, k, v, table, ints(lens), tree)
    assert not got["out"][0].any() and bool((got["lse"][0] == -math.inf).all())
    assert bool(torch.isfinite(got["lse"][4:]).all())


@pytest.mark.parametrize("cache", [BF16, E4M3, FP32])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf"), "lowest"])
def test_attention_masked_places(fovea, cache, value):
    """What stands behind a sequence, or at a node that a row does not see, is not used; a
    row that sees it takes it."""
    g = gen(3)
    lens, nodes, page = [45, 20], 6, 16
    k, v, table, scales = make_cache(g, cache, lens, 2, 128, page)
    wide = 448.0 if cache is E4M3 else torch.finfo(cache).max
    x = -wide if value == "lowest" else value
    if cache is E4M3 and x in (float("inf"), -float("inf")):
        x = float("nan")                           # what such a value is stored as
    for b, n in enumerate(lens):
        spoiled = [(n + i, (k, v)) for i in range(-(-n // page) * page - n)] + [(n - nodes + 2, (v,))]
        for e, pools in spoiled:
            for pool in pools:
                pool[int(table[b, e // page]), :, e % page, ::3] = torch.tensor(x).to(cache).cuda()
    q = normal(g, 2 * nodes, 4, 128).to(FP32 if cache is FP32 else BF16)
    check_attention(fovea, q, k, v, table, ints(lens), tree_bits(g, 2, nodes), scales=scales)
    check_attention(fovea, q, k, v, table, ints(lens), scales=scales)
    # a key that is no number, at a node
    k[int(table[0, 41 // page]), 1, 41 % page, 5] = torch.tensor(float("nan")).to(cache).cuda()
    got = check_attention(fovea, q, k, v, table, ints(lens), tree_bits(g, 2, nodes), scales=scales)
    assert bool(torch.isfinite(got["lse"][:, :2]).all())


def test_attention_large_scores(fovea):
    """Scores beyond what e^x holds, a key that dominates, rows of equal scores."""
    g = gen(5)
    for cache in (BF16, FP32, E4M3):
        k, v, table, scales = make_cache(g, cache, [500, 500], 1, 64, 16)
        q = normal(g, 2, 8, 64).to(FP32 if cache is FP32 else BF16)
        q[0] *= 1000
        q[1] = 0
        check_attention(fovea, q, k, v, table, ints([500, 500]), scales=scales)
        q[1, 0] = 2.0 ** -120                      # far below fp16's range
        q[1, 1] = 2.0 ** 100
        k2 = k if cache is E4M3 else (k.float() * 2.0 ** -90).to(cache)
        check_attention(fovea, q, k2, v, table, ints([500, 500]), scale=2.0 ** -10, scales=scales)


def test_attention_bad_pages(fovea):
    """Pages outside the pool and lengths beyond the table make the rows that need them NaN."""
    g = gen(6)
    for cache in (BF16, E4M3, FP32):
        lens = [100, 100, 100, 100, 30]
        k, v, table, scales = make_cache(g, cache, lens, 2, 64, 16, width=8)
        q = normal(g, 5, 4, 64).to(FP32 if cache is FP32 else BF16)
        want = check_attention(fovea, q, k, v, table, ints(lens), scales=scales)
        table[0, 3] = -1
        table[1, 6] = k.shape[0]
        table[4, 2:] = 2 ** 31 - 1                 # behind the last one: not used
        got = fovea.paged_attention(q, k, v, table, ints(lens), want_lse=True, **scales)
        for x, y in ((got["out"], want["out"]), (got["lse"], want["lse"])):
            assert bool(torch.isnan(x[:2]).all()) and same(x[2:], y[2:])
        # other lengths cut the sums elsewhere: two results, each within the bound
        got = fovea.paged_attention(q, k, v, table, ints([100, 100, 129, 100, -5]), want_lse=True, **scales)
        assert bool(torch.isnan(got["out"][:3]).all()) and bool(torch.isnan(got["lse"][:3]).all())
        within(got["out"][3], want["out"][3].double(), 2 * want["bounds"][3].view_as(got["out"][3]))
        assert not got["out"][4].any() and bool((got["lse"][4] == -math.inf).all())
        # a node's own row alone needs the page of the newest entries
        got = fovea.paged_attention(q[:4], k, v, table[1:3], ints([97, 97]), **scales,
                                    tree=ints([[[1], [2]], [[1], [2]]]))
        assert bool(torch.isfinite(got["out"][0]).all()) and bool(torch.isnan(got["out"][1]).all())
        assert bool(torch.isfinite(got["out"][2:]).all())


def test_attention_strides_and_shared_pages(fovea):
    g = gen(7)
    k, v, table, _ = make_cache(g, BF16, [200, 200, 90], 4, 128, 32)
    table[1, :3] = table[0, :3]                    # a forked sequence
    table[2] = table[0]
    lens = ints([200, 200, 90])
    x = normal(g, 3, (28 + 8) * 128 + 5).to(BF16)
    q = x[:, 1:1 + 28 * 128].unflatten(1, (28, 128))
    check_attention(fovea, q, k, v, table, lens)
    by_head = normal(g, 28, 3, 128).to(BF16).transpose(0, 1)
    check_attention(fovea, by_head, k, v, table, lens)
    check_attention(fovea, x[:, :128].unflatten(1, (1, 128)).expand(3, 8, 128), k, v, table, lens)


def test_attention_many_sequences(fovea):
    """More sequences than a CTA has threads, most of them short or empty."""
    g = gen(8)
    lens = [(7 * i) % 50 if i % 3 else 0 for i in range(300)]
    k, v, table, _ = make_cache(g, BF16, lens, 1, 64, 16)
    q = normal(g, 300, 2, 64).to(BF16)
    check_attention(fovea, q, k, v, table, ints(lens))
    check_attention(fovea, q, k, v, table, ints([0] * 300))


# ---------------------------------------------------------------------------
# cache_append
# ---------------------------------------------------------------------------

def stored(x, scale, cache):
    """(value of the stored 8 bits or the row itself, bound) in 64 bits."""
    x = x.double()
    if cache is not E4M3:
        return x, x.abs() * HALF_ULP[cache]
    y = (x / scale.double()[:, None]).clamp(-448, 448)
    return y, y.abs() * (2.0 ** -4 + 4 * U) + 2.0 ** -10


@pytest.mark.parametrize("cache", [BF16, E4M3, FP32])
@pytest.mark.parametrize("rotate,adjacent", [(False, False), (True, False), (True, True)])
@pytest.mark.parametrize("n,heads,kv,dim,page", [(1, 4, 1, 64, 16), (37, 28, 4, 128, 48), (150, 3, 3, 256, 16),
                                                 (9, 40, 40, 128, 64)])
def test_append(fovea, cache, rotate, adjacent, n, heads, kv, dim, page):
    g = gen(n + dim)
    dt = FP32 if cache is FP32 else BF16
    starts, news = [5, 0, 30], [n - n // 3, 0, n // 3]
    k_pages, v_pages, table, scales = make_cache(g, cache, [s + c for s, c in zip(starts, news)], kv, dim, page)
    sequence = torch.cat([torch.full((c,), b, **I32) for b, c in enumerate(news)])
    entry = torch.cat([torch.arange(s, s + c, **I32) for s, c in zip(starts, news)])
    order = torch.randperm(n, generator=g, device="cuda")
    sequence, entry = sequence[order], entry[order]
    if n > 4:
        sequence[3] = -1                            # a padded row
    x = normal(g, n, heads + 2 * kv, dim).to(dt)
    q, k, v = x[:, :heads], x[:, heads:heads + kv], x[:, heads + kv:]
    more = {}
    want_k, size = k.double(), torch.zeros(())
    if rotate:
        f, axis = fovea.rotary_frequencies(dim - 16, [dim // 4, dim // 4 - 8], base=1e4)
        positions = torch.randint(0, 10000, (2, n), generator=g, **I32)
        more = dict(q=q, positions=positions, frequencies=f, axis=axis, adjacent=adjacent)
        want_k, size = rotated(k, positions, f, axis, adjacent)
    before = k_pages.clone(), v_pages.clone()
    got = fovea.cache_append(k, v, k_pages, v_pages, table, sequence, entry, **scales, **more)
    torch.cuda.synchronize()
    if rotate:
        want, mag = rotated(q, positions, f, axis, adjacent)
        within(got, want, want.abs() * HALF_ULP[dt] + mag * ROTARY + 1e-40, "q")
    else:
        assert got is None
    touched = torch.zeros(k_pages.shape[0], page, dtype=torch.bool, device="cuda")
    use = sequence >= 0
    place = table[sequence[use].long(), entry[use].long() // page].long(), entry[use].long() % page
    touched[place] = True
    for pool, old, want, mag, scale in ((k_pages, before[0], want_k, size, scales.get("k_scale")),
                                        (v_pages, before[1], v.double(), torch.zeros(()), scales.get("v_scale"))):
        flat = pool.view(torch.uint8).view(*pool.shape[:3], -1) if cache is E4M3 else pool
        there = flat[place[0], :, place[1]]
        there = there.view(E4M3) if cache is E4M3 else there
        y, bound = stored(want, scale, cache)
        mag = mag.to(y) if mag.dim() == 0 else mag
        if scale is not None:
            mag = mag / scale.double()[:, None]
        mag = torch.broadcast_to(mag, y.shape)
        within(there, y[use], bound[use] + mag[use] * ROTARY * 1.1 + 1e-40, "entries")
        same_old = [a.transpose(1, 2)[~touched] for a in (pool, old)] if cache is not E4M3 else \
            [a.view(torch.uint8).view(*a.shape[:3], -1).transpose(1, 2)[~touched] for a in (pool, old)]
        assert same(*same_old)                       # all others as they were


def test_append_ends_and_bad_places(fovea):
    g = gen(3)
    k_pages, v_pages, table, scales = make_cache(g, E4M3, [32, 32], 1, 64, 16, width=2)
    table[1, 1] = k_pages.shape[0]
    before = k_pages.clone(), v_pages.clone()
    k = torch.tensor([1e30, -1e30, float("inf"), float("nan"), 0.0, 1e-30, -0.0, 3.0], device="cuda").to(BF16)
    k = k.repeat(8)[None, None].expand(7, 1, 64).contiguous()
    sequence, entry = ints([0, 2, -1, 0, 0, 1, -2 ** 31]), ints([3, 0, 0, 32, -1, 20, 0])
    fovea.cache_append(k, k, k_pages, v_pages, table, sequence, entry,
                       k_scale=torch.ones(1, device="cuda"), v_scale=torch.full((1,), 2.0, device="cuda"))
    row, page = k_pages[int(table[0, 0]), 0, 3].float(), int(table[0, 0])
    assert row[:3].tolist() == [448.0, -448.0, 448.0] and bool(torch.isnan(row[3])) and row[4:8].tolist() == [0, 0, 0, 3]
    assert float(v_pages[page, 0, 3, 7].float()) == 1.5
    for pool, old in zip((k_pages, v_pages), before):
        a, b = pool.view(torch.uint8).clone(), old.view(torch.uint8)
        a[page, 0, 3] = b[page, 0, 3]
        assert torch.equal(a, b)


# ---------------------------------------------------------------------------
# cache_keep
# ---------------------------------------------------------------------------

@pytest.mark.parametrize("cache", [BF16, E4M3, FP32])
@pytest.mark.parametrize("dim,kv,page,size,paths", [
    (128, 4, 16, 64, [[0, 3, 9, 20, 35, 50], [0], [], [5, 4, 3, 2], [63, 63, 0]]),
    (64, 1, 48, 7, [[0, 1, 2, 3, 4, 5, 6], [6], [1, 2, 99, 3]]),
    (256, 2, 64, 256, [list(range(0, 256, 2)), list(range(255, -1, -1))]),
])
def test_keep(fovea, cache, dim, kv, page, size, paths):
    g = gen(size)
    lens = [size + 13 * b for b in range(len(paths))] + [size - 1, 0]
    k, v, table, _ = make_cache(g, cache, lens, kv, dim, page)
    most = max(len(p) for p in paths)
    nodes = ints([p + [-1] * (most - len(p)) for p in paths] + [[0] * most] * 2)
    if most > 2:
        nodes[0, len(paths[0]):] = -7
    before = k.clone(), v.clone()
    got = fovea.cache_keep(k, v, table, ints(lens), nodes, size)
    torch.cuda.synchronize()
    want = [x.view(torch.uint8).view(*x.shape[:3], -1).clone() for x in before]
    new = []
    for b, n in enumerate(lens):
        path = nodes[b].tolist()
        path = path[:next((i for i, x in enumerate(path) if not 0 <= x < size), len(path))]
        if n < size:
            new.append(n)
            continue
        new.append(n - size + len(path))
        for pool, old in zip(want, before):
            old = old.view(torch.uint8).view(*old.shape[:3], -1)
            for i, x in enumerate(path):
                to, src = n - size + i, n - size + x
                pool[int(table[b, to // page]), :, to % page] = old[int(table[b, src // page]), :, src % page]
    assert got.tolist() == new
    for pool, x in zip((k, v), want):
        assert torch.equal(pool.view(torch.uint8).view(*pool.shape[:3], -1), x)


def test_keep_bad_pages(fovea):
    g = gen(1)
    k, v, table, _ = make_cache(g, BF16, [40], 1, 64, 16)
    before = k.clone()
    table[0, 1] = -1                                # entries 16 to 31
    got = fovea.cache_keep(k, v, table, ints([40]), ints([[2, 30, 35, 39]]), 40)
    assert got.tolist() == [4]
    p, last = int(table[0, 0]), int(table[0, 2])
    assert same(k[p, 0, 0], before[p, 0, 2]) and same(k[p, 0, 1], before[p, 0, 1])
    assert same(k[p, 0, 2], before[last, 0, 3]) and same(k[p, 0, 3], before[last, 0, 7])
    # a length beyond the table
    before = k.clone()
    assert fovea.cache_keep(k, v, table, ints([60]), ints([[19]]), 20).tolist() == [41]
    assert same(k, before)
    # lengths below zero, down to the lowest
    for n in (-1, -2 ** 31, -2 ** 31 + 19):
        assert fovea.cache_keep(k, v, table, ints([n]), ints([[19]]), 20).tolist() == [n]
    assert same(k, before)


# ---------------------------------------------------------------------------
# cache_fork
# ---------------------------------------------------------------------------

def fork_reference(table, lens, parents, keep, room, n_pages, page, width):
    """(new table, lengths, free pages, copies (from, to, entries)) by the definition."""
    kept = []
    for c, p in enumerate(parents):
        n = 0
        if 0 <= p < len(lens):
            n = max(0, min(lens[p], len(table[p]) * page, width * page))
            n = max(0, min(n, keep[c])) if keep is not None else n
        kept.append((p, n))
    ok = lambda x: 0 <= x < n_pages
    whole = {x for p, n in kept if n for x in table[p][:n // page] if ok(x)}
    part = {}
    for c, (p, n) in enumerate(kept):
        if n % page and ok(table[p][n // page]):
            part.setdefault(table[p][n // page], c)
    free = [x for x in range(n_pages) if x not in whole and x not in part]
    fresh, rows, copies = iter(free + [-1] * 10 ** 6), [], []
    used = 0
    for c, (p, n) in enumerate(kept):
        row = list(table[p][:n // page]) if n else []
        need = min(-(-(n + max(0, room[c] if room is not None else 0)) // page), width)
        if n % page:
            last = table[p][n // page]
            if not ok(last) or (last not in whole and part[last] == c):
                row.append(last)
            else:
                copies.append((last, c, len(row), n % page))
        while len(row) < need:
            row.append(next(fresh))
            used += 1
        rows.append(row + [-1] * (width - len(row)))
    copies = [(src, rows[c][i], n) for src, c, i, n in copies]
    return rows, [n for _, n in kept], len(free) - used, copies


def check_fork(fovea, k, v, table, lens, parents, keep=None, room=None, width=None):
    before = [x.view(torch.uint8).view(*x.shape[:3], -1).clone() for x in (k, v)]
    got = fovea.cache_fork(k, v, table, ints(lens), ints(parents), None if keep is None else ints(keep),
                           None if room is None else ints(room), width=width)
    torch.cuda.synchronize()
    rows, new, free, copies = fork_reference(table.tolist(), lens, parents, keep, room, k.shape[0], k.shape[2],
                                             width or table.shape[1])
    assert got["table"].tolist() == rows
    assert got["lens"].tolist() == new and got["free"].tolist() == [free]
    for x, old in zip((k, v), before):
        if free >= 0:
            for src, dst, n in copies:
                old[dst, :, :n] = old[src, :, :n].clone()
        assert torch.equal(x.view(torch.uint8).view(*x.shape[:3], -1), old)
    return got


@pytest.mark.parametrize("cache", [BF16, E4M3, FP32])
def test_fork(fovea, cache):
    g = gen(1)
    lens = [100, 37, 0, 64, 1, 200]
    k, v, table, _ = make_cache(g, cache, lens, 2, 64, 16, spare=40, width=20)
    check_fork(fovea, k, v, table, lens, [0, 1, 2, 3, 4, 5])                              # as it was
    check_fork(fovea, k, v, table, lens, [0, 0, 0, 1, 1, 5])                              # forked, dropped
    check_fork(fovea, k, v, table, lens, [5, 5, 5, 5], [200, 195, 192, 20], [64, 0, 1, 33])   # cut inside others' pages
    check_fork(fovea, k, v, table, lens, [-1, 6, 100, 2, 0], None, [16, 0, 1, 17, -5])    # of none
    check_fork(fovea, k, v, table, lens, [0, 1], [-3, 1000], [400, 400])                  # bounds of keep, of width
    check_fork(fovea, k, v, table, lens, [0, 1, 5, 5], [100, 37, 170, 200], width=5)      # a narrower table
    check_fork(fovea, k, v, table, lens, [5, 0], room=[100, 7], width=31)                 # a wider one
    check_fork(fovea, k, v, table, lens, [])


def test_fork_shortage_and_bad_pages(fovea):
    g = gen(2)
    lens = [50, 50]
    k, v, table, _ = make_cache(g, BF16, lens, 1, 64, 16, spare=0, width=6)
    got = check_fork(fovea, k, v, table, lens, [0, 0, 0, 1, 1])                           # nothing is free
    assert got["free"].tolist() == [-3]
    check_fork(fovea, k, v, table, lens, [0, 0], None, [30, 0])                           # the dropped one's pages
    table[0, 1], table[0, 3], table[1, 3] = -1, k.shape[0], -9
    check_fork(fovea, k, v, table, lens, [0, 0, 1, 1])


def test_fork_many(fovea):
    """Many continuations and pages: more of both than threads."""
    g = gen(3)
    lens = [int(x) for x in torch.randint(0, 300, (1500,), generator=g, device="cuda").tolist()]
    k, v, table, _ = make_cache(g, BF16, lens, 1, 64, 16, spare=30000)
    parents = torch.randint(-1, 1500, (2048,), generator=g, device="cuda").tolist()
    room = torch.randint(0, 200, (2048,), generator=g, device="cuda").tolist()
    check_fork(fovea, k, v, table, lens, parents, None, room, width=table.shape[1] + 8)


# ---------------------------------------------------------------------------
# Together, and as programs call them
# ---------------------------------------------------------------------------

@pytest.mark.parametrize("cache,n_pages", [(BF16, 36000), (E4M3, 70000), (FP32, 18000)])
def test_offsets_beyond_32_bits(fovea, cache, n_pages):
    """Pools of more than 2^32 bytes (of 8 bits: elements), entries in their last pages."""
    g = gen(18)
    kv, page, dim, dt = 8, 64, 128, FP32 if cache is FP32 else BF16
    assert n_pages * kv * page * dim * torch.empty(0, dtype=cache).element_size() > 1 << 32
    k_pages, v_pages = (torch.empty(n_pages, kv, page, dim, dtype=cache, device="cuda") for _ in range(2))
    scales = dict(k_scale=torch.full((kv,), 0.02, device="cuda"), v_scale=torch.full((kv,), 0.01, device="cuda")) \
        if cache is E4M3 else {}
    table = ints([[n_pages - 1, n_pages - 3, n_pages - 5], [n_pages - 2, 1, n_pages - 4]])
    lens, nodes = [170, 129], 20
    sequence = torch.cat([torch.full((n,), b, **I32) for b, n in enumerate(lens)])
    entry = torch.cat([torch.arange(n, **I32) for n in lens])
    x = normal(g, sum(lens), 2 * kv, dim).to(dt)
    fovea.cache_append(x[:, :kv], x[:, kv:], k_pages, v_pages, table, sequence, entry, **scales)
    for heads in (16, 40):                          # few rows a key head, and many
        q = normal(g, 2 * nodes, heads, dim).to(dt)
        check_attention(fovea, q, k_pages, v_pages, table, ints(lens), scales=scales)
    rows = entries(v_pages, table, 0, 170).clone()
    held = fovea.cache_keep(k_pages, v_pages, table, ints(lens), ints([[3, 19], [0, -1]]), nodes)
    assert held.tolist() == [152, 110]
    assert same(entries(v_pages, table, 0, 152)[150:], rows[[153, 169]])
    r = fovea.cache_fork(k_pages, v_pages, table, held, ints([0, 0]), None, ints([0, 0]))
    assert r["table"].tolist() == [[n_pages - 1, n_pages - 3, n_pages - 5], [n_pages - 1, n_pages - 3, 0]]
    assert same(entries(k_pages, r["table"], 1, 152), entries(k_pages, table, 0, 152))

@pytest.mark.parametrize("cache", [BF16, E4M3, FP32])
def test_a_draft_round(fovea, cache):
    """Prompts stored, trees drafted, verified and kept, sequences forked, one token decoded:
    the attention at each step against the rows that a plain list of entries gives."""
    g = gen(11)
    dt, kv, heads, dim, page, nodes = FP32 if cache is FP32 else BF16, 2, 6, 64, 16, 12
    f, axis = fovea.rotary_frequencies(dim, [12, 10, 10], base=1e4)
    lens = [33, 1, 20]
    n_pages = 60
    k_pages, v_pages = (torch.zeros(n_pages, kv, page, dim, device="cuda").to(cache) for _ in range(2))
    scales = dict(k_scale=torch.full((kv,), 0.02, device="cuda"), v_scale=torch.full((kv,), 0.01, device="cuda")) \
        if cache is E4M3 else {}
    empty = torch.full((1, 8), -1, **I32)
    r = fovea.cache_fork(k_pages, v_pages, empty, ints([0]), ints([-1, -1, -1]), None, ints([n + nodes for n in lens]))
    table = r["table"]
    assert r["free"].tolist() == [n_pages - 3 - 1 - 2]

    def add(table, counts, starts):
        sequence = torch.cat([torch.full((c,), b, **I32) for b, c in enumerate(counts)])
        entry = torch.cat([torch.arange(s, s + c, **I32) for s, c in zip(starts, counts)])
        n = sequence.numel()
        x = normal(g, n, heads + 2 * kv, dim).to(dt)
        positions = torch.randint(0, 500, (3, n), generator=g, **I32)
        return fovea.cache_append(x[:, heads:heads + kv], x[:, heads + kv:], k_pages, v_pages, table, sequence, entry,
                                  q=x[:, :heads], positions=positions, frequencies=f, axis=axis, **scales)

    add(table, lens, [0, 0, 0])
    q = add(table, [nodes] * 3, lens)
    held = ints([n + nodes for n in lens])
    tree = tree_bits(g, 3, nodes)
    check_attention(fovea, q, k_pages, v_pages, table, held, tree, scales=scales)
    rows = [entries(v_pages, table, b, n + nodes).clone() for b, n in enumerate(lens)]
    path = ints([[0, 2, 7], [0, -1, -1], [0, 11, -1]])
    held = fovea.cache_keep(k_pages, v_pages, table, held, path, nodes)
    assert held.tolist() == [36, 2, 22]
    for b, n in enumerate(lens):
        p = [x for x in path[b].tolist() if x >= 0]
        want = torch.cat((rows[b][:n].view(-1, kv, dim).float(), rows[b].float()[[n + x for x in p]]))
        assert torch.equal(entries(v_pages, table, b, n + len(p)).float(), want)
    r = fovea.cache_fork(k_pages, v_pages, table, held, ints([0, 0, 2, 2]), ints([36, 35, 22, 22]), ints([1, 1, 1, 1]))
    assert r["lens"].tolist() == [36, 35, 22, 22] and int(r["free"]) > 0
    for c, b in enumerate([0, 0, 2, 2]):
        n = int(r["lens"][c])
        assert same(entries(k_pages, r["table"], c, n), entries(k_pages, table, b, n))
    q = add(r["table"], [1] * 4, r["lens"].tolist())
    check_attention(fovea, q, k_pages, v_pages, r["table"], r["lens"] + 1, scales=scales)


def test_other_stream_and_graph(fovea):
    """A side stream; a step captured into a graph and replayed on new contents."""
    g = gen(12)
    lens = [300, 40]
    k, v, table, _ = make_cache(g, BF16, lens, 4, 128, 16)
    f, axis = fovea.rotary_frequencies(128, [16, 24, 24])
    x = normal(g, 2, 36, 128).to(BF16)
    q, nk, nv = x[:, :28], x[:, 28:32], x[:, 32:]
    sequence, entry, positions = ints([0, 1]), ints([299, 39]), ints([[299, 39]] * 3)
    held = ints(lens)
    ws = torch.empty(fovea.paged_attention_workspace_size(2, 1, 28, 4, 128), dtype=torch.uint8, device="cuda")

    def step(stream=None):
        y = fovea.cache_append(nk, nv, k, v, table, sequence, entry, q=q, positions=positions, frequencies=f,
                               axis=axis, stream=stream)
        a = fovea.paged_attention(y, k, v, table, held, want_lse=True, workspace=ws, stream=stream)
        b = fovea.cache_keep(k, v, table, held, path, 1, stream=stream)
        c = fovea.cache_fork(k, v, table, b, parents, stream=stream)
        return [y, a["out"], a["lse"], b, c["table"], c["lens"], c["free"]]

    path, parents = ints([[0], [0]]), ints([1, 0])
    want = step()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = step(side)
    torch.cuda.synchronize()
    assert all(same(a, b) for a, b in zip(got, want))
    ws.fill_(255)                                   # whatever the memory holds
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        held_out = step(torch.cuda.current_stream())
    for shift in (0, 1):
        x.copy_(normal(gen(50 + shift), 2, 36, 128))
        held.copy_(ints([300 - shift, 40 - 39 * shift]))
        entry.copy_(held - 1)
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in held_out]
        want = step()
        torch.cuda.synchronize()
        assert all(same(a, b) for a, b in zip(got, want))


def test_workspaces_of_two_streams(fovea):
    """Calls on two streams, each with a workspace of its own, at the same time."""
    g = gen(13)
    k, v, table, _ = make_cache(g, BF16, [4000, 3000], 2, 128, 64)
    qs = [normal(g, 2, 8, 128).to(BF16) for _ in range(2)]
    lens = ints([4000, 3000])
    want = [fovea.paged_attention(q, k, v, table, lens)["out"] for q in qs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in qs]
    got = []
    for _ in range(20):
        for q, s in zip(qs, streams):
            got.append(fovea.paged_attention(q, k, v, table, lens, stream=s)["out"])
    torch.cuda.synchronize()
    assert all(same(a, want[i % 2]) for i, a in enumerate(got))


def test_empty_calls(fovea):
    g = gen(14)
    k, v, table, _ = make_cache(g, BF16, [5], 1, 64, 16)
    none = torch.empty(0, 1, 64, dtype=BF16, device="cuda")
    f, axis = fovea.rotary_frequencies(64)
    q, _ = fovea.rotary_axes(none, none, torch.empty(1, 0, **I32), f, axis)
    assert q.shape == none.shape
    assert fovea.cache_append(none, none, k, v, table, torch.empty(0, **I32), torch.empty(0, **I32)) is None
    no_table = torch.empty(0, 3, **I32)
    assert fovea.paged_attention(none, k, v, no_table, torch.empty(0, **I32))["out"].shape == none.shape
    assert fovea.cache_keep(k, v, no_table, torch.empty(0, **I32), torch.empty(0, 2, **I32), 4).numel() == 0
    assert fovea.cache_fork(k, v, no_table, torch.empty(0, **I32), torch.empty(0, **I32))["free"].tolist() == [4]
    got = fovea.cache_fork(k, v, no_table, torch.empty(0, **I32), ints([0, -1]), None, ints([17, 16]))
    assert got["table"].tolist() == [[0, 1, -1], [2, -1, -1]]
    assert got["lens"].tolist() == [0, 0] and got["free"].tolist() == [1]


def test_refusals_of_the_binding(fovea):
    g = gen(15)
    k, v, table, _ = make_cache(g, BF16, [5], 2, 64, 16)
    q, lens = normal(g, 1, 4, 64).to(BF16), ints([5])
    f, axis = fovea.rotary_frequencies(64)
    pos = ints([[3]])
    ok = dict(q=q, k_pages=k, v_pages=v, table=table, lens=lens)
    for bad in (dict(q=q.float()), dict(q=q[:, :3]), dict(q=q[..., :32]), dict(q=q.cpu()), dict(v_pages=v[:, :1]),
                dict(v_pages=v.float()), dict(table=table.long()), dict(lens=lens.long()), dict(lens=ints([5, 5])),
                dict(k_pages=k.transpose(0, 1)), dict(tree=ints([[1]])), dict(tree=ints([[[1]], [[1]]])),
                dict(k_scale=torch.ones(2, device="cuda")), dict(workspace=torch.empty(256, dtype=torch.uint8)),
                dict(q=torch.cat((q, q))[:, :, ::2])):
        with pytest.raises(ValueError):
            fovea.paged_attention(**{**ok, **bad})
    with pytest.raises(fovea.FoveaError):
        fovea.paged_attention(**ok, workspace=torch.empty(256, dtype=torch.uint8, device="cuda"))
    with pytest.raises(fovea.FoveaError):
        fovea.paged_attention(**ok, scale=float("nan"))
    for args, kw in (((q, None, pos.long(), f), {}), ((q, None, ints([[3, 4]]), f), {}), ((q, None, pos, f.float()), {}),
                     ((q, None, pos, f, axis[:3]), {}), ((q, q.float(), pos, f), {}), ((q[0], None, pos, f), {})):
        with pytest.raises(ValueError):
            fovea.rotary_axes(*args, **kw)
    with pytest.raises(fovea.FoveaError):
        fovea.rotary_axes(q, None, pos, torch.ones(33, dtype=torch.float64, device="cuda"))
    nk, at = normal(g, 1, 2, 64).to(BF16), ints([0])
    for kw in (dict(q=q), dict(positions=pos), dict(frequencies=f), dict(axis=axis),
               dict(k_scale=torch.ones(2, device="cuda")), dict(q=q.float(), positions=pos, frequencies=f)):
        with pytest.raises(ValueError):
            fovea.cache_append(nk, nk, k, v, table, at, at, **kw)
    with pytest.raises(ValueError):
        fovea.cache_append(nk[:, :1], nk[:, :1], k, v, table, at, at)
    with pytest.raises(fovea.FoveaError):
        fovea.cache_append(nk.float(), nk.float(), k, v, table, at, at)
    for bad in (dict(nodes=ints([[0, 1]]), size=1), dict(nodes=ints([[0]]), size=257)):
        with pytest.raises(fovea.FoveaError):
            fovea.cache_keep(k, v, table, lens, **bad)
    with pytest.raises(ValueError):
        fovea.cache_keep(k.cpu(), v, table, lens, ints([[0]]), 1)
    with pytest.raises(ValueError):
        fovea.cache_fork(k, v, table, lens, ints([0]), ints([0, 1]))
    with pytest.raises(ValueError):
        fovea.cache_fork(k, v, table, lens, ints([0]), width=0)
    with pytest.raises(ValueError):
        fovea.rotary_frequencies(16, [3, 4])


def test_a_wait_that_gives_up(fovea):
    """Trees through the tensor cores with waits that give up: NaN, an error for the
    workspace, and the next call on it as ever."""
    g = gen(16)
    for cache in (BF16, E4M3):
        lens = [900, 400]
        k, v, table, scales = make_cache(g, cache, lens, 4, 128, 64)
        q = normal(g, 2 * 64, 8, 128).to(BF16)
        ws = torch.full((fovea.paged_attention_workspace_size(2, 64, 8, 4, 128, cache),), 255, dtype=torch.uint8,
                        device="cuda")
        args = (q, k, v, table, ints(lens))
        want = fovea.paged_attention(*args, workspace=ws, want_lse=True, **scales)
        fovea.sync_errors(ws)
        fovea.debug_wait_limit(1)
        try:
            got = fovea.paged_attention(*args, workspace=ws, want_lse=True, **scales)
            torch.cuda.synchronize()
        finally:
            fovea.debug_wait_limit(0)
        assert torch.isnan(got["out"]).any() and torch.isnan(got["lse"]).any()
        again = fovea.paged_attention(*args, workspace=ws, want_lse=True, **scales)
        with pytest.raises(fovea.FoveaError) as e:
            fovea.sync_errors(ws)
        assert e.value.status == fovea.ERR_TIMEOUT
        fovea.sync_errors(ws)
        assert same(again["out"], want["out"]) and same(again["lse"], want["lse"])
