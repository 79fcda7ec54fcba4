"""Edges of the drafter's cache that random rows do not reach: the bits of
probabilities, values that are no numbers in front of a tree, long paths, far and
small angles, outputs in the inputs' place, scales and rows at the ends of their range."""

import math

import pytest
import torch

from test_cache_operators_gpu import (BF16, E4M3, FP32, I32, U, check_attention, entries, fovea,  # noqa: F401
                                      gen, ints, make_cache, normal, same, tree_bits, within)

pytestmark = pytest.mark.gpu

# (cache, nodes, heads, key heads, dim): each form of the attention, by rows of a key head
FORMS = [
    (BF16, 1, 6, 2, 64), (BF16, 6, 4, 2, 128), (BF16, 3, 8, 2, 256),                      # few rows
    (BF16, 7, 8, 2, 256),                                                                 # staged tiles
    (BF16, 32, 8, 2, 128), (BF16, 20, 2, 1, 64), (BF16, 160, 2, 2, 128),                  # tensor memory
    (FP32, 1, 4, 2, 128), (FP32, 6, 4, 2, 64), (FP32, 9, 4, 2, 256),
    (E4M3, 1, 4, 2, 256), (E4M3, 1, 8, 2, 128), (E4M3, 2, 4, 2, 64),                      # four rows and fewer
    (E4M3, 6, 4, 2, 64), (E4M3, 6, 4, 2, 128),
    (E4M3, 6, 8, 2, 128), (E4M3, 9, 4, 2, 64), (E4M3, 7, 8, 2, 256),
    (E4M3, 32, 8, 2, 128), (E4M3, 70, 2, 2, 64), (E4M3, 160, 2, 2, 128),
]


def rows_type(cache):
    return FP32 if cache is FP32 else BF16


def put(pool, table, b, e, dims, value):
    """value at entry e of sequence b, in these dims of all heads."""
    page = pool.shape[2]
    pool[int(table[b, e // page]), :, e % page, dims] = torch.tensor(value).to(pool.dtype).cuda()


# ---------------------------------------------------------------------------
# The bits of p
# ---------------------------------------------------------------------------

def cancelling():
    """(a, b) in 4 significant bits with a as near to b e^(i / 8) as there are, for i = 1 .. 15."""
    found = []
    for i in range(1, 16):
        r = math.exp(i / 8)
        pairs = [(x * 2.0 ** s, float(y)) for x in range(8, 16) for y in range(8, 16) for s in range(4)]
        found.append(min(pairs, key=lambda p: abs(p[0] / p[1] - r)))
    return found


@pytest.mark.parametrize("cache,nodes,heads,kv,dim", [f for f in FORMS if f[0] is E4M3])
def test_values_that_cancel(fovea, cache, nodes, heads, kv, dim):
    """Sixteen entries in front of a tree that is not seen, with exact scores 0, 1/8, ..., 15/8, and in
    each dim two values whose products with p nearly cancel: what is left shows p's roundings."""
    n = 16 + nodes
    k, v, table, _ = make_cache(gen(1), cache, [n, n], kv, dim, 16)
    for b in range(2):
        for e in range(16):
            put(k, table, b, e, slice(None), 0.0)
            put(k, table, b, e, 0, e / 8)
            put(v, table, b, e, slice(None), 0.0)
        for d, (x, y) in zip(range(dim), cancelling() * dim):
            put(v, table, b, 0, d, -x)
            put(v, table, b, 1 + d % 15, d, y)
    q = torch.zeros(2 * nodes, heads, dim, dtype=BF16, device="cuda")
    q[..., 0] = 1.0
    got = fovea.paged_attention(q, k, v, table, ints([n, n]), tree=torch.zeros(1, nodes, -(-nodes // 32), **I32), scale=1.0)
    z = torch.arange(16, dtype=torch.float64, device="cuda") / 8
    p = torch.softmax(z, 0)
    x = entries(v, table, 0, 16)[:, 0].double()
    want, size = p @ x, p @ x.abs()
    assert bool((want.abs() < size / 100).all())
    # Of an element of p: 22 bits in its product (2^-22), its score times log2 e in two roundings
    # (2 * 15/8 u) and the exponential's 2^-22; of the sums: a block's truncated addition to 2^-23
    # of its magnitudes and the joins of eight parts (8 * 2^-23); the last rounding.
    bound = want.abs() * 2.0 ** -9 * 2 + size * (2 * 2.0 ** -22 + 4 * U + 9 * 2.0 ** -23)
    out = got["out"].double()
    within(out, want.expand_as(out), bound, "cancelling values")


# ---------------------------------------------------------------------------
# Paths of every length
# ---------------------------------------------------------------------------

@pytest.mark.parametrize("cache,dim", [(BF16, 64), (BF16, 128), (BF16, 256), (FP32, 64), (FP32, 128), (FP32, 256),
                                       (E4M3, 64), (E4M3, 256)])
def test_paths_of_every_length(fovea, cache, dim):
    """The staging of a path takes what shared memory is left beside the places of its entries."""
    g = gen(dim)
    size, page, n = 256, 64, 300
    k, v, table, _ = make_cache(g, cache, [n], 1, dim, page)
    before = [entries(x, table, 0, n).clone() for x in (k, v)]
    stored = [x.clone() for x in (k, v)]
    for path in list(range(1, 257, 5)) + [43, 44, 45, 48, 49, 88, 89, 96, 97, 176, 177, 192, 193, 255, 256]:
        for pool, old in zip((k, v), stored):
            pool.copy_(old)
        nodes = torch.randint(0, size, (1, path), generator=g, **I32)
        got = fovea.cache_keep(k, v, table, ints([n]), nodes, size)
        assert got.tolist() == [n - size + path]
        for pool, old in zip((k, v), before):
            kept = entries(pool, table, 0, n - size + path)
            assert same(kept[:n - size], old[:n - size]) and same(kept[n - size:], old[n - size + nodes[0].long()]), path


# ---------------------------------------------------------------------------
# Values that are no numbers
# ---------------------------------------------------------------------------

def spoiled(fovea, form, lens, marks, seed=3):
    """The attention with values marked in front of (entry negative: from the tree's first on
    backwards) or within the trees: marks (sequence, entry from the tree's first, first dim, value)."""
    cache, nodes, heads, kv, dim = form
    g = gen(seed)
    k, v, table, scales = make_cache(g, cache, lens, kv, dim, 16)
    for b, at, d, value in marks:
        if 0 <= lens[b] - nodes + at < lens[b]:
            put(v, table, b, lens[b] - nodes + at, slice(d, None, 8), value)
    q = normal(g, len(lens) * nodes, heads, dim).to(rows_type(cache))
    for tree in (None, tree_bits(g, len(lens), nodes), tree_bits(g, 1, nodes)):
        check_attention(fovea, q, k, v, table, ints(lens), tree, scales=scales)


def spots(nodes, n):
    """In front of a tree of a sequence of n entries: its last, and the first of the blocks of 16, 32
    and 64 in which the tree begins."""
    at = n - nodes
    return sorted({-1} | {at // size * size - at for size in (16, 32, 64) if at % size})


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("more", [39, 700, 61])
def test_nan_in_front_of_a_tree(fovea, form, more):
    """Every row sees the entries in front of a tree, those that share a tile with it too."""
    nodes = form[1]
    lens = [nodes + more, nodes + 2 * more + 1, nodes + 5]
    marks = [(b, at, i % 8, float("nan")) for b in (0, 1) for i, at in enumerate(spots(nodes, lens[b]))]
    spoiled(fovea, form, lens, marks)


@pytest.mark.parametrize("form", [f for f in FORMS if f[1] > 1])
def test_nan_at_a_node(fovea, form):
    """A node's value reaches the rows that see it, in every form."""
    nodes = form[1]
    lens = [nodes + 39, nodes, nodes + 900]
    spoiled(fovea, form, lens, [(b, (3 * b + 2) % nodes, b, float("nan")) for b in range(3)] + [(2, nodes - 1, 5, float("nan"))])


@pytest.mark.parametrize("form", [f for f in FORMS if f[0] is not E4M3])
@pytest.mark.parametrize("more", [39, 700, 3000])
def test_infinite_values(fovea, form, more):
    """An infinite value makes its dim infinite in the rows that see it, wherever it stands; with
    one of the other sign, or with a NaN, there is no number."""
    nodes, inf = form[1], math.inf
    lens = [nodes + more, nodes + more // 2, nodes + 5]
    marks = []
    for b in (0, 1):
        at = spots(nodes, lens[b])
        marks += [(b, at[0], 0, inf), (b, at[-1], 1, -inf),
                  (b, nodes - lens[b], 2, inf), (b, -more // 3, 3, -inf),             # first, and far in front
                  (b, -1, 4, inf), (b, 0, 4, inf),                                    # in both places
                  (b, -more // 4, 5, inf), (b, -2, 5, -inf),                          # of both signs
                  (b, -more // 4, 6, inf), (b, nodes - 1, 6, -inf),                   # the other at a node
                  (b, 0, 7, -inf), (b, nodes - lens[b], 7, float("nan"))]
    spoiled(fovea, form, lens, marks)


@pytest.mark.parametrize("form", FORMS)
def test_rows_without_numbers_stay_so(fovea, form):
    """A row whose scores are no numbers has none in any dim, with infinite values or without."""
    cache, nodes, heads, kv, dim = form
    g = gen(6)
    lens = [nodes + 70, nodes + 700]
    k, v, table, scales = make_cache(g, cache, lens, kv, dim, 16)
    for b in range(2):
        put(k, table, b, 20, 3, float("nan"))
        put(v, table, b, 30, slice(0, None, 2), float("nan") if cache is E4M3 else math.inf)
    q = normal(g, 2 * nodes, heads, dim).to(rows_type(cache))
    q[0] = 0
    got = fovea.paged_attention(q, k, v, table, ints(lens), want_lse=True, **scales)
    assert bool(torch.isnan(got["out"]).all()) and bool(torch.isnan(got["lse"]).all())
    # a page that is not there, and a length beyond the table
    k, v, table, scales = make_cache(g, cache, lens, kv, dim, 16)
    for b in range(2):
        put(v, table, b, 30, slice(0, None, 2), float("nan") if cache is E4M3 else math.inf)
    table[0, 0] = -1
    lens[1] = table.shape[1] * 16 + 1
    got = fovea.paged_attention(q, k, v, table, ints(lens), want_lse=True, **scales)
    assert bool(torch.isnan(got["out"]).all()) and bool(torch.isnan(got["lse"]).all())


# ---------------------------------------------------------------------------
# Angles
# ---------------------------------------------------------------------------

def turned(fovea, frequencies, at):
    """(cos, sin) [positions, frequencies] as the operator has them, and the angles' own in 64 bits."""
    from fractions import Fraction
    half = len(frequencies)
    q = torch.zeros(len(at), 1, 2 * half, device="cuda")
    q[..., :half] = 1.0
    got, _ = fovea.rotary_axes(q, None, ints([at]), torch.tensor(frequencies, dtype=torch.float64, device="cuda"))
    turn = Fraction(int("6283185307179586476925286766559005768394338798750211641949889184615632812572417997256069650684234135"),
                    10 ** 99)
    want = torch.empty(2, len(at), half, dtype=torch.float64)
    for n, p in enumerate(at):
        for j, w in enumerate(frequencies):
            x = Fraction(w) * p / turn
            x -= round(x)                          # within half a turn, exactly
            want[0, n, j], want[1, n, j] = math.cos(float(x * turn)), math.sin(float(x * turn))
    got = got[:, 0].double().cpu()
    return torch.stack((got[:, :half], got[:, half:])), want


def test_far_angles_of_fast_pairs(fovea):
    """The angle's error does not grow with the position or the frequency."""
    w = [0.92, 2.5, 100.0, 1e4, 12345.678, 2.0 ** 20 + 1 / 3, 1e9, 2.0 ** 40 - 1 / 7]
    got, want = turned(fovea, w, [2139596203, 2 ** 31 - 1, -2 ** 31, 1999999973, 1, 77])
    # the rest of an angle, up to pi / 4, in three roundings (2.4 u); the series' last two
    # steps (1.5 u); the fixed point's 2^-33 and the product's lower part (below u / 16)
    assert float((got - want).abs().max()) <= 4 * U


def test_small_angles(fovea):
    """The sine of a small angle keeps its bits, which a pair with one half zero shows."""
    w = [1e-6, 3e-5, 1e-8, 1e-10, 7.7e-4, 0.01]
    got, want = turned(fovea, w, [1, 7, -3, 1000, -12345])
    # the angle in three roundings, the series in three, the product in one; 2^-64 of a turn
    # beside the frequency's 1e-10 / 2 pi (2^-30)
    assert float(((got - want).abs() / want.abs())[1].max()) <= 8 * U
    assert float((got - want).abs()[0].max()) <= 4 * U


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("adjacent", [0, 1])
@pytest.mark.parametrize("n,heads,kv,dim,rot", [(1, 4, 1, 128, 128), (300, 28, 4, 128, 96), (1000, 40, 40, 64, 64), (33, 3, 2, 81, 34)])
def test_rotated_in_place(fovea, dtype, adjacent, n, heads, kv, dim, rot):
    """The outputs may be the inputs' own memory (at the C entry)."""
    g = gen(n)
    q, k, v = (normal(g, n, h, dim).to(dtype) for h in (heads, kv, kv))
    f, axis = fovea.rotary_frequencies(rot, [rot // 4, rot // 2 - rot // 4])
    positions = torch.randint(0, 5000, (2, n), generator=g, **I32)
    want = fovea.rotary_axes(q, k, positions, f, axis, adjacent=bool(adjacent))
    kind = fovea.BF16 if dtype is BF16 else fovea.FP32
    stream = torch.cuda.current_stream().cuda_stream
    turns = (positions.data_ptr(), n, 2, f.data_ptr(), axis.data_ptr(), rot, adjacent)
    x, y = q.clone(), k.clone()
    assert fovea.lib().fovea_rotary_axes(x.data_ptr(), heads * dim, dim, heads, y.data_ptr(), kv * dim, dim, kv, n, dim, kind,
                                         *turns, 0, x.data_ptr(), y.data_ptr(), stream) == 0
    assert same(x, want[0]) and same(y, want[1])
    if dim not in (64, 128):
        return
    pages, table = torch.empty(2, n // 16 + 1, kv, 16, dim, dtype=dtype, device="cuda"), torch.arange(n // 16 + 1, **I32)[None]
    x, sequence, entry = q.clone(), torch.zeros(n, **I32), torch.arange(n, **I32)
    assert fovea.lib().fovea_cache_append(x.data_ptr(), heads * dim, dim, heads, k.data_ptr(), kv * dim, dim, v.data_ptr(),
                                          kv * dim, dim, n, kind, *turns, x.data_ptr(), pages[0].data_ptr(),
                                          pages[1].data_ptr(), kind, None, None, n // 16 + 1, 16, kv, dim, table.data_ptr(),
                                          1, n // 16 + 1, sequence.data_ptr(), entry.data_ptr(), stream) == 0
    assert same(x, want[0]) and same(entries(pages[0], table, 0, n), want[1]) and same(entries(pages[1], table, 0, n), v)


# ---------------------------------------------------------------------------
# Scales and rows at the ends of their range
# ---------------------------------------------------------------------------

def as_entries(x, scale):
    """x / scale in 8 bits, by one division in 32 bits."""
    y = (x.double() / scale.double()[:, None]).float()
    return y.clamp(-448, 448).to(E4M3)


@pytest.mark.parametrize("rotate", [False, True])
def test_entries_next_to_a_border(fovea, rotate):
    """Scales that bring x next to the middle of two 8-bit values: the quotient is rounded once."""
    g = gen(2)
    kv, dim = 400, 64
    x = normal(g, 1, kv, 1).to(BF16)
    middle = (torch.randint(8, 16, (kv,), generator=g, device="cuda") + 0.5) * 2.0 ** torch.randint(-4, 4, (kv,), generator=g, device="cuda")
    scale = (x[0, :, 0].double().abs() / middle.double()).float()
    scale[:3] = torch.tensor([1e-39, 3e38, 2.0 ** -149], device="cuda")           # no reciprocal, or a rounded one
    x[0, :3, 0] = torch.tensor([1e-38, 3e38, 0.0], device="cuda").to(BF16)
    x = x.expand(1, kv, dim).contiguous()
    k_pages, v_pages = (torch.zeros(1, kv, 16, dim, device="cuda").to(E4M3) for _ in range(2))
    more = {}
    if rotate:                                     # by nothing
        f, _ = fovea.rotary_frequencies(dim)
        more = dict(positions=ints([[0]]), frequencies=f)
    fovea.cache_append(x, x, k_pages, v_pages, ints([[0]]), ints([0]), ints([5]), k_scale=scale, v_scale=scale, **more)
    want = as_entries(x[0], scale)
    for pool in (k_pages, v_pages):
        assert same(pool[0, :, 5], want)


def test_entries_of_odd_quotients(fovea):
    """Zeros, infinities, numbers that are none, under scales of both signs and of all sizes."""
    x = torch.tensor([0.0, -0.0, 1.0, -2.5, 1e-40, -1e-38, 3e38, -3e38, math.inf, -math.inf, math.nan, 448, 300, 1e-3, 2e-3, 5e-3],
                     device="cuda").to(BF16)
    scale = torch.tensor([1.0, -1.0, 3e-3, 1e-39, -1e-30, 2.0 ** -60, 1e-12, 1e12, 2.0 ** 41, 1e30, -3e38, math.inf, math.nan],
                         device="cuda")
    kv, dim = scale.numel(), 64
    x = x.repeat(4)[None, None].expand(1, kv, dim).contiguous()
    pages = [torch.zeros(1, kv, 16, dim, device="cuda").to(E4M3) for _ in range(2)]
    fovea.cache_append(x, x, *pages, ints([[0]]), ints([0]), ints([0]), k_scale=scale, v_scale=scale)
    want = as_entries(x[0], scale).float()
    want[11, 8:10] = want[11, 24:26] = want[11, 40:42] = want[11, 56:58] = 0       # of two infinities: not asked
    for pool in pages:
        got = pool[0, :, 0].float()
        got[11, 8:10] = got[11, 24:26] = got[11, 40:42] = got[11, 56:58] = 0
        assert torch.equal(torch.isnan(got), torch.isnan(want)) and torch.equal(got.nan_to_num(0), want.nan_to_num(0))


@pytest.mark.parametrize("form", [f for f in FORMS if f[0] is E4M3])
@pytest.mark.parametrize("power,scale,k_scale", [(127, 2.0 ** -120, 2.0 ** -9), (126, 2.0 ** -120, 2.0 ** -8),
                                                 (-126, 2.0 ** 26, 2.0 ** 98), (-131, 2.0 ** 26, 2.0 ** 101)])
def test_rows_at_the_ends_of_their_range(fovea, form, power, scale, k_scale):
    """Rows of q beside 8-bit keys are brought to fp16's range, from bf16's largest and smallest."""
    cache, nodes, heads, kv, dim = form
    g = gen(power + 200)
    lens = [nodes + 40, nodes + 300]
    k, v, table, scales = make_cache(g, cache, lens, kv, dim, 16)
    k.copy_((k.float() / 64).to(E4M3))
    scales["k_scale"] = torch.full((kv,), k_scale, device="cuda")
    q = normal(g, 2 * nodes, heads, dim).sign() * (1 + torch.randint(0, 4, (2 * nodes, heads, dim), generator=g, device="cuda") / 4)
    q = (q.double() * 2.0 ** power).to(BF16)
    assert bool(torch.isfinite(q).all()) and float((q == 0).float().mean()) < 1e-3
    check_attention(fovea, q, k, v, table, ints(lens), scale=scale, scales=scales)


# ---------------------------------------------------------------------------
# Products of an fp32 cache
# ---------------------------------------------------------------------------

@pytest.mark.parametrize("dim", [64, 128, 256])
def test_bits_of_fp32_products(fovea, dim):
    """One entry a sequence: the score is one product, the output its value."""
    g = gen(dim)
    B, kv = 500, 8
    k_pages, v_pages = (torch.zeros(B, kv, 16, dim, device="cuda") for _ in range(2))
    k, v, q = (normal(g, B, kv, n).exp() for n in (1, dim, 1))
    v[0, 0, :2] = torch.tensor([3.4028e38, -3.4028e38], device="cuda")             # rounded up, they would be infinite
    k_pages[:, :, 0, :1], v_pages[:, :, 0] = k, v
    rows = torch.zeros(B, kv, dim, device="cuda")
    rows[..., :1] = q
    got = fovea.paged_attention(rows, k_pages, v_pages, torch.arange(B, **I32)[:, None].contiguous(), torch.ones(B, **I32),
                                scale=1.0, want_lse=True)
    # a factor is its upper 11 bits and 11 of the others, off by 2^-21; the product of both
    # lower parts (2^-10 each) is left out: 2 * 2^-21 + 2^-20; sums that truncate to 2^-23 (two),
    # roundings of the score by log2 e, of the factor and of the way back (four).  p is 1, exactly.
    want = q.double()[..., 0] * k.double()[..., 0]
    within(got["lse"], want, want * (2.0 ** -19 + 2 * 2.0 ** -23 + 4 * U), "score")
    within(got["out"], v.double(), v.double().abs() * (2.0 ** -21 + 2 * 2.0 ** -23 + U), "value")


def test_stored_zeros_keep_their_sign(fovea):
    x = torch.tensor([0.0, -0.0, -1e-30, 1e-30], device="cuda").to(BF16).repeat(16)[None, None]
    pages = [torch.ones(1, 1, 16, 64, device="cuda").to(E4M3) for _ in range(2)]
    for s in (0.3, 1e-45, 1e20):
        scale = torch.tensor([s], device="cuda")
        fovea.cache_append(x, x, *pages, ints([[0]]), ints([0]), ints([0]), k_scale=scale, v_scale=scale)
        for pool in pages:
            assert pool[0, 0, 0].view(torch.uint8)[:2].tolist() == [0, 128]
            assert same(pool[0, :, 0], as_entries(x[0], scale))
