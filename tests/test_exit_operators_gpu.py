"""The operators of the drafter's exit (add_rms_norm, quantize_w4, linear_w4,
token_logprobs and its gradient) against their definitions in 64 bits.

Bounds count fp32 roundings (u = 2^-24 each): of a row's or a group's sums, of
the operations on one element, and of the last rounding to the stored type."""

import math

import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
BF16, FP32, E4M3 = torch.bfloat16, torch.float32, torch.float8_e4m3fn
HALF_ULP = {BF16: 2.0 ** -8, FP32: U}      # of 8 and of 24 significant bits


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


def within(got, want, bound, what=""):
    """|got - want| <= bound element by element; equal where want is not finite."""
    got, want = got.double(), want.double()
    fine = torch.isfinite(want)
    assert torch.equal(torch.isnan(got), torch.isnan(want)), what
    assert torch.equal(got[~fine & ~torch.isnan(want)], want[~fine & ~torch.isnan(want)]), what
    err, b = (got - want).abs()[fine], torch.broadcast_to(bound, want.shape)[fine]
    assert bool((err <= b).all()), f"{what}: {float((err / b.clamp(min=1e-300)).max()):.3g} of the bound"


# ---------------------------------------------------------------------------
# add_rms_norm
# ---------------------------------------------------------------------------

def norm_reference(x, r, gamma, eps):
    s = (x.float() + r.float()) if r is not None else x.float()
    v = s.double()
    return s, v / torch.sqrt((v * v).mean(1, keepdim=True) + eps) * gamma.double()


def check_norm(fovea, x, r, gamma, q8_group, eps=1e-6, want_out=True, stream=None):
    got = fovea.add_rms_norm(x, gamma, r, eps=eps, want_out=want_out, q8_group=q8_group, stream=stream)
    torch.cuda.synchronize()
    n, d = x.shape
    s, y = norm_reference(x, r, gamma, eps)
    # a thread's chain of at most 16 squares and ten levels of the tree, halved by
    # the root, then two products; generously 40 roundings
    rel = 40 * U
    if r is None:
        assert got["sum"] is None
    else:
        assert torch.equal(got["sum"], s.to(x.dtype))
    if want_out:
        within(got["out"], y, y.abs() * (HALF_ULP[x.dtype] + rel) + 1e-38, "out")
    else:
        assert got["out"] is None
    if q8_group is None:
        assert "q8" not in got
        return got
    width = q8_group or d
    pad = torch.nn.functional.pad(y, (0, -(-d // width) * width - d)).view(n, -1, width)
    scale = pad.abs().amax(2) / 448
    assert got["q8_scale"].shape == ((n, scale.shape[1]) if q8_group else (n,))
    within(got["q8_scale"].view(n, -1), scale, scale * rel + 1e-45, "q8_scale")
    full = got["q8_scale"].double().view(n, -1).repeat_interleave(width, 1)[:, :d]
    # e4m3 keeps four significant bits: half a step is 2^-4 of the value, 2^-10 below the normal ones
    within(got["q8"].double() * full, y, y.abs() * (2.0 ** -4 + 2 * rel) + full * 2.0 ** -10 * (1 + rel), "q8")
    return got


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("n,d,pad,q8", [
    (1, 4096, 0, 0), (3, 1, 0, 0), (5, 7, 0, 32), (2, 127, 3, 64), (130, 256, 8, 128), (1, 8192, 0, 128),
    (9, 8191, 1, 0), (700, 3584, 0, 64), (2500, 320, 0, 32), (4, 1032, 8, 128), (33, 100, 4, None),
])
def test_norm(fovea, dtype, n, d, pad, q8):
    g = gen(d)
    x = torch.empty((n, d + pad), device="cuda", dtype=dtype)[:, :d]
    x.copy_(torch.randn((n, d), generator=g, device="cuda"))
    r = (3 * torch.randn((n, d), generator=g, device="cuda")).to(dtype)
    gamma = (1 + 0.1 * torch.randn(d, generator=g, device="cuda")).to(dtype)
    check_norm(fovea, x, r, gamma, q8)
    check_norm(fovea, x, None, gamma, q8, want_out=q8 is None)


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("d", [1, 5, 9, 255, 1003, 2050, 4103, 8189])
def test_norm_rows_anywhere(fovea, dtype, d):
    """Every offset from the vectors' boundary, of the inputs (residual and gamma at
    other offsets) and of the outputs; the sum in x's place; nothing outside written."""
    n, size = 5, 2 if dtype is BF16 else 4
    g = gen(d)
    eight = d % 2 == 1
    for off in range(16 // size):
        def rows(at, v=None):
            b = torch.full((n * d + 64,), 7.0, device="cuda", dtype=dtype)
            if v is not None:
                b[at:at + n * d] = v.flatten()
            return b, b[at:at + n * d].view(n, d)
        v = torch.randn((n, d), generator=g, device="cuda").to(dtype)
        w = torch.randn((n, d), generator=g, device="cuda").to(dtype)
        xb, x = rows(16 + off, v)
        rb, r = rows(16 + 3 * off % 8, w)
        ob, out = rows(16 + 5 * off % 8)
        gamma = torch.ones(d + 8, device="cuda", dtype=dtype)[off % 8:off % 8 + d]
        gamma.copy_(1 + 0.1 * torch.randn(d, generator=g, device="cuda"))
        q8b = torch.full((n * d + 64,), 99, device="cuda", dtype=torch.uint8)
        scale = torch.empty((n,), device="cuda")
        s, y = norm_reference(v, w, gamma, 1e-6)
        st = fovea.lib().fovea_add_rms_norm(
            x.data_ptr(), d, r.data_ptr(), d, gamma.data_ptr(), n, d, fovea._DTYPES[dtype], 1e-6, x.data_ptr(),
            out.data_ptr(), q8b.data_ptr() + 16 + off if eight else None, scale.data_ptr() if eight else None, 0,
            torch.cuda.current_stream().cuda_stream)
        assert st == 0
        torch.cuda.synchronize()
        assert torch.equal(x, s.to(dtype)) and torch.equal(r, w)
        within(out, y, y.abs() * (HALF_ULP[dtype] + 40 * U) + 1e-38, "out")
        for b, at in ((xb, 16 + off), (rb, 16 + 3 * off % 8), (ob, 16 + 5 * off % 8)):
            assert bool((b[:at] == 7).all()) and bool((b[at + n * d:] == 7).all())
        if eight:
            at = 16 + off
            assert bool((q8b[:at] == 99).all()) and bool((q8b[at + n * d:] == 99).all())
            q = q8b[at:at + n * d].view(E4M3).view(n, d).double() * scale.double()[:, None]
            within(q, y, y.abs() * (2.0 ** -4 + 80 * U) + scale.double()[:, None] * 2.0 ** -10 * (1 + 40 * U), "q8")


def test_norm_rows_without_size(fovea):
    # zeros, a group of zeros, the smallest and the largest values
    x = torch.zeros((4, 256), device="cuda")
    x[1, 128:] = 1.0
    x[2] = 1e-30
    x[3] = 1e15
    gamma = torch.ones(256, device="cuda")
    got = check_norm(fovea, x, None, gamma, 128)
    assert got["q8"].float()[0].abs().max() == 0 and got["q8_scale"][1, 0] == 0
    assert got["q8"].float()[1, :128].abs().max() == 0
    assert (got["q8"].float()[3] == 448).all()


def test_norm_not_finite(fovea):
    x = torch.randn((4, 300), device="cuda", generator=gen(0))
    x[1, 7] = math.nan
    x[2, 299] = math.inf
    gamma = torch.ones(300, device="cuda")
    for q8 in (0, 64):
        got = fovea.add_rms_norm(x, gamma, None, q8_group=q8)
        assert torch.isnan(got["out"][1]).all() and torch.isnan(got["q8_scale"][1]).all()
        assert torch.isnan(got["out"][2, 299]) and (got["out"][2, :299] == 0).all()
        assert torch.isnan(got["q8_scale"].view(4, -1)[2, -1]) and torch.isnan(got["q8"].float()[2, 299])
        assert torch.isfinite(got["q8"].float()[[0, 3]]).all()


def test_norm_empty_and_offset_rows(fovea):
    gamma = torch.ones(64, device="cuda", dtype=BF16)
    got = fovea.add_rms_norm(torch.empty((0, 64), device="cuda", dtype=BF16), gamma, q8_group=32)
    assert got["out"].shape == (0, 64) and got["q8_scale"].shape == (0, 2)
    # rows more than 2^31 elements apart, from a pointer off every vector's boundary
    big = torch.empty(3 * (1 << 30) + 64, device="cuda", dtype=BF16)
    x = big[1:].as_strided((3, 64), (1 << 30, 1))
    x.copy_(torch.randn((3, 64), device="cuda", generator=gen(1)))
    check_norm(fovea, x, x, gamma, 0)


# ---------------------------------------------------------------------------
# quantize_w4
# ---------------------------------------------------------------------------

def quantize_reference(W, group, symmetric):
    """The definition in fp32 on the CPU: each step is one IEEE operation, so codes are equal."""
    W = W.float().cpu()
    o, k = W.shape
    gs = -(-k // group)
    w = torch.nn.functional.pad(W, (0, gs * group - k)).view(o, gs, group)
    if symmetric:
        scale = (w.abs().amax(2) / torch.tensor(7.0)).to(BF16)
        zero = torch.full((o, gs), 8.0)
    else:
        lo, hi = w.amin(2).clamp(max=0), w.amax(2).clamp(min=0)
        scale = ((hi - lo) / torch.tensor(15.0)).to(BF16)
        zero = torch.where(scale > 0, torch.round(-lo / scale.float()), 8.0).clamp(0, 15)
    f = scale.float()[:, :, None]
    q = torch.where(f > 0, torch.round(w / f), 0.0)
    code = torch.maximum(torch.minimum(q, 15 - zero[:, :, None]), -zero[:, :, None]) + zero[:, :, None]
    code = code.view(o, -1)[:, :k].to(torch.uint8)
    return code[:, 0::2] | code[:, 1::2] << 4, scale, zero.to(torch.uint8)


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("o,k,pad", [(1, 32, 0), (37, 256, 0), (5, 160, 8), (130, 96, 1), (64, 1024, 0), (3, 32768, 0)])
def test_quantize(fovea, dtype, group, o, k, pad):
    g = gen(o * k + group)
    W = torch.empty((o, k + pad), device="cuda", dtype=dtype)[:, :k]
    W.copy_(torch.randn((o, k), generator=g, device="cuda") + 0.3)
    W[0, :32] = 0.0                                       # a group (or part of one) of zeros
    W[-1, :32] = torch.arange(32, device="cuda") * 0.5 - 3.5   # quotients halfway between codes
    for symmetric in (True, False):
        got = fovea.quantize_w4(W, group, symmetric=symmetric)
        codes, scales, zeros = quantize_reference(W, group, symmetric)
        assert torch.equal(got["scales"].cpu(), scales)
        assert torch.equal(got["codes"].cpu(), codes)
        if symmetric:
            assert got["zeros"] is None
        else:
            assert torch.equal(got["zeros"].cpu(), zeros)


def test_quantize_one_sided_tiny_and_not_finite(fovea):
    W = torch.zeros((4, 64), device="cuda")
    W[0] = torch.linspace(1, 2, 64)                       # zero point 0
    W[1] = -torch.linspace(1, 2, 64)                      # zero point 15
    W[2] = 1e-42                                          # a scale below the smallest bf16
    W[3, 5] = math.nan
    for symmetric in (True, False):
        got = fovea.quantize_w4(W, 64, symmetric=symmetric)
        codes, scales, zeros = quantize_reference(W[:3], 64, symmetric)
        assert torch.equal(got["scales"].cpu()[:3], scales) and torch.equal(got["codes"].cpu()[:3], codes)
        if not symmetric:
            assert torch.equal(got["zeros"].cpu()[:3], zeros)
        assert torch.isnan(got["scales"][3]).all()


def test_quantize_beyond_2_to_31_elements(fovea):
    o, k = 70000, 32768
    W = torch.zeros((o, k), device="cuda", dtype=BF16)
    W[-3:] = torch.randn((3, k), device="cuda", generator=gen(3)).to(BF16)
    got = fovea.quantize_w4(W, 128)
    codes, scales, _ = quantize_reference(W[-3:], 128, True)
    assert torch.equal(got["codes"][-3:].cpu(), codes) and torch.equal(got["scales"][-3:].cpu(), scales)
    assert int(got["codes"][:-3].max()) == 0x88 and int(got["codes"][:-3].min()) == 0x88
    # and the product reads them there
    x = torch.randn((2, k), device="cuda", generator=gen(4)).to(BF16)
    y = fovea.linear_w4(x, got["codes"], got["scales"])
    torch.cuda.synchronize()
    assert (y[:, :-3] == 0).all()
    check_product(y[:, -3:], x, None, got["codes"][-3:], got["scales"][-3:], None, 128, None)


# ---------------------------------------------------------------------------
# linear_w4
# ---------------------------------------------------------------------------

def dequantize(codes, scales, zeros, group, k):
    c = torch.stack((codes & 15, codes >> 4), 2).flatten(1).double()
    z = 8.0 if zeros is None else zeros.double().repeat_interleave(group, 1)[:, :k]
    return (c - z) * scales.double().repeat_interleave(group, 1)[:, :k]


def check_product(y, x, x_scale, codes, scales, zeros, group, bias):
    k = x.shape[1]
    w = dequantize(codes, scales, zeros, group, k)
    v = x.double()
    if x_scale is not None:
        v = v * (x_scale.double()[:, None] if x_scale.dim() == 1
                 else x_scale.double().repeat_interleave(group, 1)[:, :k])
    want = v @ w.T
    # fp32 accumulation in some order: at most k + 8 roundings of the sum of magnitudes
    bound = (k + 8) * U * (v.abs() @ w.abs().T)
    if bias is not None:
        want = want + bias.double()
        bound = bound + bias.double().abs() * U
    within(y, want, bound + want.abs() * HALF_ULP[y.dtype] + 1e-37, "y")


def make_w4(g, o, k, group, zeros):
    gs = -(-k // group)
    codes = torch.randint(0, 256, (o, k // 2), generator=g, device="cuda", dtype=torch.uint8)
    scales = (torch.rand((o, gs), generator=g, device="cuda") * k ** -0.5).to(BF16)
    z = torch.randint(0, 16, (o, gs), generator=g, device="cuda", dtype=torch.uint8) if zeros else None
    return codes, scales, z


@pytest.mark.parametrize("x_type", ["bf16", "fp32", "e4m3-row", "e4m3-group"])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("n,o,k,pad", [
    (1, 1, 32, 0), (1, 500, 4096, 0), (2, 33, 96, 0), (5, 129, 160, 3), (7, 250, 1024, 8), (8, 64, 8192, 0),
    (9, 100, 3584, 0), (16, 300, 256, 0), (17, 40, 8192, 0), (33, 129, 544, 8), (64, 640, 1024, 0), (65, 257, 224, 1),
    (150, 90, 512, 0), (3, 20, 32768, 0),
])
def test_linear(fovea, x_type, group, n, o, k, pad):
    g = gen(n * o + k + group)
    codes, scales, zeros = make_w4(g, o, k, group, n % 2 == 1)
    v = torch.randn((n, k), generator=g, device="cuda")
    x_scale = None
    if x_type.startswith("e4m3"):
        x_scale = 0.01 + torch.rand((n, -(-k // group)) if x_type == "e4m3-group" else (n,), generator=g, device="cuda")
    x = torch.empty((n, k + pad), device="cuda", dtype=dict(bf16=BF16, fp32=FP32).get(x_type, E4M3))[:, :k]
    x.copy_(v)
    bias = torch.randn(o, generator=g, device="cuda") if n % 3 == 0 else None
    for out in (FP32, BF16):
        y = fovea.linear_w4(x, codes, scales, zeros, group=group, x_scale=x_scale, bias=bias, out_dtype=out)
        torch.cuda.synchronize()
        assert y.dtype == out
        check_product(y, x, x_scale, codes, scales, zeros, group, bias)


@pytest.mark.parametrize("n,o,k,group", [
    (1, 40001, 512, 128), (3, 39000, 320, 32),           # more tiles than the device has warps
    (33, 20100, 768, 64), (64, 39100, 256, 128),         # more tiles than it has SMs
    (20, 20000, 512, 32),
])
def test_linear_many_tiles(fovea, n, o, k, group):
    g = gen(o)
    codes, scales, zeros = make_w4(g, o, k, group, n % 2 == 1)
    for dtype in (BF16, FP32):
        x = torch.randn((n, k), generator=g, device="cuda").to(dtype)
        y = fovea.linear_w4(x, codes, scales, zeros, group=group)
        torch.cuda.synchronize()
        check_product(y, x, None, codes, scales, zeros, group, None)


@pytest.mark.parametrize("x_type", ["bf16", "fp32", "e4m3-row", "e4m3-group"])
@pytest.mark.parametrize("n,o,k,pad", [
    (1, 9729, 2048, 0), (2, 9759, 2080, 0), (5, 9985, 2176, 3), (8, 10016, 4096, 8), (8, 9745, 13824, 0),
    (1, 39111, 2048, 0),
])
def test_linear_wide_tiles(fovea, x_type, n, o, k, pad):
    # many weight rows in symmetric groups of 128, a few rows of x: the last tile is ragged
    g = gen(n + o + k)
    codes, scales, _ = make_w4(g, o, k, 128, False)
    x_scale = None
    if x_type.startswith("e4m3"):
        x_scale = 0.01 + torch.rand((n, -(-k // 128)) if x_type == "e4m3-group" else (n,), generator=g, device="cuda")
    x = torch.empty((n, k + pad), device="cuda", dtype=dict(bf16=BF16, fp32=FP32).get(x_type, E4M3))[:, :k]
    x.copy_(torch.randn((n, k), generator=g, device="cuda"))
    bias = torch.randn(o, generator=g, device="cuda") if n > 1 else None
    y = fovea.linear_w4(x, codes, scales, x_scale=x_scale, bias=bias)
    torch.cuda.synchronize()
    check_product(y, x, x_scale, codes, scales, None, 128, bias)


@pytest.mark.parametrize("o", [300, 6000])               # tiles split over clusters, and not
def test_linear_wait_that_gives_up(fovea, o):
    """A bounded wait that runs out is told by the workspace and by NaN, and the
    workspace serves the next call."""
    g = gen(o)
    n, k = 64, 16384
    codes, scales, _ = make_w4(g, o, k, 128, False)
    x = torch.randn((n, k), generator=g, device="cuda").to(BF16)
    ws = torch.empty(fovea.linear_w4_workspace_size(n, k), device="cuda", dtype=torch.uint8)
    want = fovea.linear_w4(x, codes, scales, workspace=ws)
    fovea.sync_errors(ws)
    fovea.debug_wait_limit(1)
    try:
        y = fovea.linear_w4(x, codes, scales, workspace=ws)
        with pytest.raises(fovea.FoveaError) as e:
            fovea.sync_errors(ws)
    finally:
        fovea.debug_wait_limit(0)
    assert e.value.status == fovea.ERR_TIMEOUT
    assert torch.isnan(y).any()
    assert torch.equal(fovea.linear_w4(x, codes, scales, workspace=ws), want)
    fovea.sync_errors(ws)


def test_linear_fp32_rows_keep_all_their_bits(fovea):
    # codes and scales of 1: y is the row's sum; values that bf16 cannot hold
    k = 64
    codes = torch.full((16, k // 2), 0x99, device="cuda", dtype=torch.uint8)
    scales = torch.ones((16, 2), device="cuda", dtype=BF16)
    x = torch.zeros((4, k), device="cuda")
    x[0, 3] = 1 + 2.0 ** -23
    x[1, 17] = 3.4e38
    x[2, 63] = -(2.0 ** -100) * (1 + 2.0 ** -12 + 2.0 ** -23)
    x[3, 0] = 16777215.0
    y = fovea.linear_w4(x, codes, scales, group=32)
    assert torch.equal(y, x.sum(1, keepdim=True).expand(4, 16))


def test_linear_not_finite(fovea):
    g = gen(5)
    codes, scales, _ = make_w4(g, 64, 256, 64, False)
    scales[7, 2] = math.nan
    for dtype in (BF16, FP32):
        x = torch.randn((3, 256), generator=g, device="cuda").to(dtype)
        x[1, 100] = math.nan
        y = fovea.linear_w4(x, codes, scales, group=64)
        assert torch.isnan(y[1]).all() and torch.isnan(y[:, 7]).all()
        keep = [i for i in range(64) if i != 7]
        assert torch.isfinite(y[0, keep]).all() and torch.isfinite(y[2, keep]).all()


def test_linear_repeats_bit_for_bit(fovea):
    g = gen(6)
    codes, scales, zeros = make_w4(g, 5000, 4096, 128, True)
    for n in (1, 8, 40, 64):
        x = torch.randn((n, 4096), generator=g, device="cuda").to(BF16)
        y = fovea.linear_w4(x, codes, scales, zeros)
        assert all(torch.equal(y, fovea.linear_w4(x, codes, scales, zeros)) for _ in range(3))


# ---------------------------------------------------------------------------
# token_logprobs and its gradient
# ---------------------------------------------------------------------------

def pack_bits(keep):
    n, v = keep.shape
    w = torch.nn.functional.pad(keep.long(), (0, -(-v // 32) * 32 - v)).view(n, -1, 32)
    w = (w << torch.arange(32, device=keep.device)).sum(2)
    return torch.where(w >= 1 << 31, w - (1 << 32), w).to(torch.int32)


def scores_reference(logits, row_scale, keep):
    """Masked logits, z (a product in 32 bits), and logp, p, lse, entropy, largest z and log sum in 64."""
    x = logits.float()
    if keep is not None:
        x = torch.where(keep, x, -math.inf)
    z = (x if row_scale is None else x * row_scale[:, None]).double()
    m = z.amax(1, keepdim=True)
    zm = z - torch.where(m == -math.inf, 0.0, m)
    log_sum = torch.log(torch.exp(zm).sum(1, keepdim=True))
    lp = zm - torch.where(m == -math.inf, 0.0, log_sum)
    p = torch.exp(lp)
    H = -torch.where(p > 0, p * lp, torch.where(torch.isnan(p), p, 0.0)).sum(1)
    return x, z, lp, p, (m + log_sum)[:, 0], H, m[:, 0], log_sum[:, 0]


def check_scores(fovea, logits, tokens, k, row_scale=None, keep=None, allowed=None, stream=None):
    if keep is not None and allowed is None:
        allowed = pack_bits(keep)
    got = fovea.token_logprobs(logits, tokens, k, row_scale=row_scale, allowed=allowed, stream=stream)
    torch.cuda.synchronize()
    n, v = logits.shape
    x, z, lp, p, lse, H, m, log_sum = scores_reference(logits, row_scale, keep)
    # the sum of positive terms: a thread's chain and the tree above it, each term off by
    # the exponential's 2^-22 and its argument's rounding (up to |z - max| roundings,
    # weighted with e^(z - max))
    chain = v / 256 + 60
    within(got["stats"][:, 0], m, m.abs() * U + 1e-38, "largest")
    within(got["stats"][:, 1], log_sum, chain * U * (1 + log_sum.abs()), "log sum")
    within(got["lse"], lse, chain * U * (1 + log_sum.abs()) + U * 2 * (1 + lse.abs()), "lse")
    # terms of H weigh (1 + |log p|) with p
    within(got["entropy"], H, chain * U * (2 + 2 * H), "entropy")
    off = (chain * U * (1 + log_sum.abs()))[:, None]
    if tokens is not None:
        at = tokens.long()
        want = lp.gather(1, at.clamp(0, v - 1))
        want = torch.where(at < 0, 0.0, torch.where(at >= v, math.nan, want))
        within(got["logprobs"], want, off + 4 * U * (1 + want.abs()), "logprobs")
    if k:
        order = torch.sort(x + 0.0, dim=1, descending=True, stable=True).indices[:, :min(k, v)]
        value = lp.gather(1, order)
        none = z.gather(1, order) == -math.inf
        want = torch.where(none, -1, order)
        pad = k - want.shape[1]
        want = torch.nn.functional.pad(want, (0, pad), value=-1)
        value = torch.nn.functional.pad(value, (0, pad), value=-math.inf)
        assert torch.equal(got["top_idx"].long(), want), "top_idx"
        within(got["top_logprobs"], value, off + 4 * U * (1 + value.abs()), "top_logprobs")
    return got


def make_logits(g, n, v, dtype, pad=0, offset=0):
    x = torch.empty(n * (v + pad) + offset, device="cuda", dtype=dtype)[offset:].view(n, v + pad)[:, :v]
    x.copy_(3 * torch.randn((n, v), generator=g, device="cuda"))
    return x


SHAPES = [  # n, v, T, k, pad, offset
    (1, 1, 1, 1, 0, 0), (3, 5, 2, 6, 0, 1), (1, 32000, 1, 6, 0, 0), (7, 1000, 6, 32, 5, 3), (64, 32000, 6, 6, 0, 0),
    (2, 50257, 3, 10, 0, 1), (40, 8191, 1, 1, 1, 0), (700, 999, 4, 6, 0, 0), (1, 160001, 16, 32, 0, 0),
    (620, 4097, 0, 0, 0, 0), (2, 300, 1, 32, 0, 0), (5, 2049, 1024, 2, 0, 0),
]


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("n,v,T,k,pad,offset", SHAPES)
def test_scores(fovea, dtype, n, v, T, k, pad, offset):
    g = gen(n * v + k)
    x = make_logits(g, n, v, dtype, pad, offset)
    tokens = torch.randint(-1, v, (n, T), generator=g, device="cuda", dtype=torch.int32) if T else None
    check_scores(fovea, x, tokens, k)
    t = torch.empty(n, device="cuda").uniform_(0.3, 3.0, generator=g)
    keep = torch.rand((n, v), generator=g, device="cuda") < 0.4
    keep &= torch.rand((n, 1), generator=g, device="cuda") < 0.8         # some rows keep no token
    x[~keep] = torch.where(torch.rand_like(x[~keep].float()) < 0.5, math.nan, math.inf).to(dtype)
    check_scores(fovea, x, tokens, k, t, keep)
    check_scores(fovea, torch.where(keep, x, -math.inf), tokens, k, t)


def test_scores_one_mask_for_all_rows(fovea):
    g = gen(9)
    x = make_logits(g, 6, 777, BF16)
    keep = torch.rand((1, 777), generator=g, device="cuda") < 0.3
    check_scores(fovea, x, None, 6, keep=keep.expand(6, -1), allowed=pack_bits(keep))


@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_scores_masks_of_the_lowest_value(fovea, dtype):
    low = torch.finfo(dtype).min
    x = make_logits(gen(10), 6, 5000, dtype)
    x[0] = low                                  # nothing but masked tokens: all alike
    x[1, 100:] = low
    x[2, :4990] = low
    x[3] = -1e9
    x[4, 1:] = -math.inf
    x[5] = -math.inf
    tokens = torch.tensor([[0, 4999]] * 6, device="cuda", dtype=torch.int32)
    got = check_scores(fovea, x, tokens, 6)
    assert abs(float(got["logprobs"][0, 0]) + math.log(5000)) < 1e-5
    assert abs(float(got["logprobs"][3, 1]) + math.log(5000)) < 1e-5
    for row_scale in (0.5, 2.0):                # 2 * lowest is -inf
        check_scores(fovea, x, tokens, 6, torch.full((6,), row_scale, device="cuda"))


def test_scores_ties_take_the_smaller_token(fovea):
    for v in (40, 3000, 100000):
        x = torch.zeros((5, v), device="cuda")
        x[1] = -0.0
        x[1, 1::2] = 0.0
        x[2] = torch.arange(v, device="cuda") // 7 % 3
        x[3, v // 2:] = 1.0
        x[4] = torch.randint(0, 2, (v,), device="cuda", generator=gen(v)).float()
        for k in (1, 6, 32):
            got = check_scores(fovea, x, None, k)
            assert got["top_idx"][0].tolist() == list(range(k))
            assert got["top_idx"][1].tolist() == list(range(k))
            assert got["top_idx"][3].tolist()[0] == v // 2
        check_scores(fovea, x.to(BF16), None, 32)


@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_scores_sorted_and_crowded_rows(fovea, dtype):
    """Rows whose largest logits crowd into the tokens of one group of lanes, so that
    more tokens pass its threshold than are kept, and sorted rows."""
    v = 400000
    x = torch.empty((4, v), device="cuda", dtype=dtype)
    x[0] = torch.linspace(-5, 5, v, device="cuda")
    x[1] = torch.linspace(5, -5, v, device="cuda")
    x[2] = torch.randn(v, device="cuda", generator=gen(2))
    per = 8 if dtype == BF16 else 4
    lane = torch.arange(v, device="cuda") // per % 256
    x[2] += torch.where(lane < 4, 10.0, 0.0)
    x[3] = torch.where(lane < 8, 2.0, -2.0)
    for k in (1, 6, 32):
        check_scores(fovea, x, None, k)
        check_scores(fovea, x[2:], None, k)


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("height", [3.0, 40.0, 300.0, 3e4])
def test_scores_spikes(fovea, dtype, height):
    # one token far above, or far below, all others, in the first chunks and in later ones
    v = 40003
    at = [0, 7, 2047, 2048, 9000, 30000, v - 1]
    x = torch.randn((2 * len(at), v), generator=gen(v), device="cuda")
    for i, a in enumerate(at):
        x[2 * i, a] = height
        x[2 * i + 1] += height
        x[2 * i + 1, a] = -height
    tokens = torch.tensor([[a, 1] for a in at for _ in range(2)], device="cuda", dtype=torch.int32)
    check_scores(fovea, x.to(dtype), tokens, 3)
    keep = torch.rand(x.shape, generator=gen(1), device="cuda") < 0.5
    check_scores(fovea, x.to(dtype), tokens, 3, keep=keep)


def test_scores_not_finite_rows(fovea):
    x = make_logits(gen(11), 4, 3000, FP32)
    x[0, 17] = math.nan
    x[1, 5] = math.inf
    x[2, 9] = -math.inf
    tokens = torch.tensor([[3, 9]] * 4, device="cuda", dtype=torch.int32)
    got = fovea.token_logprobs(x, tokens, 6)
    for name in ("logprobs", "lse", "entropy", "top_logprobs"):
        assert torch.isnan(got[name][:2]).all(), name
        assert not torch.isnan(got[name][2:]).any(), name
    assert got["top_idx"][0, 0] == 17 and got["top_idx"][1, 0] == 5
    assert got["logprobs"][2, 1] == -math.inf


def test_scores_tokens_out_of_range(fovea):
    x = make_logits(gen(12), 2, 100, BF16)
    tokens = torch.tensor([[0, 100, -1], [99, -7, 2 ** 31 - 1]], device="cuda", dtype=torch.int32)
    got = check_scores(fovea, x, tokens, 0)
    assert torch.isnan(got["logprobs"][0, 1]) and got["logprobs"][1, 1] == 0
    d = fovea.token_logprobs_grad(x, got["stats"], got["entropy"], tokens=tokens,
                                  grad_logprobs=torch.ones((2, 3), device="cuda"))
    assert torch.isnan(d).all()


def test_scores_rows_beyond_2_to_31_elements(fovea):
    big = torch.empty(3 * (1 << 30) + 4096, device="cuda", dtype=BF16)
    x = big[3:].as_strided((3, 2000), (1 << 30, 1))
    x.copy_(torch.randn((3, 2000), device="cuda", generator=gen(13)))
    tokens = torch.tensor([[1], [5], [1999]], device="cuda", dtype=torch.int32)
    check_scores(fovea, x, tokens, 6)
    check_grad(fovea, x, tokens, 6, gen(14))


def test_scores_more_rows_than_a_grid_holds(fovea):
    g = gen(15)
    n = 70001
    x = make_logits(g, n, 40, BF16)
    tokens = torch.randint(-1, 40, (n, 2), generator=g, device="cuda", dtype=torch.int32)
    t = torch.empty(n, device="cuda").uniform_(0.3, 3.0, generator=g)
    keep = torch.rand((n, 40), generator=g, device="cuda") < 0.5
    check_scores(fovea, x, tokens, 3, t, keep)
    check_grad(fovea, x, tokens, 3, g, t, keep)


def grad_reference(logits, tokens, top_idx, gl, gt, gH, gz, row_scale, keep):
    """Formula in 64 bits, and what bounds its rounding: sums of magnitudes."""
    x, z, lp, p, lse, H, m, log_sum = scores_reference(logits, row_scale, keep)
    n, v = x.shape
    dz = torch.zeros_like(z)
    size = torch.zeros_like(z)
    for ids, g in ((tokens, gl), (top_idx, gt)):
        if ids is None:
            continue
        at = ids.long().clamp(0, v - 1)
        w = torch.where((ids >= 0) & (z.gather(1, at) > -math.inf), g.double(), 0.0)
        dz.scatter_add_(1, at, w)
        size.scatter_add_(1, at, w.abs())
        dz -= p * w.sum(1, keepdim=True)
        size += p * w.abs().sum(1, keepdim=True)
    if gH is not None:
        t = torch.where(p > 0, p * (torch.where(p > 0, lp, 0.0) + H[:, None]), 0.0)
        dz -= gH.double()[:, None] * t
        size += gH.double().abs()[:, None] * p * (torch.where(p > 0, -lp, 0.0) + H[:, None] + 1)
    if gz is not None:
        dz += gz.double()[:, None] * p
        size += gz.double().abs()[:, None] * p
    s = 1.0 if row_scale is None else row_scale.double()[:, None]
    return dz * s, size * s, torch.where(torch.isfinite(lp), lp.abs(), 0.0), log_sum.abs()[:, None]


def check_grad(fovea, logits, tokens, k, g, row_scale=None, keep=None, in_place=False, parts="tkHz"):
    n, v = logits.shape
    allowed = pack_bits(keep) if keep is not None else None
    f = fovea.token_logprobs(logits, tokens, k, row_scale=row_scale, allowed=allowed)
    normal = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    if "t" not in parts:
        tokens = None
    gl = normal(*tokens.shape) if tokens is not None else None
    top = f["top_idx"] if k and "k" in parts else None
    gt = normal(n, k) if top is not None else None
    gH = normal(n) if "H" in parts else None
    gz = normal(n) if "z" in parts else None
    want, size, lp, log_sum = grad_reference(logits, tokens, top, gl, gt, gH, gz, row_scale, keep)
    got = fovea.token_logprobs_grad(logits, f["stats"], f["entropy"], tokens=tokens, grad_logprobs=gl, top_idx=top,
                                    grad_top=gt, grad_entropy=gH, grad_lse=gz, row_scale=row_scale, allowed=allowed,
                                    out=logits if in_place else None)
    torch.cuda.synchronize()
    # p is off by its exponent's error (the log sum's, |logp| times the roundings of its
    # argument), the bracket by the entries' sum and H's error
    chain = v / 256 + 60
    entries = (tokens.shape[1] if tokens is not None else 0) + k
    count = chain * (3 + torch.where(torch.isfinite(log_sum), log_sum, 0.0)) + 8 * (1 + lp) + entries
    within(got, want, size * U * count + want.abs() * HALF_ULP[logits.dtype] + 1e-37, "dlogits")
    return got


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("n,v,T,k,pad,offset", SHAPES)
def test_grad(fovea, dtype, n, v, T, k, pad, offset):
    g = gen(n + v + k)
    x = make_logits(g, n, v, dtype, pad, offset)
    tokens = torch.randint(-1, v, (n, T), generator=g, device="cuda", dtype=torch.int32) if T else None
    check_grad(fovea, x, tokens, k, g)
    t = torch.empty(n, device="cuda").uniform_(0.3, 3.0, generator=g)
    keep = torch.rand((n, v), generator=g, device="cuda") < 0.4
    keep &= torch.rand((n, 1), generator=g, device="cuda") < 0.8
    x[~keep] = math.nan
    got = check_grad(fovea, x, tokens, k, g, t, keep)
    assert (got[~keep] == 0).all()
    x[~keep] = -math.inf
    for parts in ("t", "k", "H", "z"):
        check_grad(fovea, x, tokens, k, g, t, parts=parts)


@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_grad_in_place(fovea, dtype):
    g = gen(20)
    for n, v in ((1, 32000), (5, 999), (50, 4001)):
        x = make_logits(g, n, v, dtype)
        tokens = torch.randint(-1, v, (n, 6), generator=g, device="cuda", dtype=torch.int32)
        check_grad(fovea, x, tokens, 6, g, in_place=True)


def test_grad_repeated_tokens(fovea):
    g = gen(21)
    x = make_logits(g, 3, 500, FP32)
    tokens = torch.tensor([[7, 7, 7, 2], [-1, 4, 4, -1], [0, 499, 0, 499]], device="cuda", dtype=torch.int32)
    a = check_grad(fovea, x, tokens, 6, gen(22))
    assert all(torch.equal(a, check_grad(fovea, x, tokens, 6, gen(22))) for _ in range(3))


@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_grad_masks_of_the_lowest_value(fovea, dtype):
    x = make_logits(gen(23), 4, 3000, dtype)
    x[0] = torch.finfo(dtype).min
    x[1, 10:] = torch.finfo(dtype).min
    x[2] = -math.inf
    x[3] = -1e9
    tokens = torch.tensor([[0, 20]] * 4, device="cuda", dtype=torch.int32)
    got = check_grad(fovea, x, tokens, 6, gen(24))
    assert (got[2] == 0).all()


def test_grad_against_differences(fovea):
    """Central differences of the 64-bit outputs at the same logits: the third
    derivatives of log p, H and lse are at most 2 in size here, so a step of
    2^-10 is off by less than 2^-20 of the gradients' sum."""
    g = gen(25)
    n, v, k, h = 3, 60, 4, 2.0 ** -10
    x = make_logits(g, n, v, FP32) / 3
    t = torch.empty(n, device="cuda").uniform_(0.5, 1.5, generator=g)
    tokens = torch.randint(0, v, (n, 5), generator=g, device="cuda", dtype=torch.int32)
    f = fovea.token_logprobs(x, tokens, k, row_scale=t)
    normal = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    gl, gt, gH, gz = normal(n, 5), normal(n, k), normal(n), normal(n)
    got = fovea.token_logprobs_grad(x, f["stats"], f["entropy"], tokens=tokens, grad_logprobs=gl, top_idx=f["top_idx"],
                                    grad_top=gt, grad_entropy=gH, grad_lse=gz, row_scale=t)

    def loss(xx):
        z = xx * t.double()[:, None]
        lse = torch.logsumexp(z, 1)
        lp = z - lse[:, None]
        H = -(lp.exp() * lp).sum(1)
        return ((gl.double() * lp.gather(1, tokens.long())).sum(1) + gH.double() * H + gz.double() * lse
                + (gt.double() * lp.gather(1, f["top_idx"].long())).sum(1))

    total = gl.abs().sum(1) + gt.abs().sum(1) + 4 * gH.abs() + gz.abs()
    for i in range(v):
        e = torch.zeros((1, v), device="cuda", dtype=torch.float64)
        e[0, i] = h
        want = (loss(x.double() + e) - loss(x.double() - e)) / (2 * h)
        within(got[:, i], want, (2.0 ** -17 * (1 + total.double())), f"token {i}")


# ---------------------------------------------------------------------------
# Streams, graphs, errors, and the operators together
# ---------------------------------------------------------------------------

def test_other_streams_and_graphs(fovea):
    g = gen(30)
    x = torch.randn((7, 512), generator=g, device="cuda").to(BF16)
    gamma = torch.ones(512, device="cuda", dtype=BF16)
    codes, scales, zeros = make_w4(g, 1000, 512, 64, True)

    def step(stream=None):
        a = fovea.add_rms_norm(x, gamma, x, q8_group=64, stream=stream)
        y = fovea.linear_w4(a["q8"], codes, scales, zeros, group=64, x_scale=a["q8_scale"], stream=stream)
        s = fovea.token_logprobs(y, None, 6, stream=stream)
        d = fovea.token_logprobs_grad(y, s["stats"], s["entropy"], top_idx=s["top_idx"],
                                      grad_top=torch.ones((7, 6), device="cuda") if stream is None else ones,
                                      stream=stream)
        return [a["q8"].float(), y, s["top_idx"], s["top_logprobs"], d]

    ones = torch.ones((7, 6), device="cuda")
    want = step()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for stream in (side, side.cuda_stream):
        got = step(stream)
        side.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(want, got))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    x.copy_(torch.randn((7, 512), generator=g, device="cuda"))
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(step(), got))


def test_refusals(fovea):
    x = torch.randn((4, 128), device="cuda")
    ok = fovea.quantize_w4(x)
    bad = [
        lambda: fovea.add_rms_norm(x.cpu(), x[0].contiguous()),
        lambda: fovea.add_rms_norm(x, x[0, :64].contiguous()),
        lambda: fovea.add_rms_norm(x, x[0].to(BF16)),
        lambda: fovea.add_rms_norm(x, x[0].contiguous(), x[:3]),
        lambda: fovea.add_rms_norm(x.t(), x[:, 0].contiguous()),
        lambda: fovea.add_rms_norm(x, x[0].contiguous(), q8_group=48),
        lambda: fovea.add_rms_norm(x, x[0].contiguous(), want_out=False),
        lambda: fovea.add_rms_norm(x.half(), x[0].half()),
        lambda: fovea.add_rms_norm(x, x[0].contiguous(), eps=0.0),
        lambda: fovea.add_rms_norm(torch.zeros((1, 8200), device="cuda"), torch.zeros(8200, device="cuda")),
        lambda: fovea.quantize_w4(x, 16),
        lambda: fovea.quantize_w4(x[:, :100]),
        lambda: fovea.quantize_w4(x[0]),
        lambda: fovea.linear_w4(x, ok["codes"][:, :32].contiguous(), ok["scales"]),
        lambda: fovea.linear_w4(x, ok["codes"], ok["scales"], group=64),
        lambda: fovea.linear_w4(x, ok["codes"], ok["scales"].float()),
        lambda: fovea.linear_w4(x, ok["codes"], ok["scales"], x_scale=x[:, 0].contiguous()),
        lambda: fovea.linear_w4(x.to(E4M3), ok["codes"], ok["scales"]),
        lambda: fovea.linear_w4(x, ok["codes"], ok["scales"], bias=x[0]),
        lambda: fovea.linear_w4(x, ok["codes"], ok["scales"], out_dtype=torch.float16),
        lambda: fovea.token_logprobs(x, torch.zeros((4, 1), device="cuda", dtype=torch.int64)),
        lambda: fovea.token_logprobs(x, torch.zeros((3, 1), device="cuda", dtype=torch.int32)),
        lambda: fovea.token_logprobs(x, None, 33),
        lambda: fovea.token_logprobs(x, None, -1),
        lambda: fovea.token_logprobs(x, torch.zeros((4, 1025), device="cuda", dtype=torch.int32)),
        lambda: fovea.token_logprobs(x, allowed=torch.zeros((4, 3), device="cuda", dtype=torch.int32)),
        lambda: fovea.token_logprobs(x, allowed=torch.zeros((2, 4), device="cuda", dtype=torch.int32)),
        lambda: fovea.token_logprobs(x, row_scale=x[0]),
        lambda: fovea.token_logprobs_grad(x, x[:, :2].contiguous(), x[:, 0].contiguous(),
                                          tokens=torch.zeros((4, 1), device="cuda", dtype=torch.int32)),
        lambda: fovea.token_logprobs_grad(x[:, :100], x[:, :2].contiguous(), x[:, 0].contiguous(),
                                          grad_lse=x[:, 0].contiguous(), out=x[:, :100]),
    ]
    for i, call in enumerate(bad):
        with pytest.raises((ValueError, fovea.FoveaError)):
            call()
            pytest.fail(f"call {i} was not refused")
    torch.cuda.synchronize()


def test_empty_batches(fovea):
    x = torch.zeros((0, 128), device="cuda")
    w = fovea.quantize_w4(torch.ones((5, 128), device="cuda"))
    assert fovea.linear_w4(x, w["codes"], w["scales"]).shape == (0, 5)
    s = fovea.token_logprobs(x, torch.zeros((0, 2), device="cuda", dtype=torch.int32), 6)
    assert s["logprobs"].shape == (0, 2) and s["top_idx"].shape == (0, 6)
    assert fovea.token_logprobs_grad(x, s["stats"], s["entropy"]).shape == (0, 128)
