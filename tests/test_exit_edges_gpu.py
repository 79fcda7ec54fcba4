"""Edges of the drafter-exit operators that a plain comparison on random rows
does not reach: ties and non-numbers in the selection, rows and tokens without
probability in the gradient, exponents, zero points, the error word and devices."""

import math

import pytest
import torch

from test_exit_operators_gpu import BF16, FP32, U, check_product, fovea, gen, make_w4, pack_bits, within  # noqa: F401

pytestmark = pytest.mark.gpu


def at_offset(x, offset):
    """x with its first element `offset` elements behind a 16-byte boundary."""
    buf = torch.empty(offset + x.numel(), device="cuda", dtype=x.dtype)
    assert buf.data_ptr() % 16 == 0
    out = buf[offset:].view(x.shape)
    out.copy_(x)
    return out


def expected_top(x, k):
    # NaN above +inf, the smaller token first on ties (x: no zeros of both signs)
    return torch.sort(x.float(), dim=1, descending=True, stable=True).indices[:, :k]


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("offset", range(8))
def test_ties_with_the_first_chunk_of_a_row_off_the_boundary(fovea, dtype, offset):
    """The largest logit stands in a row's first, ragged chunk, again in a later chunk of
    the thread that takes it (the first whole one, or 256 or 512 further on), and in
    another group of lanes."""
    per = 16 // dtype.itemsize
    v = 20000 if dtype == BF16 else 10000
    rows = []
    for first in (0, 1, per - 1, per):
        for later in (per, per * 257, per * 513 - 1):
            for other in (per * 5, per * 40 + 3):
                rows.append({first, later, other})
                rows.append({first, later})
    x = torch.randn((len(rows), v), generator=gen(offset), device="cuda").clamp(-3, 3)
    for r, at in enumerate(rows):
        x[r, list(at)] = 4.0
    x = at_offset(x.to(dtype), offset)
    keep = torch.ones(x.shape, device="cuda", dtype=torch.bool)
    for k in (1, 2, 6):
        for allowed in (None, pack_bits(keep)):
            got = fovea.token_logprobs(x, None, k, allowed=allowed)
            assert torch.equal(got["top_idx"].long(), expected_top(x, k)), k


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("v", [5000, 4999, 32001, 70001])
def test_ties_of_many_tokens_in_odd_vocabularies(fovea, dtype, v):
    # dense rows of an odd width start at every offset; few rows are cut over a cluster
    g = gen(v)
    for n in (2, 300):
        x = torch.zeros((n, v), device="cuda")
        at = torch.randint(0, v, (n, 40), generator=g, device="cuda")
        at[:, 0] = torch.arange(n, device="cuda") % 3
        x.scatter_(1, at, 1.0)
        x = x.to(dtype)
        for k in (1, 6, 32):
            got = fovea.token_logprobs(x, None, k)
            assert torch.equal(got["top_idx"].long(), expected_top(x, k)), (n, k)


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("v,offset", [(1, 0), (3000, 0), (3000, 1), (100001, 3)])
def test_a_nan_at_the_first_token_is_an_alternative(fovea, dtype, v, offset):
    places = [{0: math.nan}, {0: math.nan, v // 2: math.nan}, {0: math.nan, v - 1: math.nan, v // 3: math.inf},
              {0: math.inf}, {v - 1: math.nan}]
    x = torch.randn((len(places), v), generator=gen(v), device="cuda")
    x += torch.arange(v, device="cuda") * 1e-4
    for r, place in enumerate(places):
        for at, value in place.items():
            x[r, at] = value
    x = at_offset(x.to(dtype), offset)
    for k in (1, 2, 6):
        got = fovea.token_logprobs(x, None, k)
        want = expected_top(x, k)
        assert torch.equal(got["top_idx"][:, :want.shape[1]].long(), want), k
        assert torch.isnan(got["top_logprobs"][:, :want.shape[1]]).all()
        assert (got["top_idx"][:, want.shape[1]:] == -1).all()


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("v", [1, 40, 3001])
def test_gradient_of_a_row_without_tokens_is_zero_whatever_comes_back(fovea, dtype, v):
    """lse is -inf there, so that a loss of it, squared for instance, sends an infinity
    back; rows with tokens beside it keep theirs."""
    x = torch.randn((4, v), generator=gen(v), device="cuda").to(dtype)
    x[0] = -math.inf
    keep = torch.ones((4, v), device="cuda", dtype=torch.bool)
    keep[1] = False
    tokens = torch.zeros((4, 1), device="cuda", dtype=torch.int32)
    allowed = pack_bits(keep)
    f = fovea.token_logprobs(x, tokens, 1, allowed=allowed)
    assert (f["lse"][:2] == -math.inf).all() and torch.isfinite(f["lse"][2:]).all()
    one = torch.ones(4, device="cuda")
    for value in (-math.inf, math.inf, math.nan, 1.0):
        back = one.clone()
        back[:2] = value
        for gH, gz in ((back, None), (None, back), (back, back), (one, 2 * f["lse"])):
            d = fovea.token_logprobs_grad(x, f["stats"], f["entropy"], tokens=tokens, grad_logprobs=back[:, None],
                                          top_idx=f["top_idx"], grad_top=back[:, None], grad_entropy=gH, grad_lse=gz,
                                          allowed=allowed)
            assert (d[:2] == 0).all()
            assert torch.isfinite(d[2:]).all()


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("n,v", [(6, 40), (6, 3001), (3, 50000)])
def test_gradient_of_tokens_that_are_not_allowed_is_zero_in_any_row(fovea, dtype, n, v):
    g = gen(v)
    keep = torch.rand((n, v), generator=g, device="cuda") < 0.5
    keep[:, 1] = True
    x = torch.randn((n, v), generator=g, device="cuda").to(dtype)
    x[0, 1] = math.nan                                     # every probability of the row is NaN
    x[1, 1] = math.inf
    tokens = torch.ones((n, 1), device="cuda", dtype=torch.int32)
    tokens[2] = v                                          # no such token
    allowed = pack_bits(keep)
    f = fovea.token_logprobs(x, tokens, 2, allowed=allowed)
    d = fovea.token_logprobs_grad(x, f["stats"], f["entropy"], tokens=tokens, top_idx=f["top_idx"],
                                  grad_logprobs=torch.ones((n, 1), device="cuda"),
                                  grad_top=torch.ones((n, 2), device="cuda"),
                                  grad_entropy=torch.ones(n, device="cuda"), allowed=allowed)
    assert (d[~keep] == 0).all()
    for r in range(3):
        assert torch.isnan(d[r][keep[r]]).all()
    assert torch.isfinite(d[3:]).all()


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("v", [40, 3001, 100003])
def test_no_log_probability_is_above_zero_under_a_temperature(fovea, dtype, v):
    """z is the product of logit and temperature rounded once, wherever it stands: the
    largest one's log probability is minus the log sum exactly, which is 0 or more."""
    g = gen(v)
    n = 200
    x = torch.randn((n, v), generator=g, device="cuda")
    x[:, v // 3] = 10 + 20 * torch.rand(n, generator=g, device="cuda")
    x = x.to(dtype)
    t = torch.empty(n, device="cuda").uniform_(0.3, 3.0, generator=g)
    tokens = torch.full((n, 1), v // 3, device="cuda", dtype=torch.int32)
    got = fovea.token_logprobs(x, tokens, 2, row_scale=t)
    assert (got["top_idx"][:, 0] == v // 3).all()
    assert torch.equal(got["stats"][:, 0], x[:, v // 3].float() * t)
    assert (got["stats"][:, 1] >= 0).all()
    assert torch.equal(got["top_logprobs"][:, 0], 0 - got["stats"][:, 1])
    assert torch.equal(got["logprobs"][:, 0], 0 - got["stats"][:, 1])


@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_a_token_with_a_gradient_of_zero_changes_no_bit(fovea, dtype):
    # its gradient is written again by another piece of code, with the same operations
    g = gen(17)
    n, v = 40, 3001
    x = (5 * torch.randn((n, v), generator=g, device="cuda")).to(dtype)
    t = torch.empty(n, device="cuda").uniform_(0.3, 3.0, generator=g)
    tokens = torch.randint(0, v, (n, 500), generator=g, device="cuda", dtype=torch.int32)
    f = fovea.token_logprobs(x, tokens, 6, row_scale=t)
    assert (f["logprobs"] <= 0).all()
    back = dict(grad_entropy=torch.randn(n, generator=g, device="cuda"),
                grad_lse=torch.randn(n, generator=g, device="cuda"), row_scale=t)
    want = fovea.token_logprobs_grad(x, f["stats"], f["entropy"], **back)
    got = fovea.token_logprobs_grad(x, f["stats"], f["entropy"], tokens=tokens, top_idx=f["top_idx"],
                                    grad_logprobs=torch.zeros((n, 500), device="cuda"),
                                    grad_top=torch.zeros((n, 6), device="cuda"), **back)
    assert torch.equal(got, want)


@pytest.mark.parametrize("lowest", [-4.0, -20.0, -80.0])
def test_gradient_keeps_the_bits_of_small_probabilities(fovea, lowest):
    """With a largest z and a log sum of 0 the logits are the log probabilities, exactly:
    grad_lse gives p = e^logit.  Its exponential is good to 2^-22, and three roundings
    follow: 7 u, and one for what the exponent's own remainder loses."""
    g = gen(7)
    n, v = 4, 50000
    x = lowest * torch.rand((n, v), generator=g, device="cuda")
    tokens = torch.randint(0, v, (n, 500), generator=g, device="cuda", dtype=torch.int32)
    stats, zero = torch.zeros((n, 2), device="cuda"), torch.zeros(n, device="cuda")
    one = torch.ones(n, device="cuda")
    want = x.double().exp()
    got = fovea.token_logprobs_grad(x, stats, zero, grad_lse=one)
    within(got, want, 8 * U * want)
    # tokens with an entry of their own are computed again
    got = fovea.token_logprobs_grad(x, stats, zero, tokens=tokens, grad_logprobs=torch.zeros((n, 500), device="cuda"),
                                    grad_lse=one)
    within(got, want, 8 * U * want)


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("n", [1, 3, 8, 9, 40])            # few rows, and through tensor memory
def test_zero_points_above_15(fovea, n, group):
    """A zero point is what its low seven bits say, in every path (formats that store it
    less one reach 16)."""
    g = gen(n + group)
    o, k = 200, 544
    codes, scales, _ = make_w4(g, o, k, group, False)
    zeros = torch.randint(0, 128, scales.shape, generator=g, device="cuda", dtype=torch.uint8)
    zeros[:, 0] = 16
    zeros[0] = 127
    for dtype in (BF16, FP32):
        x = torch.randn((n, k), generator=g, device="cuda").to(dtype)
        y = fovea.linear_w4(x, codes, scales, zeros, group=group)
        check_product(y, x, None, codes, scales, zeros, group, None)
        assert torch.equal(y, fovea.linear_w4(x, codes, scales, zeros + 128, group=group))


def exhausted(fovea, call):
    """call() with bounded waits that give up."""
    fovea.debug_wait_limit(1)
    try:
        return call()
    finally:
        fovea.debug_wait_limit(0)


def big_product(fovea, o):
    g = gen(o)
    n, k = 64, 16384
    codes, scales, _ = make_w4(g, o, k, 128, False)
    x = torch.randn((n, k), generator=g, device="cuda").to(BF16)
    ws = torch.empty(fovea.linear_w4_workspace_size(n, k), device="cuda", dtype=torch.uint8)
    return x, codes, scales, ws


def test_a_wait_that_gave_up_is_told_after_later_calls(fovea):
    x, codes, scales, ws = big_product(fovea, 6000)
    want = fovea.linear_w4(x, codes, scales, workspace=ws)
    fovea.sync_errors(ws)
    y = exhausted(fovea, lambda: fovea.linear_w4(x, codes, scales, workspace=ws))
    assert torch.equal(fovea.linear_w4(x, codes, scales, workspace=ws), want)      # through tensor memory
    fovea.linear_w4(x[:2], codes, scales, workspace=ws)                            # few rows
    with pytest.raises(fovea.FoveaError) as e:
        fovea.sync_errors(ws)
    assert e.value.status == fovea.ERR_TIMEOUT and torch.isnan(y).any()
    assert torch.equal(fovea.linear_w4(x, codes, scales, workspace=ws), want)
    fovea.sync_errors(ws)


@pytest.mark.parametrize("n", [2, 64])
@pytest.mark.parametrize("byte", [0, 1, 2, 3, 0xA5, 0xFF])
def test_an_uninitialised_workspace_reports_nothing(fovea, n, byte):
    x, codes, scales, ws = big_product(fovea, 300)
    ws.fill_(byte)
    fovea.linear_w4(x[:n], codes, scales, workspace=ws)
    fovea.sync_errors(ws)


@pytest.mark.parametrize("n", [2, 64])
def test_a_pending_error_of_another_call_is_kept(fovea, n):
    # a workspace of the step, with a depth out of range seen and not yet told
    x, codes, scales, ws = big_product(fovea, 300)
    fovea.workspace_init(ws)
    ws[0] = 1
    fovea.linear_w4(x[:n], codes, scales, workspace=ws)
    with pytest.raises(fovea.FoveaError) as e:
        fovea.sync_errors(ws)
    assert e.value.status == fovea.ERR_INVALID_ARG
    fovea.linear_w4(x[:n], codes, scales, workspace=ws)
    fovea.sync_errors(ws)


def test_a_small_workspace_that_few_rows_do_not_need(fovea):
    x, codes, scales, _ = big_product(fovea, 300)
    want = fovea.linear_w4(x[:2], codes, scales)
    for size in (0, 1, 100, 4097):
        ws = torch.full((size + 1,), 7, device="cuda", dtype=torch.uint8)[1:]
        assert torch.equal(fovea.linear_w4(x[:2], codes, scales, workspace=ws), want)
        assert (ws == 7).all()


class Elsewhere(torch.Tensor):
    """A tensor of this GPU that says it is another one's."""

    def get_device(self):
        return 1


def operator_calls(fovea):
    x = torch.randn((4, 128), device="cuda")
    w = fovea.quantize_w4(x)
    gamma, bias = torch.ones(128, device="cuda"), torch.zeros(4, device="cuda")
    x8, x_scale = x.to(torch.float8_e4m3fn), torch.ones(4, device="cuda")
    ws = torch.zeros(1 << 20, device="cuda", dtype=torch.uint8)
    tokens = torch.zeros((4, 1), device="cuda", dtype=torch.int32)
    allowed = torch.full((4, 4), -1, device="cuda", dtype=torch.int32)
    f = fovea.token_logprobs(x, tokens, 2)
    g1, g2 = torch.ones((4, 1), device="cuda"), torch.ones((4, 2), device="cuda")
    return [
        (fovea.add_rms_norm, dict(x=x, gamma=gamma, residual=x.clone())),
        (fovea.quantize_w4, dict(W=x)),
        (fovea.linear_w4, dict(x=x8, codes=w["codes"], scales=w["scales"], zeros=torch.zeros_like(w["scales"]).byte(),
                               x_scale=x_scale, bias=bias, workspace=ws)),
        (fovea.token_logprobs, dict(logits=x, tokens=tokens, row_scale=bias + 1, allowed=allowed)),
        (fovea.token_logprobs_grad, dict(logits=x, stats=f["stats"], entropy=f["entropy"], tokens=tokens,
                                         grad_logprobs=g1, top_idx=f["top_idx"], grad_top=g2, grad_entropy=bias,
                                         grad_lse=bias.clone(), row_scale=bias + 1, allowed=allowed,
                                         out=torch.empty_like(x))),
    ]


def test_tensors_of_several_devices_are_refused(fovea):
    for call, kw in operator_calls(fovea):
        call(**kw)
        for name, t in kw.items():
            with pytest.raises(ValueError, match="cuda:1"):
                call(**dict(kw, **{name: t.as_subclass(Elsewhere)}))
                pytest.fail(f"{call.__name__}: {name} was not refused")


def test_tensors_of_a_device_that_is_not_the_current_one_are_refused(fovea, monkeypatch):
    calls = operator_calls(fovea)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    for call, kw in calls:
        with pytest.raises(ValueError, match="current device"):
            call(**kw)
            pytest.fail(f"{call.__name__} was not refused")
