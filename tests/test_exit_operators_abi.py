"""Argument checks of the operators of the drafter's exit at the C boundary
(no call here reaches the device)."""

import os

import pytest

from paper_2608_22883_gb300 import fovea

P = 0x10000          # never dereferenced: every call below fails its checks first


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(fovea.LIB_PATH):
        from paper_2608_22883_gb300 import _build
        _build.build()
    return fovea.lib()


def norm(L, *, x=P, ld=64, r=None, r_ld=0, gamma=P, N=4, d=64, dtype=fovea.BF16, eps=1e-6, s=None, out=P, q8=None,
         scale=None, group=0):
    return L.fovea_add_rms_norm(x, ld, r, r_ld, gamma, N, d, dtype, eps, s, out, q8, scale, group, None)


def quantize(L, *, W=P, ld=128, o=4, k=128, dtype=fovea.BF16, group=128, codes=P, scales=P, zeros=None):
    return L.fovea_quantize_w4(W, ld, o, k, dtype, group, codes, scales, zeros, None)


def linear(L, *, x=P, ld=128, x_dtype=fovea.BF16, x_scale=None, x_group=0, N=4, codes=P, scales=P, zeros=None,
           bias=None, o=4, k=128, group=128, y=P, y_dtype=fovea.FP32, ws=P, ws_bytes=1 << 30):
    return L.fovea_linear_w4(x, ld, x_dtype, x_scale, x_group, N, codes, scales, zeros, bias, o, k, group, y, y_dtype,
                             ws, ws_bytes, None)


def scores(L, *, x=P, ld=100, N=4, V=100, dtype=fovea.BF16, scale=None, allowed=None, a_ld=0, tokens=P, T=1, k=6,
           lp=P, lse=P, H=P, stats=P, idx=P, top=P):
    return L.fovea_token_logprobs(x, ld, N, V, dtype, scale, allowed, a_ld, tokens, T, k, lp, lse, H, stats, idx, top,
                                  None)


def grad(L, *, x=P, ld=100, N=4, V=100, dtype=fovea.BF16, scale=None, allowed=None, a_ld=0, stats=P, H=P, tokens=P,
         gl=P, T=1, idx=P, gt=P, k=6, gH=None, gz=None, out=P + 65536):
    return L.fovea_token_logprobs_grad(x, ld, N, V, dtype, scale, allowed, a_ld, stats, H, tokens, gl, T, idx, gt, k,
                                       gH, gz, out, None)


BAD, NO = fovea.ERR_INVALID_ARG, fovea.ERR_UNSUPPORTED


@pytest.mark.parametrize("call,kw,status", [
    (norm, dict(dtype=2), BAD), (norm, dict(d=0), BAD), (norm, dict(d=8193, ld=8193), NO), (norm, dict(eps=0.0), BAD),
    (norm, dict(eps=float("nan")), BAD), (norm, dict(group=16), BAD), (norm, dict(N=-1), BAD), (norm, dict(ld=63), BAD),
    (norm, dict(r=P, r_ld=10), BAD), (norm, dict(gamma=None), BAD), (norm, dict(x=None), BAD), (norm, dict(x=P + 1), BAD),
    (norm, dict(out=None), BAD), (norm, dict(q8=P), BAD), (norm, dict(s=P + 1), BAD),
    (quantize, dict(dtype=2), BAD), (quantize, dict(o=0), BAD), (quantize, dict(k=0), BAD), (quantize, dict(k=100), BAD),
    (quantize, dict(k=32800, ld=32800), NO), (quantize, dict(group=256), BAD), (quantize, dict(ld=127), BAD),
    (quantize, dict(W=None), BAD), (quantize, dict(codes=P + 2), BAD), (quantize, dict(scales=P + 1), BAD),
    (linear, dict(x_dtype=3), BAD), (linear, dict(y_dtype=2), BAD), (linear, dict(k=48), BAD), (linear, dict(N=-2), BAD),
    (linear, dict(x_scale=P), BAD), (linear, dict(x_dtype=2), BAD), (linear, dict(x_dtype=2, x_scale=P, x_group=64), BAD),
    (linear, dict(codes=P + 8), BAD), (linear, dict(scales=None), BAD), (linear, dict(bias=P + 2), BAD),
    (linear, dict(x=None), BAD), (linear, dict(y=None), BAD), (linear, dict(ld=100), BAD),
    (linear, dict(N=17, ws=None), BAD), (linear, dict(N=17, ws=P + 16), BAD), (linear, dict(N=17, ws_bytes=5000), BAD),
    (linear, dict(N=6, x_dtype=fovea.FP32, ws=None), BAD),
    (scores, dict(dtype=2), BAD), (scores, dict(V=0), BAD), (scores, dict(V=(1 << 24) + 1, ld=1 << 25), NO),
    (scores, dict(T=-1), BAD), (scores, dict(T=1025), NO), (scores, dict(k=33), NO), (scores, dict(k=-1), BAD),
    (scores, dict(N=-1), BAD), (scores, dict(ld=99), BAD), (scores, dict(allowed=P, a_ld=3), BAD),
    (scores, dict(allowed=P + 2), BAD), (scores, dict(x=None), BAD), (scores, dict(tokens=None), BAD),
    (scores, dict(lp=None), BAD), (scores, dict(lse=None), BAD), (scores, dict(H=None), BAD),
    (scores, dict(stats=None), BAD), (scores, dict(idx=None), BAD), (scores, dict(top=None), BAD),
    (grad, dict(dtype=2), BAD), (grad, dict(stats=None), BAD), (grad, dict(H=None), BAD), (grad, dict(gl=None), BAD),
    (grad, dict(idx=None), BAD), (grad, dict(gt=None), BAD), (grad, dict(out=None), BAD), (grad, dict(gH=P + 2), BAD),
    (grad, dict(out=P, ld=104), BAD),
])
def test_refusals(L, call, kw, status):
    assert call(L, **kw) == status
    assert fovea.last_error() != ""


@pytest.mark.parametrize("call", [norm, linear, scores, grad])
def test_no_rows_is_no_work(L, call):
    assert call(L, N=0) == fovea.OK


def test_linear_workspace_sizes():
    import torch
    size = fovea.linear_w4_workspace_size
    assert size(2, 16384, dtype=torch.float32) == 0 and size(8, 16384) == 0 and size(0, 4096) == 0
    assert size(17, 4096) >= 4096 + 17 * 4096 * 2
    assert size(6, 4096, dtype=torch.float32) >= 4096 + 18 * 4096 * 2
    assert size(17, 4096, dtype=torch.float8_e4m3fn, x_group=128) >= size(17, 4096) + 17 * 32 * 4
    for bad in (dict(N=-1, in_features=64), dict(N=1, in_features=65), dict(N=1, in_features=64, group=16)):
        with pytest.raises(fovea.FoveaError):
            size(**bad)


def test_binding_refuses_host_tensors():
    import torch
    x = torch.zeros((2, 64))
    for call in (lambda: fovea.add_rms_norm(x, x[0]), lambda: fovea.quantize_w4(x),
                 lambda: fovea.linear_w4(x, x, x), lambda: fovea.token_logprobs(x),
                 lambda: fovea.token_logprobs_grad(x, x, x)):
        with pytest.raises(ValueError, match="CUDA tensor"):
            call()
