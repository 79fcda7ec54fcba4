"""Argument checks of the operators of the drafter's cache at the C boundary (no call
here reaches the device), and of their binding without one."""

import math
import os

import pytest
import torch

from paper_2608_22883_gb300 import fovea

P = 0x10000          # never dereferenced: every call below fails its checks first
BF16, FP32, E4M3 = fovea.BF16, fovea.FP32, fovea.E4M3


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(fovea.LIB_PATH):
        from paper_2608_22883_gb300 import _build
        _build.build()
    return fovea.lib()


def rotary(L, *, q=P, q_ld=512, q_hs=128, heads=4, k=P, k_ld=128, k_hs=128, kv=1, N=4, dim=128, dtype=BF16, pos=P,
           pos_ld=4, axes=3, f=P, axis=P, rot=128, q_out=2 * P, k_out=3 * P):
    return L.fovea_rotary_axes(q, q_ld, q_hs, heads, k, k_ld, k_hs, kv, N, dim, dtype, pos, pos_ld, axes, f, axis, rot, 0,
                               0, q_out, k_out, None)


def append(L, *, q=P, q_ld=512, q_hs=128, heads=4, k=P, k_ld=128, k_hs=128, v=P, v_ld=128, v_hs=128, N=4, dtype=BF16,
           pos=P, pos_ld=4, axes=1, f=P, axis=None, rot=128, q_out=2 * P, kp=P, vp=P, cache=BF16, ks=None, vs=None,
           n_pages=9, page=16, kv=1, dim=128, table=P, B=2, width=3, sequence=P, entry=P):
    return L.fovea_cache_append(q, q_ld, q_hs, heads, k, k_ld, k_hs, v, v_ld, v_hs, N, dtype, pos, pos_ld, axes, f, axis,
                                rot, 0, q_out, kp, vp, cache, ks, vs, n_pages, page, kv, dim, table, B, width, sequence,
                                entry, None)


def attention(L, *, q=P, q_ld=512, q_hs=128, heads=4, kp=P, vp=P, cache=BF16, ks=None, vs=None, n_pages=9, page=16, kv=1,
              dim=128, table=P, B=2, width=3, lens=P, nodes=1, tree=None, tree_rows=0, scale=0.1, out=P, lse=P, ws=P,
              ws_bytes=1 << 30):
    return L.fovea_paged_attention(q, q_ld, q_hs, heads, kp, vp, cache, ks, vs, n_pages, page, kv, dim, table, B, width,
                                   lens, nodes, tree, tree_rows, scale, out, lse, ws, ws_bytes, None)


def keep(L, *, kp=P, vp=P, cache=BF16, n_pages=9, page=16, kv=1, dim=128, table=P, B=2, width=3, lens=P, nodes=P, path=2,
         size=4, new=2 * P):
    return L.fovea_cache_keep(kp, vp, cache, n_pages, page, kv, dim, table, B, width, lens, nodes, path, size, new, None)


def fork(L, *, kp=P, vp=P, cache=BF16, n_pages=9, page=16, kv=1, dim=128, table=P, B=2, width=3, lens=P, parents=P,
         kept=None, room=None, C=2, new=2 * P, new_width=3, new_lens=3 * P, free=P):
    return L.fovea_cache_fork(kp, vp, cache, n_pages, page, kv, dim, table, B, width, lens, parents, kept, room, C, new,
                              new_width, new_lens, free, None)


BAD, NO = fovea.ERR_INVALID_ARG, fovea.ERR_UNSUPPORTED
#: What every call on a cache refuses.
CACHE = [(dict(cache=3), BAD), (dict(dim=96), NO), (dict(dim=0), NO), (dict(page=8), BAD), (dict(page=24), BAD),
         (dict(page=0), BAD), (dict(page=1040), NO), (dict(kv=0), BAD), (dict(n_pages=0), BAD), (dict(B=-1), BAD),
         (dict(width=0), BAD), (dict(B=2049), NO), (dict(width=1 << 27), NO), (dict(kp=None), BAD), (dict(vp=None), BAD),
         (dict(kp=P + 8), BAD), (dict(table=None), BAD), (dict(table=P + 2), BAD), (dict(kv=1025), NO)]


@pytest.mark.parametrize("call,kw,status", [
    (rotary, dict(dtype=E4M3), BAD), (rotary, dict(N=-1), BAD), (rotary, dict(dim=1), BAD), (rotary, dict(dim=513), NO),
    (rotary, dict(heads=0), BAD), (rotary, dict(kv=-1), BAD), (rotary, dict(heads=1024), NO), (rotary, dict(rot=0), BAD),
    (rotary, dict(rot=7), BAD), (rotary, dict(rot=130), BAD), (rotary, dict(axes=0), BAD), (rotary, dict(axes=9), NO),
    (rotary, dict(pos_ld=-1), BAD), (rotary, dict(pos=None), BAD), (rotary, dict(f=None), BAD), (rotary, dict(f=P + 4), BAD),
    (rotary, dict(axis=P + 1), BAD), (rotary, dict(q=None), BAD), (rotary, dict(k=None), BAD), (rotary, dict(q=P + 1), BAD),
    (rotary, dict(q_out=None), BAD), (rotary, dict(k_out=None), BAD), (rotary, dict(q_ld=-1), BAD),
    (rotary, dict(q_out=P, q_ld=640), BAD), (rotary, dict(k_out=P, k_ld=129), BAD),
    (append, dict(dtype=E4M3), BAD), (append, dict(N=-1), BAD), (append, dict(dtype=FP32), NO), (append, dict(cache=FP32), NO),
    (append, dict(ks=P), BAD), (append, dict(heads=0), BAD), (append, dict(heads=1023), NO), (append, dict(rot=0), BAD),
    (append, dict(rot=130), BAD), (append, dict(k=None), BAD), (append, dict(v=None), BAD), (append, dict(v=P + 1), BAD),
    (append, dict(sequence=None), BAD), (append, dict(entry=P + 2), BAD), (append, dict(q_out=None), BAD),
    (append, dict(q_out=P, q_ld=640), BAD), (append, dict(cache=E4M3, vs=P + 2), BAD), (append, dict(v_hs=-4), BAD),
    (attention, dict(heads=3, kv=2), BAD), (attention, dict(heads=0), BAD), (attention, dict(nodes=0), BAD),
    (attention, dict(nodes=257), NO), (attention, dict(heads=1025), NO), (attention, dict(tree=P, tree_rows=3), BAD),
    (attention, dict(tree=P + 2, tree_rows=1), BAD), (attention, dict(scale=math.nan), BAD),
    (attention, dict(scale=math.inf), BAD), (attention, dict(q=None), BAD), (attention, dict(lens=None), BAD),
    (attention, dict(out=None), BAD), (attention, dict(out=P + 8), BAD), (attention, dict(lse=P + 2), BAD),
    (attention, dict(ws=None), BAD), (attention, dict(ws=P + 16), BAD), (attention, dict(ws_bytes=4096), BAD),
    (attention, dict(ks=P), BAD),
    (keep, dict(path=0), BAD), (keep, dict(path=5), BAD), (keep, dict(size=257), NO), (keep, dict(lens=None), BAD),
    (keep, dict(nodes=None), BAD), (keep, dict(new=None), BAD), (keep, dict(new=P), BAD),
    (fork, dict(C=-1), BAD), (fork, dict(C=2049), NO), (fork, dict(new_width=0), BAD), (fork, dict(new_width=1 << 27), NO),
    (fork, dict(n_pages=(1 << 20) + 1), NO), (fork, dict(lens=None), BAD), (fork, dict(parents=None), BAD),
    (fork, dict(new=None), BAD), (fork, dict(new=P), BAD), (fork, dict(new_lens=P), BAD), (fork, dict(free=None), BAD),
    (fork, dict(C=2048, new_width=1 << 26), NO), (fork, dict(C=17, new_width=1 << 26), NO),
    (fork, dict(kept=P + 1), BAD), (fork, dict(room=P + 2), BAD),
] + [(call, kw, status) for call in (append, attention, keep, fork) for kw, status in CACHE])
def test_refusals(L, call, kw, status):
    assert call(L, **kw) == status
    assert fovea.last_error() != ""


@pytest.mark.parametrize("call,kw", [(rotary, dict(N=0)), (append, dict(N=0)), (attention, dict(B=0)), (keep, dict(B=0))])
def test_no_rows_is_no_work(L, call, kw):
    assert call(L, **kw) == fovea.OK


def test_attention_workspace_sizes():
    size = fovea.paged_attention_workspace_size
    for heads, kv, nodes, dim, dtype in ((32, 32, 1, 128, torch.bfloat16), (28, 4, 64, 64, torch.float8_e4m3fn),
                                         (8, 8, 1, 256, torch.float32)):
        n = size(3, nodes, heads, kv, dim, dtype)
        # partial sums of a row for each of a CTA per SM, at least
        assert n >= 152 * 8 * (dim + 2) * 4 and n == size(2000, nodes, heads, kv, dim, dtype)
    for bad in (dict(nodes=0), dict(heads=5), dict(dim=80), dict(B=-1)):
        with pytest.raises(fovea.FoveaError):
            size(**{**dict(B=1, nodes=1, heads=4, kv_heads=2, dim=64), **bad})


def test_rotary_frequencies():
    f, axis = fovea.rotary_frequencies(128, base=1e4, device="cpu")
    assert f.dtype == torch.float64 and axis.dtype == torch.int32 and not axis.any()
    assert torch.allclose(f, 1e4 ** (-torch.arange(64, dtype=torch.float64) / 64), rtol=1e-14, atol=0)
    f, axis = fovea.rotary_frequencies(16, [2, 3, 3], base=1e4, device="cpu")
    assert axis.tolist() == [0, 0, 1, 1, 1, 2, 2, 2] and f[5] == 1e4 ** -0.625
    f, axis = fovea.rotary_frequencies(16, [2, 3, 3], base=1e4, interleaved=True, device="cpu")
    assert axis.tolist() == [0, 1, 2, 0, 1, 2, 1, 2] and f[5] == 1e4 ** -0.625
    f, _ = fovea.rotary_frequencies(16, [2, 3, 3], base=1e4, restart=True, device="cpu")
    assert f.tolist() == [1.0, 1e4 ** -0.5, 1.0, 1e4 ** -(1 / 3), 1e4 ** -(2 / 3), 1.0, 1e4 ** -(1 / 3), 1e4 ** -(2 / 3)]
    for bad in ((15, None), (0, None), (16, [4, 5]), (16, [-1, 9])):
        with pytest.raises(ValueError):
            fovea.rotary_frequencies(*bad, device="cpu")


def test_binding_refuses_host_tensors():
    x, i = torch.zeros((2, 1, 64)), torch.zeros(2, dtype=torch.int32)
    pages, table = torch.zeros((2, 1, 16, 64)), torch.zeros((2, 1), dtype=torch.int32)
    for call in (lambda: fovea.rotary_axes(x, x, table.T, x[0, 0].double()),
                 lambda: fovea.cache_append(x, x, pages, pages, table, i, i),
                 lambda: fovea.paged_attention(x, pages, pages, table, i),
                 lambda: fovea.cache_keep(pages, pages, table, i, table, 1),
                 lambda: fovea.cache_fork(pages, pages, table, i, i)):
        with pytest.raises(ValueError, match="CUDA tensor"):
            call()
