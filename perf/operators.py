"""Operators of the drafter's exit with 4-bit weights, and of its tokens' scores.

After its last block a drafter adds the block's output to the residual stream
and normalises it (``add_rms_norm``, with an 8-bit output for a quantised
product), multiplies by weights held in 4 bits (``linear_w4``; ``quantize_w4``
makes them), and a program that grows, verifies or trains a draft tree reads
the log probabilities of given tokens, the entropy and the best alternatives
from the logits (``token_logprobs``), and their gradient
(``token_logprobs_grad``).

``run`` computes each of them with elementary torch operations in 32 bits, or
(``own``) through the framework's binding.  Sizes follow this repository's
workloads: model widths 3584, 4096 and 5120, a vocabulary of 32000, trees of up
to 64 draft states, candidate width 6; drawn cases spread around them.
"""

import math

import torch

own = False

EPS = 1e-6
E4M3_MAX = 448.0


def _norm(name, dtype, rows, d, **more):
    # q8: -1 no 8-bit output, 0 a scale per row, else columns per scale;
    # pad: columns between one row of the input and the next
    return dict(dict(name=name, kind="norm", dtype=dtype, rows=rows, d=d, residual=True, out=True, q8=-1, pad=0),
                **more)


def _quantize(name, dtype, n_out, n_in, group, symmetric):
    return dict(name=name, kind="quantize", dtype=dtype, n_out=n_out, n_in=n_in, group=group, symmetric=symmetric)


def _linear(name, x, rows, n_out, n_in, group, **more):
    # x: bf16, fp32 or e4m3; x_group: e4m3's columns per scale (0: a scale per row)
    return dict(dict(name=name, kind="linear", x=x, rows=rows, n_out=n_out, n_in=n_in, group=group, x_group=0,
                     zeros=False, bias=False, out="fp32"), **more)


def _scores(name, kind, dtype, rows, vocab, tokens, top_k, **more):
    # hot: a temperature per row; allowed: a mask of allowed tokens, `empty`
    # the share of rows that it leaves nothing; pad: columns between rows
    return dict(dict(name=name, kind=kind, dtype=dtype, rows=rows, vocab=vocab, tokens=tokens, top_k=top_k,
                     hot=False, allowed=False, empty=0.0, pad=0), **more)


def listed():
    return [
        # One state at the end of a decoding step, its 8-bit row for the head.
        _norm("norm-one-state", "bf16", 1, 4096, q8=0, out=False),
        # The tokens of a prefill batch, 8-bit output in groups beside the bf16 one.
        _norm("norm-prefill", "bf16", 8192, 5120, q8=128),
        # A layer's weights laid out once, symmetric codes.
        _quantize("quantize-layer", "bf16", 4096, 4096, 128, True),
        # A whole head from full-precision weights, small groups with zero points.
        _quantize("quantize-head", "fp32", 32000, 4096, 32, False),
        # A projection of a drafter's block for the root and its six children.
        _linear("linear-layer", "bf16", 7, 3584, 3584, 64, zeros=True, bias=True, out="bf16"),
        # The head for a single token.
        _linear("linear-head-one-state", "bf16", 1, 32000, 4096, 128),
        # The head for one sequence's whole draft tree, 8-bit states.
        _linear("linear-head-tree", "e4m3", 64, 32000, 4096, 128, x_group=128),
        # Acceptance of one token: its log probability and the candidates.
        _scores("logprobs-one-state", "logprobs", "fp32", 1, 32000, 1, 6),
        # A draft tree under a temperature and a mask of allowed tokens.
        _scores("logprobs-tree", "logprobs", "fp32", 64, 32000, 6, 6, hot=True, allowed=True, empty=0.05),
        # A training batch's next tokens, with the margin to the sixth competitor.
        _scores("logprobs-training", "logprobs", "bf16", 4096, 32000, 1, 6),
        # The gradient of a tree's scores.
        _scores("grad-tree", "grad", "fp32", 40, 32000, 6, 6, hot=True, allowed=True, empty=0.05),
        # The gradient of the training batch.
        _scores("grad-training", "grad", "bf16", 4096, 32000, 1, 6),
    ]


def draw(rng):
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    kind = rng.choice(["norm", "quantize", "linear", "linear", "logprobs", "logprobs", "grad"])
    if kind == "norm":
        dtype = rng.choice(["bf16", "bf16", "fp32"])
        d = rng.choice([256, 3584, 4096, 5120, 8192, 64 * log_int(2, 128), log_int(100, 8192)])
        q8 = rng.choice([-1, 0, 0, 32, 64, 128])
        most = 8192 * 5120 // (d * (2 if dtype == "fp32" else 1))
        return dict(kind=kind, dtype=dtype, rows=log_int(1, min(16384, most)), d=d, residual=rng.random() < 0.8,
                    out=q8 < 0 or rng.random() < 0.5, q8=q8, pad=rng.choice([0, 0, 8, 3]))
    if kind == "quantize":
        n_in = 32 * log_int(8, 256)
        return dict(kind=kind, dtype=rng.choice(["bf16", "fp32"]), n_out=log_int(100, 32000 * 4096 // max(n_in, 4096)),
                    n_in=n_in, group=rng.choice([32, 64, 128]), symmetric=rng.random() < 0.6)
    if kind == "linear":
        n_in = rng.choice([3584, 4096, 5120, 32 * log_int(8, 256)])
        x, group = rng.choice(["bf16", "bf16", "fp32", "e4m3"]), rng.choice([32, 64, 128, 128])
        return dict(kind=kind, x=x, rows=log_int(1, 64), n_out=log_int(200, 32000 * 4096 // max(n_in, 4096)),
                    n_in=n_in, group=group, x_group=rng.choice([0, group]) if x == "e4m3" else 0,
                    zeros=rng.random() < 0.4, bias=rng.random() < 0.3, out=rng.choice(["fp32", "bf16"]))
    vocab = rng.choice([32000, log_int(1000, 160000), log_int(1000, 160000)])
    dtype = rng.choice(["bf16", "fp32"])
    most = 4096 * 32000 // (vocab * (2 if dtype == "fp32" else 1))
    allowed = rng.random() < 0.4
    return dict(kind=kind, dtype=dtype, rows=log_int(1, min(4096, most)), vocab=vocab, tokens=rng.choice([1, 1, 4, 6, 16]),
                top_k=rng.choice([0, 1, 6, 6, 10, 32]), hot=rng.random() < 0.4, allowed=allowed,
                empty=rng.choice([0.0, 0.05, 0.3]) if allowed else 0.0, pad=rng.choice([0, 0, 5, 64]))


# ---------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------

def _dtype(name):
    return {"bf16": torch.bfloat16, "fp32": torch.float32, "e4m3": torch.float8_e4m3fn}[name]


def _padded(rows, cols, pad, dtype):
    return torch.empty((rows, cols + pad), dtype=dtype, device="cuda")[:, :cols]


def _groups(n, group):
    return -(-n // group)


def _logits(case, g):
    """Logits as a head gives them: a spread of a few units and, in each row,
    a handful of tokens that stand out by another few."""
    n, v = case["rows"], case["vocab"]
    x = _padded(n, v, case["pad"], _dtype(case["dtype"]))
    step = max(1, (1 << 26) // v)
    for r in range(0, n, step):
        m = min(step, n - r)
        z = 2.0 * torch.randn((m, v), generator=g, device="cuda")
        at = torch.randint(0, v, (m, 8), generator=g, device="cuda")
        z.scatter_add_(1, at, 12.0 * torch.rand((m, 8), generator=g, device="cuda"))
        x[r:r + m] = z.to(x.dtype)
    return x


def _bits(keep):
    """[N, V] truth values as words of 32, the lowest token in the lowest bit."""
    n, v = keep.shape
    full = torch.zeros((n, _groups(v, 32) * 32), dtype=torch.int64, device=keep.device)
    full[:, :v] = keep
    words = (full.view(n, -1, 32) << torch.arange(32, device=keep.device)).sum(-1)
    return torch.where(words >= 1 << 31, words - (1 << 32), words).to(torch.int32)


def _score_inputs(case, g):
    n, v = case["rows"], case["vocab"]
    s = dict(logits=_logits(case, g), row_scale=None, allowed=None)
    # a token of -1 stands for none (a tree node with fewer children)
    tokens = torch.randint(0, v, (n, case["tokens"]), generator=g, device="cuda")
    none = torch.rand((n, case["tokens"]), generator=g, device="cuda") < 0.1
    s["tokens"] = torch.where(none, -1, tokens).to(torch.int32)
    if case["hot"]:
        t = torch.empty(n, device="cuda").uniform_(math.log(0.5), math.log(2.0), generator=g)
        s["row_scale"] = torch.exp(-t)
    if case["allowed"]:
        keep = torch.rand((n, v), generator=g, device="cuda") < 0.5
        keep &= torch.rand((n, 1), generator=g, device="cuda") >= case["empty"]
        s["allowed"] = _bits(keep)
    return s


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda")

    kind, s = case["kind"], dict(case=case)
    if kind == "norm":
        n, d, dt = case["rows"], case["d"], _dtype(case["dtype"])
        s["x"] = _padded(n, d, case["pad"], dt)
        s["x"].copy_(normal(n, d))
        s["residual"] = (3.0 * normal(n, d)).to(dt) if case["residual"] else None
        s["gamma"] = (1.0 + 0.1 * normal(d)).to(dt)
    elif kind == "quantize":
        s["W"] = (normal(case["n_out"], case["n_in"]) * case["n_in"] ** -0.5).to(_dtype(case["dtype"]))
    elif kind == "linear":
        n, k, o, group = case["rows"], case["n_in"], case["n_out"], case["group"]
        s["codes"] = torch.randint(0, 256, (o, k // 2), generator=g, device="cuda", dtype=torch.uint8)
        gs = _groups(k, group)
        s["scales"] = ((0.3 + 0.1 * torch.rand((o, gs), generator=g, device="cuda")) * k ** -0.5).to(torch.bfloat16)
        s["zeros"] = (torch.randint(5, 11, (o, gs), generator=g, device="cuda", dtype=torch.uint8)
                      if case["zeros"] else None)
        s["bias"] = 0.01 * normal(o) if case["bias"] else None
        x, s["x_scale"] = normal(n, k), None
        if case["x"] == "e4m3":
            xg = case["x_group"] or k
            full = torch.nn.functional.pad(x, (0, _groups(k, xg) * xg - k)).view(n, -1, xg)
            scale = full.abs().amax(-1) / E4M3_MAX
            x = (full / scale[..., None]).reshape(n, -1)[:, :k].clamp(-E4M3_MAX, E4M3_MAX)
            s["x_scale"] = scale if case["x_group"] else scale.view(n)
        s["x"] = x.to(_dtype(case["x"]))
    else:
        s.update(_score_inputs(case, g))
        if kind == "grad":
            n, k = case["rows"], case["top_k"]
            # what the forward pass left, and the gradients that reach it
            f = _logprobs(s["logits"], s["tokens"], k, s["row_scale"], s["allowed"])
            s.update(stats=f["stats"], entropy=f["entropy"], top_idx=f.get("top_idx"))
            s["grad_logprobs"] = normal(n, case["tokens"]) / n
            s["grad_top"] = 0.1 * normal(n, k) / n if k else None
            s["grad_entropy"] = 0.1 * normal(n) / n
            s["grad_lse"] = 0.01 * normal(n) / n
    return s


# ---------------------------------------------------------------------------
# Plain forms: elementary operations in 32 bits
# ---------------------------------------------------------------------------

def _pad_groups(x, group):
    n = x.shape[-1]
    return torch.nn.functional.pad(x, (0, _groups(n, group) * group - n)).unflatten(-1, (-1, group))


def _plain_norm(x, residual, gamma, q8, want_out):
    s = x.float() if residual is None else x.float() + residual.float()
    y = s * torch.rsqrt((s * s).mean(-1, keepdim=True) + EPS) * gamma.float()
    out = dict(sum=s.to(x.dtype) if residual is not None else None, out=y.to(x.dtype) if want_out else None)
    if q8 >= 0:
        g = _pad_groups(y, q8 or y.shape[1])
        scale = g.abs().amax(-1) / E4M3_MAX
        q = torch.where(scale[..., None] > 0, g / scale[..., None], 0.0).clamp(-E4M3_MAX, E4M3_MAX)
        out["q8"] = q.flatten(1)[:, :y.shape[1]].to(torch.float8_e4m3fn)
        out["q8_scale"] = scale if q8 else scale.view(-1)
    return out


def _plain_quantize(W, group, symmetric):
    w = _pad_groups(W.float(), group)
    if symmetric:
        scale = (w.abs().amax(-1) / w.new_tensor([7.0])).to(torch.bfloat16)
        low, zero = -8.0, 8.0
    else:
        lo, hi = w.amin(-1).clamp(max=0.0), w.amax(-1).clamp(min=0.0)
        scale = ((hi - lo) / w.new_tensor([15.0])).to(torch.bfloat16)
        zeros = torch.where(scale > 0, torch.round(-lo / scale.float()), 8.0).clamp(0.0, 15.0)
        low, zero = -zeros[..., None], zeros[..., None]
    f = scale.float()[..., None]
    q = torch.where(f > 0, torch.round(w / f), 0.0)
    q = (torch.maximum(torch.minimum(q, low + 15.0), low) if not symmetric else q.clamp(low, low + 15.0)) + zero
    q = q.to(torch.uint8).flatten(1)[:, :W.shape[1]]
    return dict(codes=q[:, 0::2] | (q[:, 1::2] << 4), scales=scale,
                zeros=None if symmetric else zeros.to(torch.uint8))


def _plain_linear(x, codes, scales, zeros, group, x_scale, bias, out):
    k = x.shape[1]
    q = torch.stack((codes & 15, codes >> 4), -1).flatten(1).float()
    z = 8.0 if zeros is None else zeros.float().repeat_interleave(group, 1)[:, :k]
    w = (q - z) * scales.float().repeat_interleave(group, 1)[:, :k]
    x = x.float()
    if x_scale is not None:
        x = x * (x_scale[:, None] if x_scale.dim() == 1 else x_scale.repeat_interleave(group, 1)[:, :k])
    y = x @ w.T
    if bias is not None:
        y = y + bias
    return y.to(out)


def _plain_scaled(logits, row_scale, allowed):
    """The allowed logits in 32 bits (-inf elsewhere), and times the rows' scales."""
    x = logits.float()
    if allowed is not None:
        bit = torch.arange(32, dtype=torch.int32, device=x.device)
        keep = ((allowed[:, :, None] >> bit) & 1).flatten(1)[:, :x.shape[1]] != 0
        x = torch.where(keep, x, -math.inf)
    return x, x if row_scale is None else x * row_scale[:, None]


def _logprobs(logits, tokens, k, row_scale, allowed):
    x, z = _plain_scaled(logits, row_scale, allowed)
    m = z.amax(-1, keepdim=True)
    none = m == -math.inf                               # a row without tokens
    z = z - torch.where(none, 0.0, m)
    e = torch.exp(z)
    total = e.sum(-1, keepdim=True)
    log_sum = torch.log(total)
    lp = z - torch.where(none, 0.0, log_sum)
    entropy = -torch.where(e > 0, e / total * lp, 0.0).sum(-1)
    at = tokens.long()
    given = torch.where(at >= 0, lp.gather(1, at.clamp(min=0)), 0.0)
    out = dict(logprobs=given, lse=(m + log_sum)[:, 0], entropy=entropy, stats=torch.cat((m, log_sum), 1))
    if k:
        # distinct keys: the logit's bits in order, then the lower token first
        bits = (x + 0.0).view(torch.int32).long()
        bits = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits)
        key = bits * (1 << 32) + (0xFFFFFFFF - torch.arange(x.shape[1], device=x.device))
        top = 0xFFFFFFFF - (torch.topk(key, k, dim=-1).values & 0xFFFFFFFF)
        value = lp.gather(1, top)
        out["top_idx"] = torch.where(value > -math.inf, top, -1).to(torch.int32)
        out["top_logprobs"] = value
    return out


def _plain_grad(s):
    _, z = _plain_scaled(s["logits"], s["row_scale"], s["allowed"])
    stats = torch.where(s["stats"] == -math.inf, 0.0, s["stats"])
    lp = (z - stats[:, :1]) - stats[:, 1:]
    p = torch.exp(lp)
    at, g = s["tokens"].long(), s["grad_logprobs"]
    if s["grad_top"] is not None:
        at, g = torch.cat((at, s["top_idx"].long()), 1), torch.cat((g, s["grad_top"]), 1)
    # a token that is none, or that has no probability, counts for nothing
    counted = (at >= 0) & (lp.gather(1, at.clamp(min=0)) > -math.inf)
    at, g = at.clamp(min=0), torch.where(counted, g, 0.0)
    dz = p * (s["grad_lse"][:, None] - g.sum(-1, keepdim=True))
    dz -= torch.where(p > 0, s["grad_entropy"][:, None] * p * (lp + s["entropy"][:, None]), 0.0)
    dz.scatter_add_(1, at, g)
    if s["row_scale"] is not None:
        dz *= s["row_scale"][:, None]
    return dz.to(s["logits"].dtype)


# ---------------------------------------------------------------------------
# One pass
# ---------------------------------------------------------------------------

def run(s):
    case = s["case"]
    kind = case["kind"]
    if own:
        from paper_2608_22883_gb300 import fovea
        if kind == "norm":
            return fovea.add_rms_norm(s["x"], s["gamma"], s["residual"], eps=EPS, want_out=case["out"],
                                      q8_group=case["q8"] if case["q8"] >= 0 else None)
        if kind == "quantize":
            return fovea.quantize_w4(s["W"], case["group"], symmetric=case["symmetric"])
        if kind == "linear":
            return fovea.linear_w4(s["x"], s["codes"], s["scales"], s["zeros"], group=case["group"],
                                   x_scale=s["x_scale"], bias=s["bias"], out_dtype=_dtype(case["out"]))
        if kind == "logprobs":
            return fovea.token_logprobs(s["logits"], s["tokens"], case["top_k"], row_scale=s["row_scale"],
                                        allowed=s["allowed"])
        return fovea.token_logprobs_grad(s["logits"], s["stats"], s["entropy"], tokens=s["tokens"],
                                         grad_logprobs=s["grad_logprobs"], top_idx=s["top_idx"],
                                         grad_top=s["grad_top"], grad_entropy=s["grad_entropy"],
                                         grad_lse=s["grad_lse"], row_scale=s["row_scale"], allowed=s["allowed"])
    if kind == "norm":
        return _plain_norm(s["x"], s["residual"], s["gamma"], case["q8"], case["out"])
    if kind == "quantize":
        return _plain_quantize(s["W"], case["group"], case["symmetric"])
    if kind == "linear":
        return _plain_linear(s["x"], s["codes"], s["scales"], s["zeros"], case["group"], s["x_scale"], s["bias"],
                             _dtype(case["out"]))
    if kind == "logprobs":
        return _logprobs(s["logits"], s["tokens"], case["top_k"], s["row_scale"], s["allowed"])
    return _plain_grad(s)


# ---------------------------------------------------------------------------
# The same from the definitions in 64 bits, a block of rows at a time
# ---------------------------------------------------------------------------

def _exact_norm(s, case):
    v = s["x"].double()
    if s["residual"] is not None:
        v = v + s["residual"].double()
    y = v / (v.pow(2).sum(1, keepdim=True) / v.shape[1] + EPS).sqrt() * s["gamma"].double()
    r = dict(sum=v if s["residual"] is not None else None, out=y if case["out"] else None)
    if case["q8"] >= 0:
        width = case["q8"] or case["d"]
        parts = [p.abs().max(1).values / E4M3_MAX for p in y.split(width, 1)]
        scale = torch.stack(parts, 1)
        full = scale.repeat_interleave(width, 1)[:, :case["d"]]
        r["q8"] = torch.where(full > 0, y / full, 0.0)      # what the 8 bits stand for, unrounded
        r["q8_scale"] = scale if case["q8"] else scale[:, 0]
    return r


def _exact_quantize(s, case):
    parts = s["W"].double().split(case["group"], 1)
    if case["symmetric"]:
        scale = [p.abs().max(1).values / 7 for p in parts]
    else:
        scale = [(p.max(1).values.clamp(min=0) - p.min(1).values.clamp(max=0)) / 15 for p in parts]
    return dict(codes=None, scales=torch.stack(scale, 1), zeros=None)


def _exact_linear(s, case):
    group, x = case["group"], s["x"].double()
    if s["x_scale"] is not None:
        xs = s["x_scale"].double().view(case["rows"], -1)
        x = x * (xs.repeat_interleave(group, 1)[:, :case["n_in"]] if case["x_group"] else xs)
    y = torch.empty((case["rows"], case["n_out"]), dtype=torch.float64, device="cuda")
    for o in range(0, case["n_out"], 4096):
        c = s["codes"][o:o + 4096]
        w = torch.empty((c.shape[0], case["n_in"]), dtype=torch.float64, device="cuda")
        w[:, 0::2], w[:, 1::2] = (c % 16).double(), (c // 16).double()
        zero = s["zeros"][o:o + 4096].double() if s["zeros"] is not None else torch.full_like(s["scales"][o:o + 4096], 8.0).double()
        for i in range(_groups(case["n_in"], group)):
            at = slice(i * group, (i + 1) * group)
            w[:, at] = (w[:, at] - zero[:, i:i + 1]) * s["scales"][o:o + 4096, i:i + 1].double()
        y[:, o:o + 4096] = x @ w.T
    return y if s["bias"] is None else y + s["bias"].double()


def _exact_rows(s, r0, r1):
    """Some rows' logits in 64 bits (-inf where not allowed), logp, p, lse, (largest, log sum) and entropy."""
    x = s["logits"][r0:r1].double()
    if s["allowed"] is not None:
        words = s["allowed"][r0:r1].long() & 0xFFFFFFFF
        token = torch.arange(x.shape[1], device="cuda")
        x = x.masked_fill((words[:, token // 32] >> (token % 32)) % 2 == 0, -math.inf)
    z = x if s["row_scale"] is None else x * s["row_scale"][r0:r1].double()[:, None]
    lse = torch.logsumexp(z, 1)
    lp = z - lse.nan_to_num(neginf=0.0)[:, None]
    p = lp.exp()
    top = z.max(1).values
    stats = torch.stack((top, lse - top.nan_to_num(neginf=0.0)), 1)
    return x, lp, p, lse, stats, -(p * lp.clamp(min=-1e300)).sum(1)


def _exact_scores(s, case):
    got = []
    step = max(1, (1 << 25) // case["vocab"])
    for r in range(0, case["rows"], step):
        x, lp, _, lse, stats, entropy = _exact_rows(s, r, r + step)
        t = s["tokens"][r:r + step].long()
        o = dict(logprobs=lp.gather(1, t.clamp(min=0)).masked_fill(t < 0, 0.0), lse=lse, stats=stats, entropy=entropy)
        if case["top_k"]:
            order = x.sort(dim=1, descending=True, stable=True).indices[:, :case["top_k"]]
            o["top_logprobs"] = lp.gather(1, order)
            o["top_idx"] = order.masked_fill(o["top_logprobs"] == -math.inf, -1).int()
        got.append(o)
    return {name: torch.cat([o[name] for o in got]) for name in got[0]}


def _exact_grad(s, case):
    # in the logits' width: 64 bits of the whole would not fit beside the rest
    got = []
    step = max(1, (1 << 25) // case["vocab"])
    for r in range(0, case["rows"], step):
        _, lp, p, _, _, entropy = _exact_rows(s, r, r + step)
        dz = p * s["grad_lse"][r:r + step].double()[:, None]
        dz -= s["grad_entropy"][r:r + step].double()[:, None] * p * (lp.clamp(min=-1e300) + entropy[:, None])
        pairs = [(s["tokens"], s["grad_logprobs"])]
        if case["top_k"]:
            pairs.append((s["top_idx"], s["grad_top"]))
        for ids, grads in pairs:
            for j in range(ids.shape[1]):
                i, w = ids[r:r + step, j].long(), grads[r:r + step, j].double()
                at = i.clamp(min=0)[:, None]
                w = torch.where((i >= 0) & (lp.gather(1, at)[:, 0] > -math.inf), w, 0.0)[:, None]
                dz -= p * w
                dz.scatter_add_(1, at, w)
        if s["row_scale"] is not None:
            dz *= s["row_scale"][r:r + step].double()[:, None]
        got.append(dz.to(torch.float32))
    return torch.cat(got)


def exact(case, seed):
    s = prepare(case, seed)
    return {"norm": _exact_norm, "quantize": _exact_quantize, "linear": _exact_linear, "logprobs": _exact_scores,
            "grad": _exact_grad}[case["kind"]](s, case)


# ---------------------------------------------------------------------------
# What a pass cannot do without
# ---------------------------------------------------------------------------

def work(case):
    kind = case["kind"]
    size = {"bf16": 2, "fp32": 4, "e4m3": 1}
    if kind == "norm":
        n, d, b = case["rows"], case["d"], size[case["dtype"]]
        moved = n * d * b * (1 + 2 * case["residual"] + case["out"]) + d * b
        if case["q8"] >= 0:
            moved += n * d + 4 * n * (_groups(d, case["q8"]) if case["q8"] else 1)
        return dict(bytes=moved, flops=6 * n * d)
    if kind == "quantize":
        o, k, gs = case["n_out"], case["n_in"], _groups(case["n_in"], case["group"])
        return dict(bytes=o * k * size[case["dtype"]] + o * k // 2 + o * gs * (2 if case["symmetric"] else 3),
                    flops=3 * o * k)
    if kind == "linear":
        n, o, k, gs = case["rows"], case["n_out"], case["n_in"], _groups(case["n_in"], case["group"])
        xs = 4 * n * (gs if case["x_group"] else 1) if case["x"] == "e4m3" else 0
        return dict(bytes=o * k // 2 + o * gs * (3 if case["zeros"] else 2) + n * k * size[case["x"]] + xs
                    + (4 * o if case["bias"] else 0) + n * o * size[case["out"]], flops=2 * n * o * k)
    n, v = case["rows"], case["vocab"]
    moved = n * v * size[case["dtype"]] * (2 if kind == "grad" else 1)
    if case["allowed"]:
        moved += 4 * n * _groups(v, 32)
    moved += n * (8 * (case["tokens"] + case["top_k"]) + 16)
    return dict(bytes=moved, flops=(8 if kind == "grad" else 6) * n * v)
