"""The drafter's exit with 4-bit weights, end to end on one GPU.

A draft tree's states leave the drafter's last block; the block's output joins the
residual stream, the norm writes 8-bit rows, a 4-bit head gives logits, and these
give what a program needs to grow, accept or train on the tree: candidates with
their log probabilities, log probabilities of given tokens, entropies, and the
gradient of a training objective (cross entropy, a margin to the K_c-th competitor
and an entropy bonus).  Weights and states are random.

    python examples/quantized_exit.py [--rows 64] [--d 4096] [--vocab 32000]
"""

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2608_22883_gb300 import fovea  # noqa: E402

K_C = 6              # candidate width of the draft tree


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--rows", type=int, default=64)
    ap.add_argument("--d", type=int, default=4096)
    ap.add_argument("--vocab", type=int, default=32000)
    a = ap.parse_args()
    g = torch.Generator(device="cuda")
    g.manual_seed(0)

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda")

    # once: the head's weights in 4 bits
    W = (normal(a.vocab, a.d) * a.d ** -0.5).to(torch.bfloat16)
    head = fovea.quantize_w4(W, group=128)
    print(f"head: {W.numel() * 2 / 1e6:.1f} MB in bf16, "
          f"{(head['codes'].numel() + 2 * head['scales'].numel()) / 1e6:.1f} MB in 4 bits")

    # each expansion: block output + residual -> norm -> head -> scores
    block, stream, gamma = normal(a.rows, a.d).bfloat16(), 2 * normal(a.rows, a.d).bfloat16(), normal(a.d).bfloat16()
    tokens = torch.randint(0, a.vocab, (a.rows, 1), generator=g, device="cuda", dtype=torch.int32)
    n = fovea.add_rms_norm(block, gamma, stream, want_out=False, q8_group=128)
    logits = fovea.linear_w4(n["q8"], head["codes"], head["scales"], x_scale=n["q8_scale"])
    s = fovea.token_logprobs(logits, tokens, K_C)
    print("first state's candidates:",
          ", ".join(f"{t} ({p:.2f})" for t, p in zip(s["top_idx"][0].tolist(), s["top_logprobs"][0].tolist())))
    print(f"entropy {s['entropy'].mean().item():.3f}, log probability of the given tokens "
          f"{s['logprobs'].mean().item():.3f}")

    # the same in bf16: how far 8-bit states and 4-bit weights are from it
    full = fovea.add_rms_norm(block, gamma, stream)["out"]
    exact = full.float() @ W.float().T
    off = (logits - exact).norm() / exact.norm()
    print(f"logits against the bf16 head: {100 * off.item():.1f} % off")

    # a training step's gradient: cross entropy, margin of the given token over the K_c-th
    # competitor, entropy bonus
    margin, weight, bonus = 0.5, 0.5, 0.01
    gap = s["logprobs"][:, 0] - s["top_logprobs"][:, K_C - 1]
    loss = -s["logprobs"][:, 0] + weight * torch.nn.functional.softplus(margin - gap) - bonus * s["entropy"]
    slope = weight * torch.sigmoid(margin - gap) / a.rows
    grad_top = torch.zeros_like(s["top_logprobs"])
    grad_top[:, K_C - 1] = slope
    d = fovea.token_logprobs_grad(
        logits, s["stats"], s["entropy"], tokens=tokens, grad_logprobs=(-1.0 / a.rows - slope)[:, None].contiguous(),
        top_idx=s["top_idx"], grad_top=grad_top, grad_entropy=torch.full_like(s["entropy"], -bonus / a.rows))
    print(f"loss {loss.mean().item():.4f}; its gradient's rows sum to {d.sum(1).abs().max().item():.1e}")


if __name__ == "__main__":
    main()
