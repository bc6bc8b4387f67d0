"""A few steps of recovery training of a quantized block, its moments in 8 bits.

A synthetic block (norm, gate, up and down projections, norm, head) whose projections have
been rounded to a few bits is trained towards the tokens that the original one predicts:

1. forward: norm, gated block, down, norm with the residual's addition, and the log
   probabilities of the tokens straight from the hidden states (no logits in memory);
2. backward through the same operators;
3. one step of AdamW over all weights at once, the gradients clipped on the device.

At the end the block runs once in 8-bit integers: the norm's integers go straight into the
product with gate's.

    python examples/recovery_step.py [--tokens 512 --d 512 --f 1024 --vocab 8000 --steps 10]
"""

from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2609_38599_amd import binding as jb  # noqa: E402


def forward(x, w, targets):
    """The log probabilities and what the backward pass takes."""
    n1 = jb.rms_norm(x, w["norm1"])
    h, pre = jb.gated_forward(n1, w["gate"], w["up"], save=True)
    n2, s = jb.rms_norm(h @ w["down"].t(), w["norm2"], residual=x)
    return jb.linear_logprobs(n2, w["head"], targets), (n1, h, pre, n2, s)


def backward(x, w, targets, r, kept, g):
    """The gradients of all weights for g, that of the log probabilities."""
    n1, h, pre, n2, s = kept
    d_n2, d_head = jb.linear_logprobs_backward(n2, w["head"], targets, r, g)
    d_s, d_norm2 = jb.rms_norm_backward(s, w["norm2"], d_n2)
    d_n1, d_gate, d_up = jb.gated_backward(n1, w["gate"], w["up"], d_s @ w["down"], pre)
    _, d_norm1 = jb.rms_norm_backward(x, w["norm1"], d_n1, need=(False, True))
    return {"norm1": d_norm1, "gate": d_gate, "up": d_up, "down": d_s.t().contiguous() @ h,
            "norm2": d_norm2, "head": d_head}


def main(tokens=512, d=512, f=1024, vocab=8000, steps=10, bits=3, lr=1e-3, seed=0, log=print):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    bf16 = torch.bfloat16

    def randn(*shape, std=1.0):
        return (torch.randn(*shape, generator=gen, device="cuda") * std).to(bf16)

    x = randn(tokens, d)
    w = {"norm1": torch.ones(d, dtype=bf16, device="cuda"), "gate": randn(f, d, std=d ** -0.5),
         "up": randn(f, d, std=d ** -0.5), "down": randn(d, f, std=f ** -0.5),
         "norm2": torch.ones(d, dtype=bf16, device="cuda"), "head": randn(vocab, d, std=2 * d ** -0.5)}
    nothing = torch.zeros(tokens, dtype=torch.int64, device="cuda")
    targets = (forward(x, w, nothing)[1][3] @ w["head"].t()).argmax(1)
    log(f"original: loss {-forward(x, w, targets)[0].logprob.mean().item():.4f}")

    for name in ("gate", "up", "down"):   # each row on 2^bits values
        row = w[name].float()
        step = row.abs().amax(1, keepdim=True) / (2 ** (bits - 1) - 0.5)
        w[name] = (((row / step - 0.5).round() + 0.5) * step).to(bf16)

    names = list(w)
    params = [w[n] for n in names]
    state = jb.adamw_state(params, bits=8)
    g = torch.full((tokens,), -1.0 / tokens, device="cuda")
    losses = []
    for t in range(1, steps + 1):
        r, kept = forward(x, w, targets)
        losses.append(-r.logprob.mean().item())
        grads = backward(x, w, targets, r, kept, g)
        grads = [grads[n] for n in names]
        norm = torch.stack([a.float().norm() for a in grads]).norm()
        jb.adamw_step(params, grads, state, t, lr, grad_mul=(1.0 / norm).clamp_max(1.0), seed=seed)
    losses.append(-forward(x, w, targets)[0].logprob.mean().item())
    log("loss " + " ".join(f"{v:.4f}" for v in losses))

    q, scale = jb.rms_norm_i8(x, w["norm1"])
    a = jb.matmul_i8(q, scale, *jb.quant_rows_i8(w["gate"]))
    want = jb.rms_norm(x, w["norm1"]).float() @ w["gate"].float().t()
    off = ((a.float() - want).norm() / want.norm()).item()
    log(f"gate in 8-bit integers: {100 * off:.2f} % off")
    return {"losses": losses, "off": off}


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    for name, value in (("tokens", 512), ("d", 512), ("f", 1024), ("vocab", 8000), ("steps", 10),
                        ("bits", 3), ("seed", 0)):
        ap.add_argument(f"--{name}", type=int, default=value)
    ap.add_argument("--lr", type=float, default=1e-3)
    main(**vars(ap.parse_args()))
