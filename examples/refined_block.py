"""A feed-forward block through refinement, calibration, evaluation and a training step.

A synthetic block (gate, up and down projections) with a head over a vocabulary:

1. gate and up are quantized and refined under the block's calibration tokens;
2. the refined gate and up run as one gated block, and its output tokens are the
   calibration of down, which is refined in turn;
3. the refined block runs with down in 8-bit integers straight from its codes, and
   the log probabilities of the next tokens compare it with the original;
4. one step of recovery: the loss's gradient goes back through the head, down and the
   gated block to the dequantized gate and up.

    python examples/refined_block.py [--tokens 512 --d 512 --f 1024 --vocab 8000]
"""

from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2609_38599_amd import binding as jb  # noqa: E402


def refine(W, X, bits, group, sweeps):
    """Codes, scales and zero points of W [rows, cols] refined under the tokens X."""
    p = jb.make_params(W.shape[0], W.shape[1], group, bits, sweeps)
    H = jb.hessian([X], W.shape[1], alpha=1.0 / X.shape[0], damp=0.01)
    codes, scales, zeros = jb.gptq(p, W, H)
    stats = jb.refine(p, W, H, codes, scales, zeros, jb.alloc_workspace(p))
    return p, codes, scales, zeros, stats["objective_after_scales"]


def main(tokens=512, d=512, f=1024, vocab=8000, bits=3, group=64, sweeps=5, seed=0, log=print):
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def randn(*shape, std=1.0):
        return torch.randn(*shape, generator=gen, device="cuda") * std

    bf16 = torch.bfloat16
    X = randn(tokens, d).to(bf16)
    gate, up = randn(f, d, std=d ** -0.5), randn(f, d, std=d ** -0.5)
    down, head = randn(d, f, std=f ** -0.5), randn(vocab, d, std=4.0 * d ** -0.5).to(bf16)

    # the original block, and tokens drawn from its own distribution
    h = jb.gated_forward(X, gate.to(bf16), up.to(bf16))
    original = (h @ down.to(bf16).t()) @ head.t()
    targets = torch.distributions.Gumbel(0.0, 1.0).sample(original.shape).cuda().add(original) \
        .argmax(1)
    base = jb.token_logprobs(original, targets, top=5)

    # 1. gate and up under the block's inputs
    layers = {}
    for name, W in (("gate", gate), ("up", up)):
        p, codes, scales, zeros, objective = refine(W, X.float(), bits, group, sweeps)
        layers[name] = jb.dequantize(p, codes, scales, zeros, dtype=bf16)
        log(f"{name}: objective {objective[0]:.4g} -> {objective[-1]:.4g}")

    # 2. down under what the refined gate and up give it
    h, pre = jb.gated_forward(X, layers["gate"], layers["up"], save=True)
    p, codes, scales, zeros, objective = refine(down, h.float(), bits, group, sweeps)
    log(f"down: objective {objective[0]:.4g} -> {objective[-1]:.4g}")

    # 3. the refined block with down in integers
    y = jb.linear_i8(h, jb.codes_i8(p, codes, zeros), scales)
    logits = y @ head.t()
    lp = jb.token_logprobs(logits, targets, top=5)
    kept = (lp.top_index[:, 0] == base.top_index[:, 0]).float().mean().item()
    log(f"perplexity {(-base.logprob.mean()).exp().item():.2f} -> "
        f"{(-lp.logprob.mean()).exp().item():.2f}, entropy {base.entropy.mean().item():.3f} -> "
        f"{lp.entropy.mean().item():.3f}, first choice kept {100 * kept:.1f} %")

    # 4. the gradient of the mean loss in gate and up (down as its dequantized weights)
    g = torch.full((tokens,), -1.0 / tokens, device="cuda")
    d_logits = jb.token_logprobs_backward(logits, targets, lp, g)
    d_h = (d_logits @ head) @ jb.dequantize(p, codes, scales, zeros, dtype=bf16)
    _, d_gate, d_up = jb.gated_backward(X, layers["gate"], layers["up"], d_h, pre,
                                        need=(False, True, True))
    # the largest weight of either moves by 0.002
    step = 0.002 / max(d_gate.abs().max().item(), d_up.abs().max().item())
    moved = [(layers[n].float() - step * dw.float()).to(bf16)
             for n, dw in (("gate", d_gate), ("up", d_up))]
    h = jb.gated_forward(X, *moved)
    after = jb.token_logprobs(jb.linear_i8(h, jb.codes_i8(p, codes, zeros), scales) @ head.t(),
                              targets)
    log(f"loss {-lp.logprob.mean().item():.4f}, after a step on gate and up "
        f"{-after.logprob.mean().item():.4f}")
    return {"base": -base.logprob.mean().item(), "refined": -lp.logprob.mean().item(),
            "after": -after.logprob.mean().item(), "kept": kept}


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    for name, value in (("tokens", 512), ("d", 512), ("f", 1024), ("vocab", 8000), ("bits", 3),
                        ("group", 64), ("sweeps", 5), ("seed", 0)):
        ap.add_argument(f"--{name}", type=int, default=value)
    main(**vars(ap.parse_args()))
