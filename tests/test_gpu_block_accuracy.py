"""Where the operators that run, train and evaluate refined layers could lose accuracy:
tails and cancellations, against float64 with bounds relative to the small result itself.
E = 2^-24 is half a unit in the last place of fp32."""

import numpy as np
import pytest
import torch

from paper_2609_38599_amd import binding as jb
from tests._gpu_common import say

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]

E = 2.0 ** -24


def _randn(seed, *shape, std=1.0):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed)) * std


# ---- log probabilities where one entry takes nearly all ----

LEADS = [(9, 32001, torch.float32), (9, 32001, torch.bfloat16), (9, 4100, torch.float16),
         (1, 128000, torch.float32), (2, 50257, torch.bfloat16), (600, 1001, torch.float32),
         (3, 5, torch.float32)]


def _leading(T, V, dt, lead, offset):
    """Logits whose entry at targets[t] is `lead` above the others' maximum, moved by `offset`."""
    x = _randn(T + V, T, V, std=2.0).to(dt).double()
    t = (torch.arange(T) * 7919 + V // 3) % V
    rows = torch.arange(T)
    x[rows, t] = -float("inf")
    x[rows, t] = x.max(1).values + lead
    return (x + offset).to(dt), t


def _others(x, t):
    """Per row, in float64: d = x - x_target beside the target, sum exp d, sum exp(d) d."""
    d = x.double()
    rows = torch.arange(len(t))
    d = d - d[rows, t][:, None]
    d[rows, t] = -float("inf")
    e = torch.exp(d)
    return d, e.sum(1), (e * torch.where(e > 0, d, 0.0)).sum(1)


def _sums(V):
    # exp off by (|d| + 1) e for |d| up to 60 here, a lane's sum of V / 256, some joins
    return (V / 256 + 80) * 2 * E


@pytest.mark.parametrize("lead", [8.0, 18.0, 22.0, 25.0])
@pytest.mark.parametrize("T,V,dt", LEADS)
def test_logprob_of_a_leading_token(T, V, dt, lead):
    # log p = -log(1 + s), s the others' sum: off by what s is, not by E
    for offset in (0.0, 100.0):
        say(f"[logprob lead] tokens {T} vocab {V} {dt} lead {lead} offset {offset}")
        x, t = _leading(T, V, dt, lead, offset)
        _, s, sd = _others(x, t)
        r = jb.token_logprobs(x.cuda(), t.cuda())
        want = -torch.log1p(s)
        off = (r.logprob.cpu().double() - want).abs() / want.abs()
        assert float(off.max()) <= _sums(V) + 4 * E
        want = torch.log1p(s) - sd / (1 + s)
        off = (r.entropy.cpu().double() - want).abs() / want
        assert float(off.max()) <= 2 * _sums(V) + 8 * E
