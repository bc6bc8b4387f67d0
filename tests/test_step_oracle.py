"""Pins of the float64 definitions of the operators around a block, on the CPU."""

import numpy as np
import pytest
import torch

from oracle import step


def _rng(seed):
    return np.random.default_rng(seed)


def test_norm_is_torchs_and_its_gradient_autograds():
    r = _rng(0)
    X, gain, dY, dH = r.normal(size=(5, 37)), r.normal(size=37), r.normal(size=(5, 37)), r.normal(size=(5, 37))
    x, g = (torch.from_numpy(a).requires_grad_() for a in (X, gain))
    y = torch.nn.functional.rms_norm(x, (37,), g, eps=1e-3)
    assert np.allclose(step.norm(X, gain, 1e-3)[0], y.detach().numpy(), rtol=1e-13)
    want = torch.autograd.grad((y * torch.from_numpy(dY)).sum() + (x * torch.from_numpy(dH)).sum(), (x, g))
    for a, b in zip(step.norm_grad(X, gain, dY, dH, 1e-3), want):
        assert np.allclose(a, b.numpy(), rtol=1e-12, atol=1e-13)


def test_norm_i8_stands_for_the_norm():
    r = _rng(1)
    H, gain = r.normal(size=(4, 64)).astype(np.float32), r.normal(size=64).astype(np.float32)
    Q, scale = step.norm_i8(H, gain, 1e-6)
    y = step.norm(H.astype(np.float64), gain, 1e-6)[0]
    # half an integer, and the fp32 roundings of a product of up to 127
    assert np.all(np.abs(Q * scale[:, None] - y) <= (0.5 + 127 * 3 * 2.0 ** -24) * scale[:, None])
    assert np.all(np.abs(Q).max(axis=1) == 127)


def test_linear_logprobs_are_torchs():
    r = _rng(2)
    X, W = r.normal(size=(6, 16)), r.normal(size=(11, 16))
    targets, g, h = np.array([0, 10, -1, 3, 3, -5]), r.normal(size=6), r.normal(size=6)
    x, w = (torch.from_numpy(a).requires_grad_() for a in (X, W))
    logits = x @ w.T
    lse = torch.logsumexp(logits, 1)
    lp = torch.stack([logits[t, v] - lse[t] if v >= 0 else torch.zeros((), dtype=torch.float64)
                      for t, v in enumerate(targets)])
    got = step.linear_logprobs(X, W, targets)
    assert np.allclose(got[0], lp.detach().numpy(), rtol=1e-12) and np.allclose(got[1], lse.detach().numpy())
    want = torch.autograd.grad((lp * torch.from_numpy(g)).sum() + (lse * torch.from_numpy(h)).sum(), (x, w))
    for a, b in zip(step.linear_logprobs_grad(X, W, targets, g, h), want):
        assert np.allclose(a, b.numpy(), rtol=1e-11, atol=1e-13)


def test_e4m3_is_torchs():
    codes = np.arange(256, dtype=np.uint8)
    want = torch.from_numpy(codes).view(torch.float8_e4m3fn).float().numpy()
    assert np.array_equal(step.e4m3(codes), want.astype(np.float64), equal_nan=True)


def test_adamw_is_torchs():
    r = _rng(3)
    p0 = r.normal(size=200)
    p = torch.from_numpy(p0.copy()).requires_grad_()
    opt = torch.optim.AdamW([p], lr=0.01, betas=(0.8, 0.95), eps=1e-6, weight_decay=0.1)
    m = v = np.zeros(200)
    mine = p0
    for t in range(1, 6):
        g = r.normal(size=200)
        p.grad = torch.from_numpy(g)
        opt.step()
        m, v = 0.8 * m + 0.2 * g, 0.95 * v + 0.05 * g * g
        mine = step.adamw(mine, m, v, t, 0.01, 0.8, 0.95, 1e-6, 0.1)
        assert np.allclose(mine, p.detach().numpy(), rtol=1e-12)


@pytest.mark.parametrize("positive", [False, True])
def test_encoding_rounds_to_a_neighbour_and_right_on_average(positive):
    r = _rng(4)
    x = (r.normal(size=128) * np.exp(3 * r.normal(size=128))).astype(np.float32)
    if positive:
        x = np.abs(x)
    n = 4096
    every = np.tile(x, n)
    low, high = step.noise(np.arange(every.size), seed=5, step=3)
    codes, exps = step.encode(every, high if positive else low, positive)
    got = step.decode(codes, exps).astype(np.float64).reshape(n, 128)
    size = np.ldexp(1.0, int(exps[0]) - 134)
    # a unit in the last place of e4m3 at x: 2^-3 of its binade, 2^-9 of the block at least
    unit = np.maximum(np.ldexp(1.0, np.frexp(np.abs(x))[1] - 4), 2.0 ** -9 * size)
    assert np.all(np.abs(got - x) < unit)
    kept = np.abs(x) >= 2.0 ** -9 * size          # (below, what is above 0 is put at 2^-9)
    # the mean of n roundings with a variance of a quarter of a unit squared at most
    assert np.all(np.abs(got.mean(axis=0) - x)[kept] <= 5 * 0.5 * unit[kept] / np.sqrt(n))
    if positive:
        assert np.all(got[:, x > 0] > 0)


def test_encoding_by_hand():
    x = np.zeros(128, dtype=np.float32)
    x[:7] = [1.0, -1.0625, 0.015625, 2.0 ** -16, -2.0 ** -16, 2.0 ** -17, 1.9375]
    nothing, most = np.zeros(128), np.full(128, 65535)
    codes, exps = step.encode(x, nothing, False)
    assert exps[0] == 127                      # 1.9375 in 2^0..2^1: the scale is 2^-7
    v = step.decode(codes, exps)
    assert list(v[:7]) == [1.0, -1.0, 0.015625, 2.0 ** -16, -2.0 ** -16, 0.0, 1.875]
    codes, exps = step.encode(x, most, False)
    v = step.decode(codes, exps)
    assert list(v[:7]) == [1.0, -1.125, 0.015625, 2.0 ** -16, -2.0 ** -16, 2.0 ** -16, 2.0]
    codes, _ = step.encode(np.abs(x), nothing, True)
    assert codes[5] == 1 and codes[7] == 0
    x[9] = np.inf
    codes, exps = step.encode(x, nothing, False)
    assert np.all(codes == 0x7F) and exps[0] == 255 and np.all(np.isnan(step.decode(codes, exps)))


def test_moments_in_8_bits_follow_those_in_32():
    # to nearest, sqrt(v) would stay where it is: a step moves it by 1/2000 of itself
    r = _rng(6)
    n, steps = 128 * 8, 3000
    scale = np.exp(r.normal(size=n))
    m8 = v8 = np.zeros(n, dtype=np.uint8)
    me = ve = np.ones(n // 128, dtype=np.uint8)
    v = np.zeros(n)
    for t in range(1, steps + 1):
        g = (r.normal(size=n) * scale * (3.0 if t < 1000 else 1.0)).astype(np.float32)
        root = step.decode(v8, ve)
        m1, _, r1 = step.moments(g, step.decode(m8, me), root * root, 0.9, 0.999)
        low, high = step.noise(np.arange(n), 1, t)
        m8, me = _encode_fast(m1, low, False)
        v8, ve = _encode_fast(r1, high, True)
        v = 0.999 * v + 0.001 * g.astype(np.float64) ** 2
    ratio = step.decode(v8, ve) / np.sqrt(v)
    # a step moves sqrt(v) by d = 1/2000 of itself where e4m3's unit is s = 1/16 to 1/8: it is rounded
    # up with a probability of d / s, a variance of d s, and forgotten in 1 / (2 d) steps: a deviation of
    # sqrt(s / 2) = 0.18 to 0.25, and a mean that is off by less than half its square
    assert abs(np.log(ratio).mean()) < 0.05 and np.log(ratio).std() < 0.3


def _encode_fast(x, noise16, positive):
    """step.encode for all blocks at once, by the fp32 form's bits."""
    b = x.reshape(-1, 128)
    field = np.maximum(np.abs(b).max(axis=1).view(np.int32) >> 23, 1)
    s = np.ldexp(np.abs(b).astype(np.float64), 14 - field[:, None]).astype(np.float32)
    code = (s.view(np.int32) + (noise16.reshape(b.shape).astype(np.int32) << 4)) >> 20
    if positive:
        code = np.where((b > 0) & (code == 0), 1, code)
    code = np.where(b < 0, code | 0x80, code)
    return code.astype(np.uint8).reshape(-1), field.astype(np.uint8)


@pytest.mark.parametrize("positive", [False, True])
def test_encoding_is_that_of_the_bits(positive):
    r = _rng(7)
    x = (r.normal(size=128 * 40) * np.exp(8 * r.normal(size=128 * 40))).astype(np.float32)
    x[:128] *= np.float32(2.0 ** -120)          # blocks of subnormal numbers
    x[128:256] *= np.float32(1e-38)
    x[300] = 0.0
    x = np.abs(x) if positive else x
    noise16 = step.noise(np.arange(x.size), 2, 9)[int(positive)]
    for a, b in zip(step.encode(x, noise16, positive), _encode_fast(x, noise16, positive)):
        assert np.array_equal(a, b)
