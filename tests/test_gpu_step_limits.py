"""The operators around a block on the GPU where numbers, tokens and arrays are at their limits:
gradients against what one rounding leaves, logits far from 0, targets and gradients that are none,
arrays that are written in place."""

import ctypes
import warnings

import numpy as np
import pytest
import torch
from torch.autograd import forward_ad

from oracle import step
from paper_2609_38599_amd import binding as jb
from tests._gpu_common import say
from tests.test_gpu_blocks import E, ROUND, _np, _randn
from tests.test_gpu_step import BF16, F16, F32, OPT, _linlog_inputs, _norm_inputs

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]


# ---- log probabilities: one rounding ----

def _gradients(x, w, targets, g, h):
    """(dl, dX, dW) in 64 bits on the GPU."""
    X, W = x.double(), w.double()
    logits = X @ W.t()
    has = targets >= 0
    G = torch.where(has, g, 0.0).double()
    dl = (h.double() - G)[:, None] * torch.softmax(logits, 1)
    dl.scatter_add_(1, targets.clamp_min(0)[:, None], G[:, None])
    return dl, dl @ W, dl.t() @ X


def _check_rounded_once(x, w, targets, g, h, say_at):
    # An output's rounding and those of dl's entries other than the targets, which are taken as
    # they are, are independent, so their squares add up over many entries.  Sums in fp32 are off
    # by sqrt(n) 2^-24 of the partial sums, far below; 15 % of margin.  With the targets' entries
    # rounded too the norm is 1.4 times one rounding's.
    dt = x.dtype
    r = jb.linear_logprobs(x, w, targets)
    back = jb.linear_logprobs_backward(x, w, targets, r, g, d_lse=h)
    dl, dX, dW = _gradients(x, w, targets, g, h)
    G = torch.where(targets >= 0, g, 0.0)
    most = torch.stack([G.abs().max(), h.abs().max(), (h - G).abs().max()]).max().item()
    by = 2.0 ** (14 - np.floor(np.log2(most))) if dt == F16 else 1.0
    e = (dl * by).to(dt).double() / by - dl
    rows = torch.nonzero(targets >= 0)[:, 0]
    e[rows, targets[rows]] = 0
    for got, want, left in ((back[0], dX, e @ w.double()), (back[1], dW, e.t() @ x.double())):
        once = want.to(dt).double() - want
        bound = (once.norm() ** 2 + left.norm() ** 2).sqrt()
        off = (got.double() - want).norm()
        say(f"  {say_at}: {(off / once.norm()).item():.3f} of one rounding, bound {(1.15 * bound / once.norm()).item():.3f}")
        assert off <= 1.15 * bound, say_at
    again = jb.linear_logprobs_backward(x, w, targets, r, g, d_lse=h)
    assert torch.equal(back[0], again[0]) and torch.equal(back[1], again[1])


@pytest.mark.parametrize("dt", [BF16, F16])
@pytest.mark.parametrize("T,d,V", [(40, 136, 3000), (513, 136, 2000), (700, 1032, 33000), (1500, 264, 5003),
                                   (4096, 72, 700), (9000, 520, 300), (4200, 1024, 40000)])
def test_linear_logprob_gradients_are_rounded_once_at_any_number_of_tokens(T, d, V, dt):
    x, w, targets, g, h = _linlog_inputs(T, d, V, dt, seed=70)
    h *= 0.1
    _check_rounded_once(x, w, targets, g, h, (T, d, V, dt))


@pytest.mark.parametrize("dt", [BF16, F16])
@pytest.mark.parametrize("T", [33, 64, 65, 600, 5000])
def test_linear_logprob_gradients_of_targets_in_one_tile_are_rounded_once(T, dt):
    x, w, targets, g, h = _linlog_inputs(T, 200, 3000, dt, seed=71)
    targets = torch.where(targets >= 0, 1290 + targets % 30, -1)
    _check_rounded_once(x, w, targets, g, h * 0.1, (T, dt, "thirty targets"))
    targets = torch.where(targets >= 0, 2999, -1)
    _check_rounded_once(x, w, targets, g, h * 0.1, (T, dt, "one target"))


@pytest.mark.parametrize("dt", [BF16, F16])
@pytest.mark.parametrize("T", [300, 5000])
def test_masked_tokens_that_share_a_target_are_as_without_one(T, dt):
    # padding by gradients of 0 instead of targets below 0
    x, w, targets, g, h = _linlog_inputs(T, 200, 3000, dt, seed=72)
    pad = torch.arange(T, device="cuda") % 2 == 0
    g[pad], h[pad] = 0, 0
    targets = targets.clamp_min(0)
    shared, none = targets.clone(), targets.clone()
    shared[pad], none[pad] = 1777, -1
    _check_rounded_once(x, w, shared, g, h * 0.1, (T, dt, "padding"))
    got, want = (jb.linear_logprobs_backward(x, w, t, jb.linear_logprobs(x, w, t), g, d_lse=h) for t in (shared, none))
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


# ---- log probabilities: logits far from 0 ----

def _far(dt, T, logits):
    """x [T][16] and w [V][16] whose logits are exactly these: the same product in four channels."""
    scale = 2.0 ** 64 if dt == BF16 else 2.0 ** 15
    w = torch.zeros(len(logits), 16, dtype=torch.float64)
    w[:, 3:7] = torch.tensor(logits, dtype=torch.float64)[:, None] / scale / 4
    x = torch.zeros(T, 16, dtype=torch.float64)
    x[:, 3:7] = scale
    assert torch.equal(w.to(dt).double(), w)
    return x.to(dt).cuda(), w.to(dt).cuda()


@pytest.mark.parametrize("dt", [BF16, F16])
@pytest.mark.parametrize("V", [1, 40, 700])
@pytest.mark.parametrize("T", [3, 90])
def test_linear_logprobs_of_finite_logits_far_from_0(T, V, dt):
    far = [1.5 * 2.0 ** 30, 1.3125 * 2.0 ** 32, 1.9375 * 2.0 ** 32] if dt == F16 else [1.25 * 2.0 ** 33, 1.625 * 2.0 ** 99, 1.9375 * 2.0 ** 127]
    for top in [s * f for f in far for s in (1, -1)]:
        for name in ("tied", "leads", "two lead"):
            low = top * (0.5 if top > 0 else 1) if name != "tied" else top
            high = top * (1 if top > 0 else 0.5) if name != "tied" else top
            logits = [low] * V
            lead = range(V) if name == "tied" else [V // 2] if name == "leads" else [0, V - 1]
            for v in lead:
                logits[v] = high
            n = len(set(lead))
            x, w = _far(dt, T, logits)
            targets = torch.arange(T, device="cuda") % V
            targets[0] = lead[0]
            g = torch.linspace(0.25, 0.5, T, device="cuda") / 64
            h = torch.linspace(-0.125, 0.125, T, device="cuda") / 64
            r = jb.linear_logprobs(x, w, targets)
            to, L = targets.cpu().numpy(), np.array(logits)
            p = np.where(L == high, 1 / n, 0.0)
            want = L[to] - high - np.log(n)
            with np.errstate(over="ignore"):
                want = want.astype(np.float32).astype(np.float64)
            assert np.all(np.abs(_np(r.logprob) - want) <= 4 * E * (np.abs(want) + 8)), (top, name)
            assert np.all(np.abs(_np(r.lse) - high) <= 4 * E * abs(high)), (top, name)
            dX, dW = (_np(t) for t in jb.linear_logprobs_backward(x, w, targets, r, g, d_lse=h))
            G, H = _np(g), _np(h)
            dl = (H - G)[:, None] * p[None]
            dl[np.arange(T), to] += G
            u, tiny = ROUND[dt]
            W, X = _np(w), _np(x)
            # p to 700 terms' sums, dl's rounding, the output's
            rel = 3 * u + (V + T + 20) * E
            for got, size, exact in ((dX, np.abs(dl) @ np.abs(W), dl @ W), (dW, np.abs(dl).T @ np.abs(X), dl.T @ X)):
                # (1 - p of a leader alone is 0, of n a difference of halves)
                bound = rel * size + 8 * E * (np.abs(W).max() if got is dX else np.abs(X).sum()) + tiny
                assert np.all(np.abs(got - exact) <= bound), (top, name)


@pytest.mark.parametrize("dt", [BF16, F16])
@pytest.mark.parametrize("T,d,V", [(1, 4096, 3000), (3, 4096, 3001), (20, 4096, 700), (32, 2056, 4100), (40, 4096, 700),
                                   (16384 + 20, 1024, 600)])
def test_gradients_of_large_logits_take_the_forward_pass_sums(T, d, V, dt):
    # Logits of several 10^8, whose sums in fp32 are off by 100 and more: the leading token takes
    # all in either order of the sum, but its probability is exp of the difference of two sums.
    x, w = (_randn(80, T, d) * 3000).to(dt).cuda(), (_randn(81, V, d) * 3000).to(dt).cuda()
    gen = torch.Generator().manual_seed(82)
    targets = torch.randint(0, V, (T,), generator=gen).cuda()
    g, h = _randn(83, T).cuda(), _randn(84, T, std=0.1).cuda()
    g, h = g * 2.0 ** -8, h * 2.0 ** -8       # (dX within float16)
    W = w.double()
    value, index = (x.double() @ W.t()).topk(2, dim=1)
    lead, clear = index[:, 0], value[:, 0] - value[:, 1] > 1e5
    r = jb.linear_logprobs(x, w, targets)
    dX, dW = jb.linear_logprobs_backward(x, w, targets, r, g, d_lse=h)
    assert clear.float().mean() > 0.9 and torch.all(torch.isfinite(dX)) and torch.all(torch.isfinite(dW))
    G, H = g.double()[:, None], h.double()[:, None]
    want = G * W[targets] + (H - G) * W[lead]
    size = G.abs() * W[targets].abs() + (H - G).abs() * W[lead].abs()
    u, tiny = ROUND[dt]
    off = (dX.double() - want).abs()
    assert torch.all((off <= 2.1 * u * size + tiny)[clear])


# ---- log probabilities: targets and gradients that are none ----

@pytest.mark.parametrize("dt", [BF16, F16])
@pytest.mark.parametrize("T,V", [(3, 300), (90, 1000), (600, 2000)])
def test_targets_outside_the_vocabulary(T, V, dt):
    x, w, targets, g, h = _linlog_inputs(T, 64, V, dt, seed=90)
    wrong = targets.clone()
    wrong[0], wrong[1] = V, 2 ** 40
    targets[0] = targets[1] = -1
    g[:2] = 0
    h[:2] = 0
    g[2] = 1
    r, s = jb.linear_logprobs(x, w, targets), jb.linear_logprobs(x, w, wrong)
    assert torch.all(torch.isnan(s.logprob[:2])) and torch.equal(r.lse, s.lse)
    for d_lse in (None, h):   # without a gradient: as no target
        want = jb.linear_logprobs_backward(x, w, targets, r, g, d_lse=d_lse)
        got = jb.linear_logprobs_backward(x, w, wrong, s, g, d_lse=d_lse)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
        assert torch.all(got[0][:2] == 0)
    for name in ("g", "h"):   # with one: NaN, as the log probability
        a, b = g.clone(), h.clone()
        (a if name == "g" else b)[1] = 0.5
        got = jb.linear_logprobs_backward(x, w, wrong, s, a, d_lse=b)
        assert torch.all(torch.isnan(got[0][1])) and torch.all(torch.isnan(got[1]))
        assert torch.equal(got[0][2:], want[0][2:]) and torch.all(got[0][0] == 0)
        for t, e in zip(got, step.linear_logprobs_grad(_np(x), _np(w), wrong.cpu().numpy(), _np(a), _np(b))):
            assert np.array_equal(np.isnan(_np(t)), np.isnan(e))


@pytest.mark.parametrize("T", [5, 90])
@pytest.mark.parametrize("bad", [float("inf"), float("-inf"), float("nan")])
def test_a_broken_gradient_is_its_tokens_alone(T, bad):
    # (float16 scales all tokens' gradients by one power of two)
    x, w, targets, g, h = _linlog_inputs(T, 64, 500, F16, seed=91)
    x, w, g, h = x / 64, w * 64, g * 1e-7, h * 1e-7
    targets = targets.clamp_min(0)
    r = jb.linear_logprobs(x, w, targets)
    g[2] = h[2] = 0
    want = jb.linear_logprobs_backward(x, w, targets, r, g, d_lse=h, need=(True, False))[0]
    assert (want != 0).float().mean() > 0.5
    for name in ("g", "h"):
        a, b = g.clone(), h.clone()
        (a if name == "g" else b)[2] = bad
        got = jb.linear_logprobs_backward(x, w, targets, r, a, d_lse=b, need=(True, False))[0]
        keep = torch.arange(T, device="cuda") != 2
        assert torch.equal(got[keep], want[keep]) and not torch.all(torch.isfinite(got[2]))


@pytest.mark.parametrize("T", [5, 90])
def test_gradients_whose_difference_passes_the_range(T):
    x, w, targets, g, h = _linlog_inputs(T, 64, 500, F16, seed=92)
    targets = targets.clamp_min(0)
    r = jb.linear_logprobs(x, w, targets)
    g[1], h[1] = 3e38, -2e38
    dX, dW = jb.linear_logprobs_backward(x, w, targets, r, g, d_lse=h)
    assert not torch.any(torch.isnan(dX)) and not torch.any(torch.isnan(dW))


def test_float16_gradients_far_below_its_range():
    # normal outputs from gradients below float16's smallest number: channels that x has large where
    # w is 0 and the other way round
    x, w, targets, g, h = _linlog_inputs(700, 264, 9000, F16, seed=93)
    x[:, :64], w[:, :64] = x[:, :64] * 4096, 0
    w[:, 64:128], x[:, 64:128] = w[:, 64:128] * 30000, 0
    _check_rounded_once(x, w, targets, g * 1e-8, h * 1e-9, "small gradients")


# ---- the norm's gradient in place ----

@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("cols", [64, 1024, 4096, 16384, 16392, 20011])
def test_norm_gradient_in_place(cols, dt):
    T, lib = 70, jb.load_library()
    x, _, gain, dy, dh = _norm_inputs(T, cols, dt, dt, seed=60)
    n = int(lib.jarq_rms_norm_workspace_bytes(T, cols))
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    for a in (None, dh):
        want = jb.rms_norm_backward(x, gain, dy, dH=a)
        for over in ("dy", "dh"):
            for wanted in (True, False):
                y, b = dy.clone(), None if a is None else a.clone()
                if over == "dh" and a is None:
                    continue
                dx, dgain = y if over == "dy" else b, torch.empty_like(gain)
                assert lib.jarq_rms_norm_backward(
                    jb.DTYPES[dt], jb.DTYPES[dt], T, cols, x.data_ptr(), gain.data_ptr(), y.data_ptr(),
                    None if b is None else b.data_ptr(), ctypes.c_float(1e-6), dx.data_ptr(),
                    dgain.data_ptr() if wanted else None, ws.data_ptr(), n,
                    torch.cuda.current_stream().cuda_stream) == jb.JARQ_OK
                assert torch.equal(dx, want[0]) and (not wanted or torch.equal(dgain, want[1]))


def test_norm_into_what_it_reads():
    for cols in (64, 4096, 20000):
        x, res, gain, _, _ = _norm_inputs(9, cols, BF16, BF16, seed=61)
        y, h = jb.rms_norm(x, gain, residual=res)
        for out, sum_out in ((0, 1), (1, 0), (1, None), (None, 1)):
            at = [x.clone(), res.clone()]
            got = jb.rms_norm(at[0], gain, residual=at[1], out=None if out is None else at[out],
                              sum_out=None if sum_out is None else at[sum_out])
            assert torch.equal(got[0], y) and torch.equal(got[1], h)
        with pytest.raises(jb.JarqError):
            jb.rms_norm(x, gain, residual=res, out=x, sum_out=x)
        flat = torch.cat([x.view(-1), x.view(-1)[:2]])
        with pytest.raises(jb.JarqError):
            jb.rms_norm(flat[:-2].view(9, cols), gain, out=flat[2:].view(9, cols))


# ---- autograd: what a call writes into, and what it loses ----

def _calls_into():
    """(name, call, the tensors that it writes into): every call with tensors of the caller's."""
    def t(*shape, dtype=BF16):
        return torch.ones(*shape, dtype=dtype, device="cuda")

    x, y, h, gain, w = t(4, 64), t(4, 64), t(4, 64), t(64), t(8, 64)
    q, s = t(4, 64, dtype=torch.int8), t(4, 1, dtype=F32)
    wq, sw = t(8, 64, dtype=torch.int8), t(8, 1, dtype=F32)
    to, g = torch.zeros(4, dtype=torch.int64, device="cuda"), t(4, dtype=F32)
    o8, o64 = t(4, 8), t(4, 64)
    p, new = t(300), t(300)
    state, other = jb.adamw_state([p], bits=8), jb.adamw_state([p], bits=8)
    prm = jb.make_params(8, 64, 32, 3)
    codes, zeros = t(8, 64, dtype=torch.uint8), t(8, 2, dtype=torch.int32)
    return [
        ("rms_norm", lambda: jb.rms_norm(x, gain, residual=y, out=h, sum_out=y), [h, y]),
        ("rms_norm out", lambda: jb.rms_norm(x, gain, out=x), [x]),
        ("rms_norm_i8", lambda: jb.rms_norm_i8(y, gain, residual=h, out=q, scale=s, sum_out=y), [q, s, y]),
        ("adamw_step", lambda: jb.adamw_step([p], [t(300)], state, 1, 1e-3),
         [p, state.master, state.m, state.v, state.m_exp, state.v_exp]),
        ("adamw_step out", lambda: jb.adamw_step([p], [t(300)], state, 1, 1e-3, out=([new], other)),
         [new, other.master, other.m, other.v, other.m_exp, other.v_exp]),
        ("gated_forward", lambda: jb.gated_forward(x, w, w, out=o8), [o8]),
        ("quant_rows_i8", lambda: jb.quant_rows_i8(x, out=q, scale=s), [q, s]),
        ("codes_i8", lambda: jb.codes_i8(prm, codes, zeros, out=wq), [wq]),
        ("matmul_i8", lambda: jb.matmul_i8(q, s, wq, sw, out=o8), [o8]),
        ("linear_i8", lambda: jb.linear_i8(x, wq, sw, out=o8), [o8]),
        ("token_logprobs_backward", lambda: jb.token_logprobs_backward(
            o64, to, jb.token_logprobs(o64, to), g, out=h), [h]),
    ]


def test_what_a_call_writes_into_has_another_version():
    for name, call, into in _calls_into():
        before = [t._version for t in into]
        call()
        assert all(t._version > v for t, v in zip(into, before)), name
    with torch.inference_mode():   # whose tensors have none
        for name, call, into in _calls_into():
            call()


def test_a_backward_pass_that_kept_what_is_overwritten_says_so():
    x = torch.ones(300, device="cuda", requires_grad=True)
    p = torch.ones(300, device="cuda")
    y = (p * x).sum()      # keeps p, which needs no gradient itself
    jb.adamw_step([p], [torch.ones_like(p)], jb.adamw_state([p]), 1, 1e-2)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.backward()
    stream = torch.ones(4, 64, device="cuda")
    a = torch.ones(4, 64, device="cuda", requires_grad=True)
    y = (stream * a).sum()
    jb.rms_norm(torch.ones(4, 64, device="cuda"), torch.ones(64, device="cuda"), residual=stream, sum_out=stream)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.backward()


def test_tangents_that_are_lost_are_said_to_be():
    def t(*shape, dtype=BF16):
        return torch.ones(*shape, dtype=dtype, device="cuda")

    gain, w = t(64), t(8, 64)
    wq, sw = t(8, 64, dtype=torch.int8), t(8, 1, dtype=F32)
    to = torch.zeros(4, dtype=torch.int64, device="cuda")
    with forward_ad.dual_level():
        x = forward_ad.make_dual(t(4, 64), t(4, 64))
        dual = forward_ad.make_dual(gain, t(64))
        calls = (lambda: jb.rms_norm(x, gain), lambda: jb.rms_norm(t(4, 64), dual),
                 lambda: jb.rms_norm(t(4, 64), gain, residual=x), lambda: jb.rms_norm_i8(x, gain),
                 lambda: jb.linear_logprobs(x, w, to), lambda: jb.gated_forward(x, w, w),
                 lambda: jb.linear_i8(x, wq, sw), lambda: jb.token_logprobs(x, to))
        for k, call in enumerate(calls):
            with pytest.warns(UserWarning, match="autograd"):
                call()
        with warnings.catch_warnings():
            warnings.simplefilter("error")
            jb.rms_norm(t(4, 64), gain)
            with torch.no_grad():
                jb.linear_logprobs(x, w, to)


# ---- AdamW: what lies between the tensors ----

@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("dt", [F32, BF16])
def test_adamw_leaves_or_clears_what_lies_between_the_tensors(dt, bits):
    # lengths that end inside eight values, inside a block, inside a work-group's share
    sizes = [1, 5, 127, 300, 2049]
    params = [_randn(k, n).to(dt).cuda() for k, n in enumerate(sizes)]
    grads = [_randn(9 + k, n).to(dt).cuda() for k, n in enumerate(sizes)]
    state = jb.adamw_state(params, bits=bits)
    between = torch.ones(len(state.m), dtype=torch.bool, device="cuda")
    at = step.offsets(sizes)[0]
    for first, n in zip(at, sizes):
        between[first:first + n] = False
    held = [a for a in (state.master, state.m, state.v) if a is not None]
    for a in held:
        raw = a.view(torch.uint8) if a.dtype != F32 else a
        raw[between] = 57
    clean = [p.clone() for p in params]
    same = jb.adamw_state(clean, bits=bits)
    jb.adamw_step(params, grads, state, 1, 1e-2, seed=4, **OPT)
    jb.adamw_step(clean, grads, same, 1, 1e-2, seed=4, **OPT)
    assert all(torch.equal(a, b) for a, b in zip(params, clean))     # it has no part in the step
    for a, b in zip(state, same):
        if a is None:
            continue
        if a.dtype == torch.uint8:
            assert torch.equal(a, b)
            continue
        a, b = (t.view(torch.uint8) if t.dtype != F32 else t for t in (a, b))
        assert torch.equal(a[~between], b[~between])
        left = a[between]
        assert torch.all((left == 0) | (left == 57))
