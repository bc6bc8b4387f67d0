"""Where the operators that run, train and evaluate refined layers could lose accuracy:
tails and cancellations, against float64 with bounds relative to the small result itself.
E = 2^-24 is half a unit in the last place of fp32."""

import math
import warnings

import pytest
import torch

from paper_2609_38599_amd import binding as jb
from tests import test_gpu_blocks as blocks_tests
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


# half a unit in the last place, and half the smallest subnormal (fp32: normal)
ROUND = {torch.float32: (2.0 ** -24, 2.0 ** -126), torch.float16: (2.0 ** -11, 2.0 ** -25),
         torch.bfloat16: (2.0 ** -8, 2.0 ** -126)}


def _check_leading_gradient(x, t, r, gl, ge):
    V, dt = x.shape[1], x.dtype
    rows = torch.arange(len(t))
    d, s, sd = _others(x, t)
    g, h = gl.double(), ge.double()
    # log p + H at the target is -sd / (1 + s): nothing cancels
    lp, ent = -torch.log1p(s), torch.log1p(s) - sd / (1 + s)
    z, u, tiny = _sums(V), *ROUND[dt]
    at = g * s / (1 + s) + h * sd / (1 + s) ** 2
    at_err = g.abs() * s / (1 + s) * (z + 8 * E) + \
        h.abs() / (1 + s) * (lp.abs() + ent) * (2 * z + 16 * E)
    logp = d + lp[:, None]
    p = torch.exp(logp)
    far = torch.where(p > 0, logp.abs(), 0.0)
    want = -p * (g[:, None] + h[:, None] * (torch.where(p > 0, logp, 0.0) + ent[:, None]))
    err = p * (g.abs()[:, None] + h.abs()[:, None] * (far + ent[:, None] + 1)) * \
        (2 * z + 16 * E + 8 * E * far)
    want[rows, t], err[rows, t] = at, at_err
    bound = err + u * (want.abs() + err) + tiny
    xc, tc, glc, gec = x.cuda(), t.cuda(), gl.cuda(), ge.cuda()
    # with what the forward pass kept, without it, and in place
    rebuilt = jb.TokenLogprobs(*r)
    for form in (r, rebuilt):
        got = jb.token_logprobs_backward(xc, tc, form, glc, gec)
        over = ((got.double().cpu() - want).abs() - bound).max()
        assert float(over) <= 0, (form is r, float(over))
        y = xc.clone()
        assert torch.equal(jb.token_logprobs_backward(y, tc, form, glc, gec, out=y), got)


@pytest.mark.parametrize("lead", [8.0, 18.0, 22.0, 25.0])
@pytest.mark.parametrize("T,V,dt", LEADS)
def test_logit_gradient_of_a_leading_token(T, V, dt, lead):
    # g (1 - p) at the target: off by what 1 - p is, wherever the logits lie
    for offset in (0.0, 100.0, 1e4) if dt == torch.float32 else (0.0, 100.0):
        say(f"[gradient lead] tokens {T} vocab {V} {dt} lead {lead} offset {offset}")
        x, t = _leading(T, V, dt, lead, offset)
        _check_leading_gradient(x, t, jb.token_logprobs(x.cuda(), t.cuda()),
                                _randn(1, T), _randn(2, T))


@pytest.mark.parametrize("dt", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("T,V", [(3, 37), (2, 40001), (700, 1003)])
def test_logit_gradient_of_rows_of_the_lowest_value(T, V, dt):
    # every entry masked by the type's lowest value: p = 1 / V
    say(f"[gradient lowest] tokens {T} vocab {V} {dt}")
    x = torch.full((T, V), torch.finfo(dt).min, dtype=dt)
    t = torch.arange(T) % V
    _check_leading_gradient(x, t, jb.token_logprobs(x.cuda(), t.cuda()), _randn(1, T), _randn(2, T))


@pytest.mark.parametrize("dt", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("V", [37, 5000, 40001])
def test_logit_gradient_without_the_kept_sums(V, dt, monkeypatch):
    # the backward pass that forms the rows' sums itself, on masked and broken rows
    kept = jb.token_logprobs_backward
    forms = []

    def both(x, t, r, gl, ge):
        forms.append(jb.TokenLogprobs(*r))
        assert r.lse_rest is not None and forms[-1].lse_rest is None
        return kept(x, t, forms[-1], gl, ge)

    monkeypatch.setattr(jb, "token_logprobs_backward", both)
    blocks_tests.test_logprobs_of_masked_and_broken_rows(V, dt)
    assert len(forms) == 1


@pytest.mark.parametrize("V,ld,first", [(1000, 1003, 0), (1001, 1001, 1), (7, 9, 2)])
def test_logit_gradient_of_unaligned_rows_without_the_kept_sums(V, ld, first):
    T = 9
    base = _randn(5, T * ld + 8).bfloat16().cuda()
    x = base[first:first + T * ld].view(T, ld)[:, :V]
    t, gl, ge = torch.arange(T).cuda() % V, _randn(1, T).cuda(), _randn(2, T).cuda()
    r = jb.TokenLogprobs(*jb.token_logprobs(x, t))
    d = jb.token_logprobs_backward(x, t, r, gl, ge)
    blocks_tests._check_grad(x, t, gl, ge, d)
    out = torch.full_like(base, 7.0)
    rows = out[first:first + T * ld].view(T, ld)
    jb.token_logprobs_backward(x, t, r, gl, ge, out=rows[:, :V])
    assert torch.equal(rows[:, :V], d) and bool((rows[:, V:] == 7.0).all())


# ---- activations in their left tail ----

def _activation64(a, act):
    """(act(a), act'(a)) of one float64 below 0, without 1 + erf or 1 + tanh."""
    if act == "silu":
        sig, w = 1 / (1 + math.exp(-a)), 1.0
    elif act == "gelu":
        cdf = 0.5 * math.erfc(-a / math.sqrt(2))
        return a * cdf, cdf + a * math.exp(-a * a / 2) / math.sqrt(2 * math.pi)
    else:
        c = math.sqrt(2 / math.pi)
        sig = 1 / (1 + math.exp(-2 * c * (a + 0.044715 * a ** 3)))
        w = 2 * c * (1 + 3 * 0.044715 * a * a)
    return a * sig, sig * (1 + a * (1 - sig) * w)


@pytest.mark.parametrize("dt", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("act", sorted(jb.ACTIVATIONS))
@pytest.mark.parametrize("T", [13, 29, 200])
def test_gated_block_in_the_left_tail(T, act, dt):
    say(f"[gated tail] tokens {T} {act} {dt}")
    x, wg, wu = torch.zeros(T, 8), torch.zeros(8, 8), torch.zeros(8, 8)
    # a is the token's first value and b is 1, exactly; dx is (act'(a), act(a)) of channel 0
    x[:, 0], x[:, 1], wg[0, 0], wu[0, 1] = torch.linspace(-9, -3, T), 1.0, 1.0, 1.0
    x, wg, wu = x.to(dt), wg.to(dt).cuda(), wu.to(dt).cuda()
    y, pre = jb.gated_forward(x.cuda(), wg, wu, act=act, save=True)
    dy = torch.zeros_like(y)
    dy[:, 0] = 1
    dx, _, _ = jb.gated_backward(x.cuda(), wg, wu, dy, pre, act=act)
    u, tiny = ROUND[dt]
    for t in range(T):
        a = float(x[t, 0])
        h, slope = _activation64(a, act)
        # erfc's and exp's arguments are of order a^2 and rounded a few times, their sums of
        # one sign or no more than halved by the other
        rel = (64 + 12 * a * a) * E
        for got, want, r in ((y[t, 0], h, rel), (dx[t, 1], h, rel), (dx[t, 0], slope, 2 * rel)):
            assert abs(float(got) - want) <= abs(want) * (r + u * (1 + r)) + tiny, (a, act)


# ---- the same row elsewhere ----

@pytest.mark.parametrize("dt", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("T,V,top", [(9, 4097, 5), (5, 32001, 20), (2, 128001, 8), (9, 7, 0),
                                     (600, 1001, 3)])
def test_logprobs_do_not_depend_on_stride_or_alignment(T, V, top, dt):
    say(f"[logprob placed] tokens {T} vocab {V} top {top} {dt}")
    base = _randn(T + V, T, V, std=2.0).to(dt).cuda()
    t, gl, ge = torch.arange(T).cuda() % V, _randn(1, T).cuda(), _randn(2, T).cuda()
    want = None
    for ld, first in ((V, 0), (V + 1, 0), (V + 2, 1), (V + 3, 3), (V + 8 - V % 8, 0), (V, 5)):
        room = torch.zeros(T * ld + 16, dtype=dt, device="cuda")
        x = room[first:first + T * ld].view(T, ld)[:, :V]
        x.copy_(base)
        r = jb.token_logprobs(x, t, top=top)
        got = [v for v in (*r, r.lse_rest) if v is not None]
        for form in (r, jb.TokenLogprobs(*r)):
            got.append(jb.token_logprobs_backward(x, t, form, gl, ge))
        want = want or got
        assert all(torch.equal(a, b) for a, b in zip(got, want)), (ld, first)


@pytest.mark.parametrize("ties", [2, 3, 5])
@pytest.mark.parametrize("T,V", [(1, 128000), (8, 65536), (40, 50257), (600, 1001)])
def test_logprob_of_an_alternative_is_its_top_logprob(T, V, ties):
    # a row cut into parts, some of which hold its maximum: every lane has the same sums
    say(f"[logprob top] tokens {T} vocab {V} ties {ties}")
    x = _randn(V + ties, T, V, std=2.0)
    for k in range(ties):
        x[:, (2 * k + 1) * V // (2 * ties)] = 14.0
    x, top = x.cuda(), 7
    first = jb.token_logprobs(x, torch.zeros(T, dtype=torch.int64).cuda(), top=top)
    for k in range(top):
        r = jb.token_logprobs(x, first.top_index[:, k].long(), top=top)
        assert torch.equal(r.top_logprob, first.top_logprob)
        assert torch.equal(r.logprob, r.top_logprob[:, k])


# ---- inputs that require gradients ----

def test_results_outside_the_graph_are_said_to_be():
    x, w = _randn(1, 4, 64).bfloat16().cuda(), _randn(2, 8, 64).bfloat16().cuda()
    wq, sw = torch.ones(8, 64, dtype=torch.int8).cuda(), torch.ones(8, 1).cuda()
    t = torch.zeros(4, dtype=torch.int64).cuda()
    calls = {"gated_backward": lambda x: jb.gated_forward(x, w, w),
             "linear_i8: .* no gradient": lambda x: jb.linear_i8(x, wq, sw),
             "token_logprobs_backward": lambda x: jb.token_logprobs(x, t)}
    for said, call in calls.items():
        with pytest.warns(UserWarning, match=said):
            call(x.clone().requires_grad_())
    with pytest.warns(UserWarning, match="matmul_i8: .* no gradient"):
        jb.matmul_i8(wq, sw, wq, sw.clone().requires_grad_())
    with warnings.catch_warnings():
        warnings.simplefilter("error")
        for call in calls.values():
            call(x)
            with torch.no_grad():
                call(x.clone().requires_grad_())
        # its gradients are asked for
        jb.gated_forward(x.clone().requires_grad_(), w, w, save=True)


# ---- every entry of every shape of tile ----

@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("T,d,f", [(40, 264, 1000), (70, 136, 4096), (100, 1000, 2752),
                                   (250, 72, 11008), (400, 4096, 1000), (700, 264, 6000),
                                   (3300, 520, 2048), (2100, 8, 2104), (129, 4104, 520),
                                   (3600, 3592, 1800)])
def test_gated_tiles_entry_by_entry(T, d, f, dt):
    # the bounds of the small sizes' test, in float64 on the GPU: sums of n products are off by
    # (n + 2) e of the sum of magnitudes, and 1.13 bounds |act'| and |act''|
    say(f"[gated entries] tokens {T} d {d} f {f} {dt}")
    x, wg, wu, dy = blocks_tests._gated_inputs(T, d, f, dt, seed=T)
    y, pre = jb.gated_forward(x, wg, wu, save=True)
    dx, dwg, dwu = jb.gated_backward(x, wg, wu, dy, pre)
    X, G, U, D = (t.double() for t in (x, wg, wu, dy))
    u, tiny = ROUND[dt]

    def check(what, got, want, err, rounded=True):
        bound = err + u * (want.abs() + err) + tiny if rounded else err
        over = float(((got.double() - want).abs() - bound).max())
        assert over <= 0, (what, over)

    a, b = X @ G.T, X @ U.T
    ea, eb = ((d + 2) * E * (X.abs() @ W.abs().T) for W in (G, U))
    check("a", pre[0], a, ea, False)
    check("b", pre[1], b, eb, False)
    sig = 1 / (1 + torch.exp(-a))
    h, slope, fn = a * sig, sig * (1 + a * (1 - sig)), 64 * E * (a.abs() + 1)
    act = 1.13 * ea + fn
    check("y", y, h * b, b.abs() * act + h.abs() * eb + 2 * ea * eb)
    da, db = D * b * slope, D * h
    eda = D.abs() * (b.abs() * act + (slope.abs() + fn) * eb + 2 * ea * eb)
    edb = D.abs() * act
    eda, edb = (e + u * (m.abs() + e) + tiny + 4 * E * m.abs() for e, m in ((eda, da), (edb, db)))
    err, sums = eda @ G.abs() + edb @ U.abs(), da.abs() @ G.abs() + db.abs() @ U.abs()
    check("dx", dx, da @ G + db @ U, err + (2 * f + 2) * E * (sums + err))
    for what, got, m, e in (("dwg", dwg, da, eda), ("dwu", dwu, db, edb)):
        err, sums = e.T @ X.abs(), m.abs().T @ X.abs()
        check(what, got, m.T @ X, err + (T + 2) * E * (sums + err))


@pytest.mark.parametrize("g", [0, 32, 64, 128])
@pytest.mark.parametrize("T,n,k", [(40, 1000, 512), (40, 4096, 384), (50, 10000, 1152),
                                   (150, 4000, 384), (400, 4000, 1152), (1000, 4100, 384),
                                   (3000, 4100, 384), (66, 700, 2688), (130, 17, 896),
                                   (3000, 4097, 384), (1993, 6966, 128), (260, 4096, 1024)])
def test_matmul_i8_tiles_entry_by_entry(T, n, k, g):
    say(f"[i8 entries] tokens {T} n {n} k {k} group {g}")
    gen = torch.Generator(device="cuda").manual_seed(T + k)
    xq, wq = (torch.randint(-128, 128, (m, k), generator=gen, device="cuda", dtype=torch.int8)
              for m in (T, n))
    G = k // g if g else 1
    sx = torch.rand(T, generator=gen, device="cuda")
    sw = torch.randn(n, G, generator=gen, device="cuda")
    want = torch.zeros(T, n, dtype=torch.float64, device="cuda")
    size = torch.zeros_like(want)
    for i in range(G):
        cut = slice(i * (k // G), (i + 1) * (k // G))
        part = (xq[:, cut].double() @ wq[:, cut].double().T) * sw[:, i].double()
        want += part
        size += part.abs()
    want, size = want * sx.double()[:, None], size * sx.double()[:, None]
    for dt in (torch.float32, torch.float16, torch.bfloat16):
        scale = 1.0 if dt != torch.float16 else 2.0 ** -8      # within its range
        y = jb.matmul_i8(xq, sx * scale, wq, sw, dtype=dt)
        u, tiny = ROUND[dt]
        err = (G + 4) * E * size * scale
        over = (y.double() - want * scale).abs() - err - u * ((want * scale).abs() + err) - tiny
        assert float(over.max()) <= 0, (dt, float(over.max()))
