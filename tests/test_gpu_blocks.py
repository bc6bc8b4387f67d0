"""The operators that run, train and evaluate refined layers on the GPU against their
float64 definitions.  Tolerances are bounds from the arithmetic: u is half a unit
in the last place of the output's type, e = 2^-24 that of fp32 sums."""

import numpy as np
import pytest
import torch

from oracle import blocks
from paper_2609_38599_amd import binding as jb
from tests._gpu_common import say

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]

E = 2.0 ** -24
# half a unit in the last place, and half the smallest subnormal
ROUND = {torch.float32: (2.0 ** -24, 2.0 ** -150), torch.float16: (2.0 ** -11, 2.0 ** -25),
         torch.bfloat16: (2.0 ** -8, 2.0 ** -134)}
ACTS = ("silu", "gelu", "gelu_tanh")


def _np(t):
    return t.detach().double().cpu().numpy()


def _randn(seed, *shape, std=1.0):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed)) * std


def _close(got, want, bound, what):
    got = _np(got)
    assert got.shape == want.shape
    fine = np.isfinite(want)
    assert np.array_equal(np.isnan(got), np.isnan(want)), what
    assert np.array_equal(got[~fine & ~np.isnan(want)], want[~fine & ~np.isnan(want)]), what
    over = np.abs(got - want)[fine] - np.broadcast_to(bound, want.shape)[fine]
    assert over.size == 0 or over.max() <= 0, (what, over.max())


# ---- the gated block ----

def _gated_inputs(T, d, f, dt, seed=0):
    x = _randn(seed, T, d).to(dt)
    wg, wu = (_randn(seed + k, f, d, std=1.5 / d ** 0.5).to(dt) for k in (1, 2))
    dy = _randn(seed + 3, T, f).to(dt)
    return [t.cuda() for t in (x, wg, wu, dy)]


def _pre_bound(X, W, d):
    # d products summed in fp32 in any order
    return (d + 2) * E * (np.abs(X) @ np.abs(W).T)


# one token to several tiles; channels inside a tile, at its edge and past it
GATED = [(1, 8, 8), (1, 1000, 40), (2, 64, 264), (16, 136, 24), (17, 72, 136), (33, 264, 72),
         (64, 128, 128), (65, 8, 200), (127, 72, 64), (129, 328, 264), (257, 192, 520)]


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("T,d,f", GATED)
def test_gated_forward_and_backward(T, d, f, dt):
    act = ACTS[(T + f) % 3]
    x, wg, wu, dy = _gated_inputs(T, d, f, dt)
    say(f"[gated] tokens {T} d {d} f {f} {dt} {act}")
    X, G, U, D = map(_np, (x, wg, wu, dy))
    y, pre = jb.gated_forward(x, wg, wu, act=act, save=True)
    assert torch.equal(y, jb.gated_forward(x, wg, wu, act=act))
    want, a, b = blocks.gated(X, G, U, act)
    ea, eb = _pre_bound(X, G, d), _pre_bound(X, U, d)
    _close(pre[0], a, ea, "a")
    _close(pre[1], b, eb, "b")
    u, tiny = ROUND[dt]
    h, slope, lip = blocks.activation(a, act)
    fn = 64 * E * (np.abs(a) + 1)            # the activation's own functions in fp32
    ey = np.abs(b) * (lip * ea + fn) + np.abs(h) * eb + 2 * ea * eb
    _close(y, want, ey + u * (np.abs(want) + ey) + tiny, "y")
    dx, dwg, dwu = jb.gated_backward(x, wg, wu, dy, pre, act=act)
    rx, rg, ru, da, db = blocks.gated_grad(X, G, U, D, act)
    # da and db: from a and b as above, then rounded to the inputs' type
    eda = np.abs(D) * (np.abs(b) * (lip * ea + fn) + (np.abs(slope) + fn) * eb + 2 * ea * eb)
    edb = np.abs(D) * (lip * ea + fn)
    eda, edb = (e + u * (np.abs(m) + e) + tiny + 4 * E * np.abs(m)
                for e, m in ((eda, da), (edb, db)))
    def product(err, sums, want, n):
        e = err + (n + 2) * E * (sums + err)
        return e + u * (np.abs(want) + e) + tiny
    _close(dx, rx, product(eda @ np.abs(G) + edb @ np.abs(U),
                           np.abs(da) @ np.abs(G) + np.abs(db) @ np.abs(U), rx, 2 * f), "dx")
    _close(dwg, rg, product(eda.T @ np.abs(X), np.abs(da).T @ np.abs(X), rg, T), "dwg")
    _close(dwu, ru, product(edb.T @ np.abs(X), np.abs(db).T @ np.abs(X), ru, T), "dwu")


def test_gated_larger_than_one_round_of_tiles():
    # enough 256-wide tiles for the large ones in all three products
    T, d, f, dt = 3600, 3592, 1800, torch.bfloat16
    x, wg, wu, dy = _gated_inputs(T, d, f, dt)
    y, pre = jb.gated_forward(x, wg, wu, save=True)
    dx, dwg, dwu = jb.gated_backward(x, wg, wu, dy, pre)
    X, G, U, D = (t.double() for t in (x, wg, wu, dy))
    a, b = X @ G.T, X @ U.T
    s = 1 / (1 + torch.exp(-a))
    da, db = D * b * s * (1 + a * (1 - s)), D * a * s
    u = ROUND[dt][0]
    # da and db carry one rounding of relative size u, independent over the sums
    for got, want in ((y, a * s * b), (dx, da @ G + db @ U), (dwg, da.T @ X), (dwu, db.T @ X)):
        off = (got.double() - want).abs()
        assert off.norm() <= 1.5 * u * want.norm()
        assert off.max() <= 8 * u * want.abs().max()


def test_gated_gradient_against_differences():
    # pre is not rounded to 16 bits: a difference of the block through it
    T, d, f, act = 24, 64, 48, "silu"
    x, wg, wu, dy = _gated_inputs(T, d, f, torch.float16, seed=9)
    _, pre = jb.gated_forward(x, wg, wu, act=act, save=True)
    dx, dwg, dwu = jb.gated_backward(x, wg, wu, dy, pre, act=act)
    def loss(x, wg, wu):
        p = _np(jb.gated_forward(x, wg, wu, act=act, save=True)[1])
        return (_np(dy) * blocks.activation(p[0], act)[0] * p[1]).sum()
    for k, (t, grad) in enumerate(((x, dx), (wg, dwg), (wu, dwu))):
        v = torch.sign(_randn(20 + k, *t.shape)).cuda() * 2.0 ** (-6 if k == 0 else -9)
        lo, hi = (t.float() - v).half(), (t.float() + v).half()
        args = [x, wg, wu]
        step = _np(hi) - _np(lo)
        f1 = loss(*[hi if i == k else a for i, a in enumerate(args)])
        f0 = loss(*[lo if i == k else a for i, a in enumerate(args)])
        want = (_np(grad) * step).sum()
        # third derivatives at these steps, and the gradients' roundings
        assert abs((f1 - f0) - want) <= 2e-3 * np.abs(_np(grad) * step).sum()


def test_gated_no_tokens_and_skipped_gradients():
    x, wg, wu, dy = _gated_inputs(5, 64, 32, torch.bfloat16)
    y, pre = jb.gated_forward(x[:0], wg, wu, save=True)
    assert y.shape == (0, 32)
    dwg = torch.full_like(wg, 3.0)
    dx, dwg, dwu = jb.gated_backward(x[:0], wg, wu, dy[:0], pre)
    assert dx.shape == (0, 64) and not dwg.any() and not dwu.any()
    y, pre = jb.gated_forward(x, wg, wu, save=True)
    full = jb.gated_backward(x, wg, wu, dy, pre)
    for k in range(3):
        need = [i == k for i in range(3)]
        some = jb.gated_backward(x, wg, wu, dy, pre, need=need)
        assert torch.equal(some[k], full[k]) and all(some[i] is None for i in range(3) if i != k)


def test_gated_rows_are_independent():
    # a token of infinities and NaN leaves the others alone, at every kernel's sizes
    for T in (3, 20, 50, 200):
        x, wg, wu, _ = _gated_inputs(T, 72, 136, torch.bfloat16)
        y = jb.gated_forward(x, wg, wu)
        x[1] = float("nan")
        x[2, 5] = float("inf")
        z = jb.gated_forward(x, wg, wu)
        keep = [i for i in range(T) if i not in (1, 2)]
        assert torch.equal(y[keep], z[keep]) and torch.isnan(z[1]).all()


def test_gated_on_another_stream_and_in_a_graph():
    x, wg, wu, dy = _gated_inputs(40, 128, 256, torch.bfloat16)
    y, pre = jb.gated_forward(x, wg, wu, save=True)
    want = (y, *jb.gated_backward(x, wg, wu, dy, pre))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    y, pre = jb.gated_forward(x, wg, wu, save=True, stream=side)
    got = (y, *jb.gated_backward(x, wg, wu, dy, pre, stream=side))
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y, pre = jb.gated_forward(x, wg, wu, save=True)
        got = (y, *jb.gated_backward(x, wg, wu, dy, pre))
    for _ in range(3):
        for t in got:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))


# ---- 8-bit integers ----

@pytest.mark.parametrize("dt", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("rows,cols", [(1, 16), (3, 160), (70, 4096), (2, 20000)])
def test_quant_rows(rows, cols, dt):
    x = _randn(1, rows, cols, std=3.0)
    x[0, cols // 2] *= 40
    x = x.to(dt)
    q, s = jb.quant_rows_i8(x.cuda())
    Q, S = blocks.quant_rows(x.float().numpy())
    assert np.array_equal(q.cpu().numpy(), Q)
    assert np.array_equal(s.cpu().numpy()[:, 0], S)


def test_quant_rows_of_zeros_infinities_and_nan():
    x = _randn(2, 7, 48)
    x[0] = 0
    x[1, 3] = float("inf")
    x[2, 47] = float("nan")
    x[3] = 1e-38
    x[4] *= 1e30
    x[5, 0] = -float("inf")
    q, s = jb.quant_rows_i8(x.cuda())
    Q, S = blocks.quant_rows(x.numpy())
    assert np.array_equal(q.cpu().numpy(), Q)
    assert np.array_equal(s.cpu().numpy()[:, 0], S, equal_nan=True)
    w = torch.ones(5, 48, dtype=torch.int8).cuda()
    y = jb.linear_i8(x.cuda(), w, torch.ones(5, 1).cuda())
    for r in range(7):
        assert bool(torch.isnan(y[r]).all()) == (r in (1, 2, 5))
    assert not y[0].any() and not y[3].any()


I8 = [(1, 1, 16, 0), (1, 40, 96, 32), (5, 17, 192, 64), (16, 33, 384, 128), (17, 20, 1376, 32),
      (31, 100, 48, 0), (64, 65, 448, 64), (65, 129, 160, 32), (130, 127, 192, 64),
      (200, 260, 640, 128), (129, 300, 272, 0), (300, 515, 1408, 64)]


@pytest.mark.parametrize("dt", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("T,n,k,g", I8)
def test_matmul_i8(T, n, k, g, dt):
    gen = torch.Generator().manual_seed(T + n)
    xq = torch.randint(-128, 128, (T, k), generator=gen, dtype=torch.int8)
    wq = torch.randint(-128, 128, (n, k), generator=gen, dtype=torch.int8)
    G = k // g if g else 1
    sx, sw = torch.rand(T, 1, generator=gen) * 0.01, torch.randn(n, G, generator=gen) * 0.01
    say(f"[i8] tokens {T} n {n} k {k} group {g} {dt}")
    y = jb.matmul_i8(xq.cuda(), sx.cuda(), wq.cuda(), sw.cuda(), dtype=dt)
    want, size = blocks.matmul_i8(xq.numpy(), sx.numpy(), wq.numpy(), sw.numpy())
    u, tiny = ROUND[dt]
    # a group's sum to fp32, its product, the sum over groups, the token's scale
    err = (G + 4) * E * size
    _close(y, want, err + u * (np.abs(want) + err) + tiny, "y")


def test_matmul_i8_sums_at_the_ends_of_int32():
    k = 131056
    xq = torch.full((2, k), -128, dtype=torch.int8)
    wq = torch.full((3, k), -128, dtype=torch.int8)
    xq[1] = 127
    for T in (2, 70):
        x = xq[[0, 1] * (T // 2)].cuda()
        y = jb.matmul_i8(x, torch.ones(T).cuda(), wq.cuda(), torch.ones(3, 1).cuda(),
                         dtype=torch.float32)
        want = torch.tensor([128 * 128 * k, -127 * 128 * k]).float()
        assert torch.equal(y[:2, 0].cpu(), want) and torch.equal(y[-2:, 2].cpu(), want)


def test_matmul_i8_large_tiles():
    T, n, k = 3400, 3600, 304
    gen = torch.Generator().manual_seed(5)
    xq, wq = (torch.randint(-127, 128, (m, k), generator=gen, dtype=torch.int8).cuda() for m in (T, n))
    sx, sw = torch.rand(T, generator=gen).cuda(), torch.rand(n, 1, generator=gen).cuda()
    want = (xq.double() @ wq.double().T) * sx.double()[:, None] * sw.double().T
    y = jb.matmul_i8(xq, sx, wq, sw, dtype=torch.float32)
    assert bool(((y.double() - want).abs() <= 4 * E * want.abs()).all())


@pytest.mark.parametrize("T", [1, 9, 40, 150])
@pytest.mark.parametrize("g,bits", [(32, 4), (64, 3), (128, 7)])
def test_linear_i8_from_a_layers_codes(T, g, bits):
    rows, cols = 72, 512
    gen = torch.Generator().manual_seed(g + T)
    q = torch.randint(0, 1 << bits, (rows, cols), generator=gen, dtype=torch.uint8)
    z = torch.randint(0, 1 << bits, (rows, cols // g), generator=gen, dtype=torch.int32)
    s = torch.randn(rows, cols // g, generator=gen) * 0.02
    p = jb.make_params(rows, cols, g, bits, 1)
    wq = jb.codes_i8(p, q.cuda(), z.cuda())
    assert torch.equal(wq.cpu().int(), q.int() - z.repeat_interleave(g, 1))
    x = _randn(3, T, cols).to(torch.bfloat16)
    y = jb.linear_i8(x.cuda(), wq, s.cuda())
    Q, S = blocks.quant_rows(x.float().numpy())
    want, size = blocks.matmul_i8(Q, S, wq.cpu().numpy(), s.numpy())
    err = (cols // g + 4) * E * size
    u, tiny = ROUND[torch.bfloat16]
    _close(y, want, err + u * (np.abs(want) + err) + tiny, "y")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    z = jb.linear_i8(x.cuda(), wq, s.cuda(), stream=side)
    side.synchronize()
    assert torch.equal(y, z)


def test_codes_outside_int8_are_refused():
    p = jb.make_params(4, 128, 64, 8, 1)
    q = torch.full((4, 128), 255, dtype=torch.uint8).cuda()
    z = torch.full((4, 2), 128, dtype=torch.int32).cuda()
    assert int(jb.codes_i8(p, q, z)[0, 0]) == 127
    z[3, 1] = 127
    with pytest.raises(jb.JarqError):
        jb.codes_i8(p, q, z)


# ---- log probabilities ----

def _check_logprobs(x, targets, top, r):
    X, tg = _np(x), targets.cpu().numpy()
    lp, ent, lse, idx, val = blocks.logprobs(X, tg, top)
    V = X.shape[1]
    # exp of 16-bit logits is off by |t| e (|t| <= 30 counts); a lane's sums are of V / 256
    # entries, a few joins on top
    z = (V / 256 + 60) * 2 * E
    size = np.where(np.isfinite(lse), np.abs(lse), 0)
    live = np.where(np.isfinite(X), np.abs(X), 0).max(1, initial=0)
    err = z + 4 * E * (size + live)
    _close(r.lse, lse, err, "lse")
    _close(r.logprob, lp, err, "logprob")
    _close(r.entropy, ent, z * (4 + 3 * np.log(V + 1)), "entropy")
    if top:
        assert np.array_equal(r.top_index.cpu().numpy(), idx)
        _close(r.top_logprob, val, err[:, None], "top")
    return lse, ent


def _check_grad(x, targets, gl, ge, got):
    X, tg = _np(x), targets.cpu().numpy()
    g, h = _np(gl), _np(ge) if ge is not None else np.zeros(len(tg))
    want = blocks.logprobs_grad(X, tg, g, h)
    V = X.shape[1]
    u, tiny = ROUND[x.dtype]
    m = X.max(1, keepdims=True)
    m = np.where(np.isfinite(m), m, 0)
    p = np.exp(np.where(np.isfinite(X), X, -np.inf) - m)
    p /= np.maximum(p.sum(1, keepdims=True), 1e-300)
    logp = np.abs(np.log(np.where(p > 0, p, 1)))
    # p is off by the errors of lse and of exp; then the sums and products of the formula
    z = (V / 256 + 80) * 2 * E + 4 * E * (np.abs(m) + logp + 20)
    err = p * (np.abs(g)[:, None] + np.abs(h)[:, None] * (logp + np.log(V) + 1)) * 2 * z
    err += 4 * E * np.abs(g)[:, None] * (np.arange(V) == tg[:, None])
    _close(got, want, err + u * (np.abs(want) + err) + tiny + 2.0 ** -126, "d_logits")


LOGPROB = [(1, 1, 1), (1, 2, 2), (3, 5, 5), (2, 63, 20), (1, 9001, 64), (5, 4099, 3), (2, 33001, 8),
           (1, 65536, 1), (530, 300, 7), (600, 67, 0)]


@pytest.mark.parametrize("dt", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("T,V,top", LOGPROB)
def test_logprobs_and_gradient(T, V, top, dt):
    say(f"[logprob] tokens {T} vocab {V} top {top} {dt}")
    x = _randn(T + V, T, V, std=3.0)
    x[:, V // 2] += 9.0 * (torch.arange(T) % 2)
    x = x.to(dt).cuda()
    gen = torch.Generator().manual_seed(V)
    t = torch.randint(0, V, (T,), generator=gen)
    t[T // 2] = V // 2
    if T > 2:
        t[1] = -1
    t = t.cuda()
    r = jb.token_logprobs(x, t, top=top)
    _check_logprobs(x, t, top, r)
    gl, ge = _randn(7, T).cuda(), _randn(8, T).cuda()
    _check_grad(x, t, gl, ge, jb.token_logprobs_backward(x, t, r, gl, ge))
    _check_grad(x, t, gl, None, jb.token_logprobs_backward(x, t, r, gl))


@pytest.mark.parametrize("dt", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("V", [37, 5000, 40001])
def test_logprobs_of_masked_and_broken_rows(V, dt):
    low = torch.finfo(dt).min
    x = _randn(V, 12, V, std=2.0).to(dt)
    x[0] = -float("inf")                     # nothing left
    x[1] = -float("inf")
    x[1, V - 1] = 2.0                        # one entry left
    x[2, ::2] = -float("inf")
    x[3] = low                               # masked by the type's lowest value
    x[4] = low
    x[4, V // 3] = 1.0
    x[5, 7] = float("nan")
    x[6, V - 1] = float("inf")
    x[7] = 0.0                               # ties everywhere
    x[7, ::3] = -0.0
    x[8] = float(torch.finfo(dt).max)
    x[9, :V // 2] = low
    x[9, V // 2:] = -float("inf")
    x[10, 0] = float("nan")
    x[11] = torch.linspace(-20, 20, V).to(dt)   # every entry above those before it
    t = torch.tensor([3, V - 1, 0, 4, 5, 6, 7, 8, 9, V - 1, -1, V], dtype=torch.int64)
    x, t = x.cuda(), t.cuda()
    top = min(V, 20)
    r = jb.token_logprobs(x, t, top=top)
    _check_logprobs(x, t, top, r)
    gl, ge = _randn(1, 12).cuda(), _randn(2, 12).cuda()
    _check_grad(x, t, gl, ge, jb.token_logprobs_backward(x, t, r, gl, ge))


@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V,ld,first", [(1000, 1003, 0), (1001, 1001, 1), (4097, 4104, 3), (7, 9, 2)])
def test_logprobs_of_strided_and_unaligned_rows(V, ld, first, dt):
    T = 9
    base = _randn(5, T * ld + 8).to(dt).cuda()
    x = base[first:first + T * ld].view(T, ld)[:, :V]
    t = torch.arange(T).cuda() % V
    gl, ge = _randn(1, T).cuda(), _randn(2, T).cuda()
    r, s = jb.token_logprobs(x, t, top=5), jb.token_logprobs(x.contiguous(), t, top=5)
    _check_logprobs(x, t, 5, r)
    assert torch.equal(r.top_index, s.top_index)
    d = jb.token_logprobs_backward(x, t, r, gl, ge)
    _check_grad(x, t, gl, ge, d)
    # into a strided view, and in place: the same bits, nothing beside it touched
    out = torch.full_like(base, 7.0)
    view = out[first:first + T * ld].view(T, ld)[:, :V]
    jb.token_logprobs_backward(x, t, r, gl, ge, out=view)
    assert torch.equal(view, d)
    rest = out.clone()
    rest[first:first + T * ld].view(T, ld)[:, :V] = 7.0
    assert bool((rest == 7.0).all())
    kept = base.clone()
    jb.token_logprobs_backward(x, t, r, gl, ge, out=x)
    assert torch.equal(x, d)
    kept[first:first + T * ld].view(T, ld)[:, :V] = d
    assert torch.equal(base, kept)


def test_logprob_gradient_against_differences():
    T, V = 6, 700
    x = _randn(3, T, V, std=2.0).cuda()
    t = torch.tensor([0, 5, -1, 699, 300, 2]).cuda()
    gl, ge = _randn(1, T).cuda(), _randn(2, T).cuda()
    r = jb.token_logprobs(x, t)
    d = jb.token_logprobs_backward(x, t, r, gl, ge)
    v = _randn(4, T, V).cuda()
    h = 2.0 ** -7
    f = []
    for s in (h, -h):
        q = jb.token_logprobs(x + s * v, t)
        f.append(_np(gl) * _np(q.logprob) + _np(ge) * _np(q.entropy))
    got, want = (f[0] - f[1]) / (2 * h), (_np(d) * _np(v)).sum(1)
    # h^2 of third derivatives (of order 10 here), and fp32 results over 2 h
    assert np.all(np.abs(got - want) <= 10 * h * h * 10 / 6 + 1e-5 / h)


def test_logprobs_no_tokens_and_graph():
    r = jb.token_logprobs(torch.zeros(0, 50).cuda(), torch.zeros(0, dtype=torch.int64).cuda(), top=3)
    assert r.logprob.shape == (0,) and r.top_index.shape == (0, 3)
    x, t = _randn(1, 2, 30000).cuda(), torch.tensor([3, 29999]).cuda()
    gl = torch.ones(2).cuda()
    want = jb.token_logprobs(x, t, top=4)
    grad = jb.token_logprobs_backward(x, t, want, gl)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = jb.token_logprobs(x, t, top=4)
        d = jb.token_logprobs_backward(x, t, got, gl)
    for _ in range(3):
        for y in (*got, d):
            y.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((*got, d), (*want, grad)))


# ---- every shape of tile ----

# The launchers choose tiles by the sizes; these reach each of them with a last tile, a
# last chunk of k and a last round of stages that are not whole.
@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("T,d,f", [(40, 264, 1000), (70, 136, 4096), (100, 1000, 2752),
                                   (250, 72, 11008), (400, 4096, 1000), (700, 264, 6000),
                                   (3300, 520, 2048), (2100, 8, 2104), (129, 4104, 520)])
def test_gated_tiles(T, d, f, dt):
    say(f"[gated tiles] tokens {T} d {d} f {f} {dt}")
    x, wg, wu, dy = _gated_inputs(T, d, f, dt)
    y, pre = jb.gated_forward(x, wg, wu, save=True)
    dx, dwg, dwu = jb.gated_backward(x, wg, wu, dy, pre)
    X, G, U, D = (t.double() for t in (x, wg, wu, dy))
    a, b = X @ G.T, X @ U.T
    s = 1 / (1 + torch.exp(-a))
    da, db = D * b * s * (1 + a * (1 - s)), D * a * s
    u = ROUND[dt][0]
    for got, want in ((pre[0], a), (pre[1], b)):
        # fp32 sums of d products
        assert (got.double() - want).norm() <= (d + 2) ** 0.5 * 4 * E * want.norm()
    for got, want in ((y, a * s * b), (dx, da @ G + db @ U), (dwg, da.T @ X), (dwu, db.T @ X)):
        # one rounding of da and db and one of the result, of relative size u at most
        assert (got.double() - want).norm() <= 1.5 * u * want.norm()


@pytest.mark.parametrize("g", [0, 32, 64, 128])
@pytest.mark.parametrize("T,n,k", [(40, 1000, 512), (40, 4096, 384), (50, 10000, 1152),
                                   (70, 1000, 1152), (150, 4000, 384), (400, 4000, 1152),
                                   (200, 11008, 640), (1000, 4100, 384), (3000, 4100, 384),
                                   (33, 8200, 128), (66, 700, 2688), (130, 17, 896)])
def test_matmul_i8_tiles(T, n, k, g):
    say(f"[i8 tiles] tokens {T} n {n} k {k} group {g}")
    gen = torch.Generator(device="cuda").manual_seed(T)
    xq, wq = (torch.randint(-128, 128, (m, k), generator=gen, device="cuda", dtype=torch.int8)
              for m in (T, n))
    G = k // g if g else 1
    sx = torch.rand(T, generator=gen, device="cuda")
    sw = torch.randn(n, G, generator=gen, device="cuda")
    w = (wq.view(n, G, -1).double() * sw.double()[:, :, None]).view(n, k)
    want = (xq.double() @ w.T) * sx.double()[:, None]
    for dt in (torch.float32, torch.bfloat16):
        y = jb.matmul_i8(xq, sx, wq, sw, dtype=dt)
        # G + 4 roundings in fp32 and the output's
        assert (y.double() - want).norm() <= ((G + 4) * E + 1.2 * ROUND[dt][0]) * want.norm()


def test_matmul_i8_scales_of_other_channels_do_not_reach_a_row():
    # the loads of a row's scales run past its last group: infinities there stay there
    for T in (3, 40, 100, 300):
        n, k, g = 200, 192, 64
        xq = torch.ones(T, k, dtype=torch.int8).cuda()
        wq = torch.ones(n, k, dtype=torch.int8).cuda()
        sw = torch.ones(n, k // g)
        sw[1::2] = float("inf")
        y = jb.matmul_i8(xq, torch.ones(T).cuda(), wq, sw.cuda(), dtype=torch.float32)
        assert bool((y[:, 0::2] == k).all()) and bool(torch.isinf(y[:, 1::2]).all())


def test_example_runs_a_refined_block():
    import importlib.util
    import os
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples",
                        "refined_block.py")
    spec = importlib.util.spec_from_file_location("refined_block", path)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    r = module.main(tokens=256, d=256, f=512, vocab=1000, sweeps=3, log=say)
    assert all(np.isfinite(v) for v in r.values())
    assert r["after"] < r["refined"] and r["base"] < r["refined"] + 0.05


@pytest.mark.parametrize("act", sorted(jb.ACTIVATIONS))
def test_gated_values_whose_square_overflows(act):
    # a = +-2^70: act(a) is a or 0 and act'(a) 1 or 0; every result is a power of two
    say(f"[gated] {act} at 2^70")
    T, d, f = 2, 8, 8
    x, wg, wu = torch.zeros(T, d), torch.zeros(f, d), torch.zeros(f, d)
    x[0, 0], x[1, 0], x[:, 1] = 2.0 ** 40, -2.0 ** 40, 1.0
    wg[:, 0], wu[:, 1] = 2.0 ** 30, 2.0 ** -3
    x, wg, wu = (t.bfloat16().cuda() for t in (x, wg, wu))
    y, pre = jb.gated_forward(x, wg, wu, act=act, save=True)
    dx, dwg, dwu = jb.gated_backward(x, wg, wu, torch.ones_like(y), pre, act=act)
    assert (y[0] == 2.0 ** 67).all() and (y[1] == 0).all()
    want = torch.zeros(T, d)
    want[0, 0], want[0, 1] = 2.0 ** 30, 2.0 ** 70
    assert torch.equal(dx.float().cpu(), want)
    for got, da in ((dwg, 2.0 ** -3), (dwu, 2.0 ** 70)):
        want = torch.zeros(f, d)
        want[:, 0], want[:, 1] = da * 2.0 ** 40, da
        assert torch.equal(got.float().cpu(), want)


@pytest.mark.parametrize("g", [32, 64, 128])
@pytest.mark.parametrize("T,n,k", [(3000, 4097, 384), (700, 2049, 640), (300, 1025, 896)])
def test_matmul_i8_last_tile_of_one_channel(T, n, k, g):
    # the loads of its scales run past the last group of the last channel
    test_matmul_i8_tiles(T, n, k, g)


@pytest.mark.parametrize("g", [0, 32, 64, 128])
@pytest.mark.parametrize("T,n,k", [(1993, 6966, 128), (611, 11008, 256), (2047, 1001, 2048),
                                   (150, 11008, 2176), (1030, 1000, 4096), (260, 4096, 1024),
                                   (150, 1000, 4096), (1100, 4096, 4096)])
def test_matmul_i8_tiles_of_many_work_groups(T, n, k, g):
    test_matmul_i8_tiles(T, n, k, g)
