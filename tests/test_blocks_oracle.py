"""The operators that run, train and evaluate refined layers: their float64 definitions
against differences, and their entry points' argument checks (CPU only)."""

import ctypes

import numpy as np
import pytest
import torch

from oracle import blocks
from paper_2609_38599_amd import binding as jb

FAKE = ctypes.c_void_p(1 << 20)          # aligned, never dereferenced
OFF = ctypes.c_void_p((1 << 20) + 2)     # aligned to two bytes alone


@pytest.fixture(scope="module")
def lib():
    return jb.load_library()


@pytest.mark.parametrize("act", ["silu", "gelu", "gelu_tanh"])
def test_gated_gradient_against_differences(act):
    rng = np.random.default_rng(3)
    X, Wg, Wu = rng.standard_normal((5, 8)), rng.standard_normal((6, 8)), rng.standard_normal((6, 8))
    dY = rng.standard_normal((5, 6))
    grads = blocks.gated_grad(X, Wg, Wu, dY, act)[:3]
    h = 1e-5
    for k, M in enumerate((X, Wg, Wu)):
        V = rng.standard_normal(M.shape)
        args = [[X, Wg, Wu], [X, Wg, Wu]]
        args[0][k], args[1][k] = M + h * V, M - h * V
        up, down = ((dY * blocks.gated(*a, act)[0]).sum() for a in args)
        # central differences: h^2 f''' / 6 and 1e-16 |f| / h
        assert abs((up - down) / (2 * h) - (grads[k] * V).sum()) < 1e-7 * (1 + np.abs(grads[k] * V).sum())


@pytest.mark.parametrize("masked", [False, True])
def test_logprob_gradient_against_differences(masked):
    rng = np.random.default_rng(4)
    x = rng.standard_normal((4, 9)) * 2
    if masked:
        x[:, 5] = -np.inf
        x[1, :] = -np.inf
    t = np.array([0, 3, -1, 8])
    gl, ge = rng.standard_normal(4), rng.standard_normal(4)
    d = blocks.logprobs_grad(x, t, gl, ge)
    h = 1e-5
    for r in (0, 2, 3):
        for v in range(9):
            if x[r, v] == -np.inf:
                assert d[r, v] == 0
                continue
            f = []
            for s in (h, -h):
                y = x.copy()
                y[r, v] += s
                lp, ent, *_ = blocks.logprobs(y, t, 1)
                f.append(gl[r] * lp[r] + ge[r] * ent[r])
            assert abs((f[0] - f[1]) / (2 * h) - d[r, v]) < 1e-8
    if masked:
        assert np.all(d[1] == 0)


def test_gated_entry_points_check_arguments(lib):
    fwd = lambda **k: lib.jarq_gated_forward(*[{**dict(  # noqa: E731
        dtype=2, act=0, t=4, d=64, f=64, X=FAKE, Wg=FAKE, Wu=FAKE, Y=FAKE, pre=None, st=None), **k}[n]
        for n in ("dtype", "act", "t", "d", "f", "X", "Wg", "Wu", "Y", "pre", "st")])
    for bad in (dict(dtype=0), dict(dtype=3), dict(act=3), dict(act=-1), dict(t=-1),
                dict(t=(1 << 22) + 1), dict(d=60), dict(d=0), dict(f=12), dict(f=(1 << 20) + 8),
                dict(X=None), dict(X=OFF), dict(Wg=OFF), dict(Wu=None), dict(Y=OFF), dict(pre=OFF)):
        assert fwd(**bad) == jb.JARQ_EINVAL, bad
    assert fwd(t=0, X=None, Y=None) == jb.JARQ_OK
    assert lib.jarq_gated_workspace_bytes(4, 60, 64) == 0
    assert lib.jarq_gated_workspace_bytes(-1, 64, 64) == 0
    need = lib.jarq_gated_workspace_bytes(4, 64, 64)
    assert need >= 2 * 4 * 64 * 2
    bwd = lambda **k: lib.jarq_gated_backward(*[{**dict(  # noqa: E731
        dtype=1, act=0, t=4, d=64, f=64, X=FAKE, Wg=FAKE, Wu=FAKE, dY=FAKE, pre=FAKE, dX=None,
        dWg=None, dWu=None, ws=FAKE, n=need, st=None), **k}[n]
        for n in ("dtype", "act", "t", "d", "f", "X", "Wg", "Wu", "dY", "pre", "dX", "dWg", "dWu",
                  "ws", "n", "st")])
    for bad in (dict(dtype=0), dict(d=4), dict(pre=None), dict(pre=OFF), dict(dY=OFF), dict(dX=OFF),
                dict(dWg=OFF), dict(dWu=OFF)):
        assert bwd(**bad) == jb.JARQ_EINVAL, bad
    for bad in (dict(ws=None), dict(n=need - 1), dict(ws=ctypes.c_void_p((1 << 20) + 128))):
        assert bwd(**bad) == jb.JARQ_EWORKSPACE, bad


def test_i8_entry_points_check_arguments(lib):
    mm = lambda **k: lib.jarq_matmul_i8(*[{**dict(  # noqa: E731
        dtype=2, t=4, n=8, k=128, g=0, Xq=FAKE, sx=FAKE, Wq=FAKE, sw=FAKE, Y=FAKE, st=None), **k}[n]
        for n in ("dtype", "t", "n", "k", "g", "Xq", "sx", "Wq", "sw", "Y", "st")])
    for bad in (dict(dtype=3), dict(t=-1), dict(n=0), dict(k=24), dict(k=131072), dict(g=16),
                dict(k=96, g=64), dict(g=256), dict(Xq=OFF), dict(Wq=None), dict(sw=OFF),
                dict(sx=None), dict(Y=None), dict(dtype=0, Y=OFF)):
        assert mm(**bad) == jb.JARQ_EINVAL, bad
    assert mm(t=0, Xq=None, sx=None, Y=None) == jb.JARQ_OK
    q = lib.jarq_quant_rows_i8
    assert q(0, FAKE, 4, 24, FAKE, FAKE, None) == jb.JARQ_EINVAL
    assert q(5, FAKE, 4, 32, FAKE, FAKE, None) == jb.JARQ_EINVAL
    assert q(0, OFF, 4, 32, FAKE, FAKE, None) == jb.JARQ_EINVAL
    assert q(0, None, 0, 32, None, None, None) == jb.JARQ_OK
    need = lib.jarq_linear_i8_workspace_bytes(4, 128)
    assert need >= 4 * 128 + 16 and lib.jarq_linear_i8_workspace_bytes(4, 24) == 0
    lin = lambda *a: lib.jarq_linear_i8(2, 4, 8, 128, 32, FAKE, FAKE, FAKE, FAKE, *a, None)  # noqa: E731
    assert lin(FAKE, need - 1) == jb.JARQ_EWORKSPACE
    assert lin(None, need) == jb.JARQ_EWORKSPACE
    p = jb.make_params(64, 256, 64, 3, 5)
    codes = lambda *a: lib.jarq_codes_i8(ctypes.byref(p), *a, None)  # noqa: E731
    assert codes(OFF, FAKE, FAKE, FAKE) == jb.JARQ_EINVAL
    assert codes(FAKE, FAKE, FAKE, None) == jb.JARQ_EINVAL
    assert lib.jarq_codes_i8(None, FAKE, FAKE, FAKE, FAKE, None) == jb.JARQ_EINVAL


def test_logprob_entry_points_check_arguments(lib):
    need = lib.jarq_token_logprobs_workspace_bytes(4, 100, 5)
    assert need > 0
    for bad in ((-1, 100, 5), (4, 0, 0), (4, 100, 65), (4, 100, -1), (4, 3, 5), ((1 << 22) + 1, 8, 0)):
        assert lib.jarq_token_logprobs_workspace_bytes(*bad) == 0, bad
    f = lambda **k: lib.jarq_token_logprobs(*[{**dict(  # noqa: E731
        dtype=2, x=FAKE, ld=100, t=4, v=100, tg=FAKE, top=5, lp=FAKE, en=FAKE, lse=FAKE, ti=FAKE,
        tl=FAKE, ws=FAKE, n=need, st=None), **k}[n]
        for n in ("dtype", "x", "ld", "t", "v", "tg", "top", "lp", "en", "lse", "ti", "tl", "ws",
                  "n", "st")])
    for bad in (dict(dtype=4), dict(x=None), dict(dtype=0, x=OFF), dict(ld=99), dict(t=-1), dict(v=0),
                dict(tg=OFF), dict(top=65), dict(top=101), dict(lp=None), dict(en=OFF),
                dict(ti=None), dict(tl=None)):
        assert f(**bad) == jb.JARQ_EINVAL, bad
    assert f(ws=None) == jb.JARQ_EWORKSPACE
    assert f(t=0, x=None, tg=None, lp=None) == jb.JARQ_OK
    b = lambda **k: lib.jarq_token_logprobs_backward(*[{**dict(  # noqa: E731
        dtype=2, x=FAKE, ld=100, t=4, v=100, tg=FAKE, lse=FAKE, en=FAKE, dl=FAKE, de=None, d=FAKE,
        ldd=100, st=None), **k}[n]
        for n in ("dtype", "x", "ld", "t", "v", "tg", "lse", "en", "dl", "de", "d", "ldd", "st")])
    for bad in (dict(lse=None), dict(dl=None), dict(de=FAKE, en=None), dict(d=None), dict(ldd=99),
                dict(dtype=0, d=OFF)):
        assert b(**bad) == jb.JARQ_EINVAL, bad


def test_binding_refuses_wrong_shapes_and_types():
    x = torch.zeros(4, 64, dtype=torch.bfloat16)
    w = torch.zeros(8, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        jb.gated_forward(x, w, w[:7], act="silu")
    with pytest.raises(ValueError):
        jb.gated_forward(x, w, w, act="relu")
    with pytest.raises(ValueError):
        jb.gated_forward(x, w, w)                       # host tensors
    with pytest.raises(ValueError):
        jb.linear_i8(x, torch.zeros(8, 32, dtype=torch.int8), torch.zeros(8, 1))
    with pytest.raises(ValueError):
        jb.linear_i8(x, torch.zeros(8, 64, dtype=torch.int8), torch.zeros(8, 3))
    with pytest.raises(ValueError):
        jb.token_logprobs(x, torch.zeros(4, dtype=torch.int64))
    with pytest.raises(ValueError):
        jb.token_logprobs(x[0], torch.zeros(4, dtype=torch.int64))
