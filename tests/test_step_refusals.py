"""What the entry points of the operators around a block refuse (CPU only: every call fails its
checks)."""

import contextlib
import ctypes

import pytest
import torch

from paper_2609_38599_amd import binding as jb
from tests.test_blocks_refusals import FAKE, OFF, _Placed, _placed

# (with a GPU a check that is lost would let a kernel loose on host memory)
pytestmark = pytest.mark.skipif(torch.cuda.is_available(), reason="host tensors stand in for a GPU's")

F32, BF16, I64 = torch.float32, torch.bfloat16, torch.int64
E8 = torch.float8_e4m3fn


@pytest.fixture(scope="module")
def lib():
    return jb.load_library()


def _f(x):
    return ctypes.c_float(x)


def test_norm_entry_points_check_arguments(lib):
    f = lambda **k: lib.jarq_rms_norm(*[{**dict(  # noqa: E731
        dtype=2, gt=2, t=4, c=64, x=FAKE, res=None, g=FAKE, eps=_f(1e-6), h=None, y=FAKE, st=None), **k}[n]
        for n in ("dtype", "gt", "t", "c", "x", "res", "g", "eps", "h", "y", "st")])
    bad = (dict(dtype=3), dict(gt=1), dict(t=-1), dict(t=(1 << 22) + 1), dict(c=0), dict(c=(1 << 20) + 1),
           dict(x=None), dict(x=ctypes.c_void_p(1 << 20 | 1)), dict(g=None), dict(gt=0, g=OFF), dict(res=FAKE),
           dict(h=FAKE), dict(res=FAKE, h=FAKE), dict(y=None), dict(eps=_f(0.0)), dict(eps=_f(-1.0)), dict(eps=_f(1e-40)),
           dict(eps=_f(float("nan"))), dict(eps=_f(float("inf"))))
    for k in bad:
        assert f(**k) == jb.JARQ_EINVAL, k
    assert f(t=0, x=None, y=None) == jb.JARQ_OK
    q = lambda **k: lib.jarq_rms_norm_i8(*[{**dict(  # noqa: E731
        dtype=2, gt=2, t=4, c=64, x=FAKE, res=None, g=FAKE, eps=_f(1e-6), h=None, q=FAKE, s=FAKE, st=None), **k}[n]
        for n in ("dtype", "gt", "t", "c", "x", "res", "g", "eps", "h", "q", "s", "st")])
    for k in bad[:-1] + (dict(c=40), dict(c=131072), dict(s=None), dict(s=OFF), dict(q=None), dict(q=OFF)):
        if "y" not in k and k != dict(res=FAKE, h=FAKE):
            assert q(**k) == jb.JARQ_EINVAL, k
    assert q(t=0, x=None, q=None, s=None) == jb.JARQ_OK
    need = lib.jarq_rms_norm_workspace_bytes(4, 64)
    assert need > 0 and lib.jarq_rms_norm_workspace_bytes(-1, 64) == 0
    assert lib.jarq_rms_norm_workspace_bytes(4, 0) == 0 and lib.jarq_rms_norm_workspace_bytes(0, 64) > 0
    b = lambda **k: lib.jarq_rms_norm_backward(*[{**dict(  # noqa: E731
        dtype=2, gt=2, t=4, c=64, h=FAKE, g=FAKE, dy=FAKE, dh=None, eps=_f(1e-6), dx=FAKE, dg=FAKE, ws=FAKE,
        n=need, st=None), **k}[n]
        for n in ("dtype", "gt", "t", "c", "h", "g", "dy", "dh", "eps", "dx", "dg", "ws", "n", "st")])
    odd = ctypes.c_void_p(1 << 20 | 1)
    for k in (dict(dtype=4), dict(gt=1), dict(c=0), dict(h=None), dict(dy=None), dict(dh=odd), dict(dx=odd),
              dict(dg=odd), dict(gt=0, dg=OFF), dict(eps=_f(0.0))):
        assert b(**k) == jb.JARQ_EINVAL, k
    assert b(ws=None) == jb.JARQ_EWORKSPACE and b(n=need - 1) == jb.JARQ_EWORKSPACE


def test_linear_logprob_entry_points_check_arguments(lib):
    need = lib.jarq_linear_logprobs_workspace_bytes(4, 64, 100)
    for bad in ((-1, 64, 100), ((1 << 22) + 1, 64, 100), (4, 0, 100), (4, 12, 100), (4, (1 << 20) + 8, 100),
                (4, 64, 0), (4, 64, (1 << 22) + 1)):
        assert lib.jarq_linear_logprobs_workspace_bytes(*bad) == 0
        assert lib.jarq_linear_logprobs_backward_workspace_bytes(*bad) == 0
    f = lambda **k: lib.jarq_linear_logprobs(*[{**dict(  # noqa: E731
        dtype=2, t=4, d=64, v=100, x=FAKE, w=FAKE, tg=FAKE, lp=FAKE, lse=FAKE, rest=FAKE, ws=FAKE, n=need,
        st=None), **k}[n]
        for n in ("dtype", "t", "d", "v", "x", "w", "tg", "lp", "lse", "rest", "ws", "n", "st")])
    for k in (dict(dtype=0), dict(dtype=3), dict(d=60), dict(v=0), dict(x=None), dict(x=OFF), dict(w=OFF),
              dict(w=None), dict(tg=None), dict(lp=None), dict(lse=OFF), dict(rest=None)):
        assert f(**k) == jb.JARQ_EINVAL, k
    assert f(ws=None) == jb.JARQ_EWORKSPACE and f(n=need - 1) == jb.JARQ_EWORKSPACE
    assert f(t=0, x=None, tg=None, lp=None) == jb.JARQ_OK
    need = lib.jarq_linear_logprobs_backward_workspace_bytes(4, 64, 100)
    b = lambda **k: lib.jarq_linear_logprobs_backward(*[{**dict(  # noqa: E731
        dtype=2, t=4, d=64, v=100, x=FAKE, w=FAKE, tg=FAKE, lp=FAKE, lse=FAKE, rest=FAKE, g=FAKE, h=None,
        dx=FAKE, dw=FAKE, ws=FAKE, n=need, st=None), **k}[n]
        for n in ("dtype", "t", "d", "v", "x", "w", "tg", "lp", "lse", "rest", "g", "h", "dx", "dw", "ws", "n",
                  "st")])
    for k in (dict(dtype=0), dict(d=60), dict(v=0), dict(x=None), dict(w=None), dict(tg=None), dict(lp=None),
              dict(lse=None), dict(rest=OFF), dict(g=None), dict(h=OFF), dict(dx=OFF), dict(dw=OFF)):
        assert b(**k) == jb.JARQ_EINVAL, k
    assert b(ws=None) == jb.JARQ_EWORKSPACE and b(n=need - 1) == jb.JARQ_EWORKSPACE


class _Tensor(ctypes.Structure):
    _fields_ = [("grad", ctypes.c_void_p), ("param", ctypes.c_void_p), ("param_out", ctypes.c_void_p),
                ("numel", ctypes.c_int64)]


MB = 1 << 20


def _adamw(lib, dtype=2, bits=8, tensors=((16, 32, 32, 100), (17, 33, 33, 300)), count=None, old=None,
           new=None, **options):
    # (addresses in MiB; none is read)
    table = (_Tensor * max(1, len(tensors)))(*[
        _Tensor(*[None if p is None else int(p * MB) for p in t[:3]], t[3]) for t in tensors])
    first = (64, 65, 66, 67, 68) if old is None else old
    second = first if new is None else new
    a, b = (jb._AdamWArrays(*[None if p is None else int(p * MB) for p in s]) for s in (first, second))
    o = dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.1, step=1, seed=0, lr_at=None,
             step_at=None, grad_mul=None)
    o.update(options)
    return lib.jarq_adamw_step(dtype, bits, len(tensors) if count is None else count,
                               ctypes.addressof(table), a, b, jb._AdamWOptions(*o.values()), None)


def test_adamw_checks_arguments(lib):
    nan, inf = float("nan"), float("inf")
    other = (74, 75, 76, 77, 78)
    apart = ((16, 32, 42, 100), (17, 33, 43, 300))
    for k in (dict(dtype=3), dict(bits=16), dict(count=-1), dict(lr=-1.0), dict(lr=nan), dict(lr=inf),
              dict(beta1=1.0), dict(beta1=-0.1), dict(beta2=nan), dict(beta2=1.0), dict(eps=0.0), dict(eps=1e-50),
              dict(eps=inf), dict(weight_decay=-1.0), dict(weight_decay=inf), dict(step=0), dict(step=-3),
              dict(lr_at=2), dict(step_at=MB + 4), dict(grad_mul=MB + 1),
              dict(tensors=((16, 32, 32, -1),)), dict(tensors=((16, 32, 32, (1 << 40) + 1),)),
              dict(tensors=((16, None, None, 4),)), dict(tensors=((16 + 1 / MB, 32, 32, 4),)),
              dict(old=(64, 65, 66, 67, None)), dict(old=(None, 65, 66, 67, 68)), dict(old=(64, None, 66, 67, 68)),
              dict(old=(64 + 8 / MB, 65, 66, 67, 68)),
              # not in place: parameters and state go together, and gradients are all there
              dict(new=other), dict(tensors=apart), dict(tensors=((None, 32, 42, 100),), new=other),
              dict(tensors=apart, new=(64, 75, 76, 77, 78))):
        assert _adamw(lib, **k) == jb.JARQ_EINVAL, k
    assert _adamw(lib, tensors=()) == jb.JARQ_OK
    assert _adamw(lib, tensors=((None, None, None, 0),)) == jb.JARQ_OK


def test_adamw_refuses_arrays_that_overlap(lib):
    # (a tensor twice would be advanced by two work-groups at once)
    near = 32 + 64 / MB
    other = (74, 75, 76, 77, 78)
    for k in (dict(tensors=((16, 32, 32, 100), (17, 32, 32, 100))),
              dict(tensors=((16, 32, 32, 100), (17, near, near, 100))),
              dict(tensors=((32, 32, 32, 100),)),
              dict(tensors=((near, 32, 32, 100),)),
              dict(tensors=((64, 32, 32, 100),)),
              dict(tensors=((16, 64, 64, 100),)),
              dict(old=(64, 64, 66, 67, 68)),
              dict(old=(64, 65, 65, 67, 68)),
              dict(old=(64, 65, 66, 67, 67)),
              dict(grad_mul=32 * MB),
              dict(tensors=((16, 32, 42, 100), (17, 42, 43, 100)), new=other),
              dict(tensors=((16, 32, 64, 100),), new=other),
              dict(tensors=((16, 32, 42, 100),), new=(74, 66, 76, 77, 78))):
        assert _adamw(lib, **k) == jb.JARQ_EINVAL, k


def test_adamw_refuses_scalars_in_what_it_writes(lib):
    # every byte of them: a step number's upper half lies where the parameters begin
    late = 32 + 4 / MB
    for k in (dict(step_at=32 * MB, tensors=((16, late, late, 100),)), dict(step_at=64 * MB),
              dict(lr_at=32 * MB + 196), dict(lr_at=68 * MB), dict(grad_mul=65 * MB + 4)):
        assert _adamw(lib, **k) == jb.JARQ_EINVAL, k


def test_adamw_state_length(lib):
    f = lambda *n: int(lib.jarq_adamw_state_length(len(n), (ctypes.c_int64 * max(1, len(n)))(*n)))  # noqa: E731
    assert f() == 0 and f(0) == 0 and f(1) == 128 and f(128, 129) == 384
    assert f(-1) == -1 and f(1 << 50) == -1 and lib.jarq_adamw_state_length(-1, None) == -1
    assert lib.jarq_adamw_state_length(2, None) == -1


# ---- the binding ----

def _calls():
    """(name, call, its tensors by argument): every entry point on tensors of one GPU."""
    x, w, g = _placed(0, 4, 64), _placed(0, 8, 64), _placed(0, 64)
    dy, dh, h, y = (_placed(0, 4, 64) for _ in range(4))
    q, sc = _placed(0, 4, 64, dtype=torch.int8), _placed(0, 4, 1, dtype=F32)
    t, v = _placed(0, 4, dtype=I64), _placed(0, 4, dtype=F32)
    r = jb.LinearLogprobs(v, v, v)
    p, gr = _placed(0, 3, 50), _placed(0, 3, 50)
    m, vv = (torch.zeros(256, dtype=torch.uint8).view(E8).as_subclass(_Placed) for _ in range(2))
    state = dict(master=_placed(0, 256, dtype=F32), m=m, v=vv, m_exp=_placed(0, 2, dtype=torch.uint8),
                 v_exp=_placed(0, 2, dtype=torch.uint8))

    def step(p, g, stream=None, **k):
        return jb.adamw_step([p], [g], jb.AdamWState(**{**state, **k}), 1, 1e-3, stream=stream)

    return [
        ("rms_norm", lambda **k: jb.rms_norm(**k), dict(X=x, residual=h, gain=g, out=y, sum_out=dy)),
        ("rms_norm_i8", lambda **k: jb.rms_norm_i8(**k),
         dict(X=x, residual=h, gain=g, out=q, scale=sc, sum_out=dy)),
        ("rms_norm_backward", lambda **k: jb.rms_norm_backward(**k), dict(H=h, gain=g, dY=dy, dH=dh)),
        ("linear_logprobs", lambda **k: jb.linear_logprobs(**k), dict(X=x, W=w, targets=t)),
        ("linear_logprobs_backward", lambda **k: jb.linear_logprobs_backward(forward=r, **k),
         dict(X=x, W=w, targets=t, d_logprob=v, d_lse=v)),
        ("adamw_step", step, dict(p=p, g=gr, **state)),
    ]


NAMES = [c[0] for c in _calls()]
SAID = {"p": r"params\[0\]", "g": r"grads\[0\]"}


@pytest.mark.parametrize("name", NAMES)
def test_tensors_off_the_current_gpu_are_refused(name, monkeypatch):
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0)
    call, tensors = next(c[1:] for c in _calls() if c[0] == name)

    def move(t):
        t = t.clone().as_subclass(_Placed)
        t.at = 1
        return t

    with pytest.raises(ValueError, match="cuda:1.*cuda:0 is the current"):
        call(**{n: move(t) for n, t in tensors.items()})
    for moved, t in list(tensors.items())[1:]:
        said = SAID.get(moved, moved)
        with pytest.raises(ValueError, match=f"{said} must be on cuda:0"):
            call(**{**tensors, moved: move(t)})


@pytest.mark.parametrize("name", NAMES)
def test_streams_of_another_gpu_are_refused(name, monkeypatch):
    class Stream:
        device_index, cuda_stream = 1, 0

    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0)
    monkeypatch.setattr(jb, "_on", lambda stream: contextlib.nullcontext())
    empty = torch.empty
    monkeypatch.setattr(torch, "empty",
                        lambda *a, **k: empty(*a, **k).as_subclass(_Placed))   # the call's own
    call, tensors = next(c[1:] for c in _calls() if c[0] == name)
    with pytest.raises(ValueError, match="stream must be of cuda:0"):
        call(**tensors, stream=Stream())


WRONG = [
    ("rms_norm", dict(gain=_placed(0, 63)), "gain must be"),
    ("rms_norm", dict(gain=_placed(0, 64, dtype=torch.float16)), "gain must be"),
    ("rms_norm", dict(residual=_placed(0, 3, 64)), "residual must"),
    ("rms_norm", dict(residual=_placed(0, 4, 64, dtype=F32)), "residual must be"),
    ("rms_norm", dict(residual=None), "sum_out needs"),
    ("rms_norm", dict(sum_out=_placed(0, 4, 63)), "sum_out must"),
    ("rms_norm", dict(out=_placed(0, 5, 64)), "out must"),
    ("rms_norm", dict(out=_placed(0, 64, 4).t()), "out must be contiguous"),
    ("rms_norm", dict(X=_placed(0, 64)), "X must be"),
    ("rms_norm", dict(X=_placed(0, 64, 4).t(), residual=None, sum_out=None), "X must be contiguous"),
    ("rms_norm_i8", dict(scale=_placed(0, 3, 1, dtype=F32)), "scale"),
    ("rms_norm_i8", dict(out=_placed(0, 4, 60, dtype=torch.int8)), "out must"),
    ("rms_norm_backward", dict(dY=_placed(0, 3, 64)), "dY and dH must"),
    ("rms_norm_backward", dict(dH=_placed(0, 4, 60)), "dY and dH must"),
    ("rms_norm_backward", dict(dY=_placed(0, 4, 64, dtype=F32)), "dY must be"),
    ("linear_logprobs", dict(W=_placed(0, 8, 56)), "W must be"),
    ("linear_logprobs", dict(W=_placed(0, 8, 64, dtype=torch.float16)), "W must be"),
    ("linear_logprobs", dict(targets=_placed(0, 3, dtype=I64)), "targets must be"),
    ("linear_logprobs", dict(targets=_placed(0, 4, dtype=torch.int32)), "targets must be"),
    ("linear_logprobs_backward", dict(d_logprob=_placed(0, 5, dtype=F32)), "d_logprob must be"),
    ("linear_logprobs_backward", dict(d_lse=_placed(0, 4, 1, dtype=F32)), "d_lse must be"),
    ("adamw_step", dict(g=_placed(0, 50, 2)), "must have 150 values"),
    ("adamw_step", dict(g=_placed(0, 3, 50, dtype=F32)), r"grads\[0\] must be"),
    ("adamw_step", dict(g=_placed(0, 50, 3).t()), r"grads\[0\] must be contiguous"),
    ("adamw_step", dict(master=None), "state.master must be a tensor"),
    ("adamw_step", dict(master=_placed(0, 255, dtype=F32)), r"state.master must be \[256\]"),
    ("adamw_step", dict(m=_placed(0, 256, dtype=F32)), "state.m must be"),
    ("adamw_step", dict(v_exp=None), "state.v_exp must be a tensor"),
    ("adamw_step", dict(m_exp=None), "state.m must be|state.v_exp must be"),
    ("adamw_step", dict(v_exp=_placed(0, 1, dtype=torch.uint8)), r"state.v_exp must be \[2\]"),
]


@pytest.mark.parametrize("name,wrong,says", WRONG)
def test_wrong_shapes_and_types_are_refused(name, wrong, says, monkeypatch):
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda d: 0, raising=False)
    call, tensors = next(c[1:] for c in _calls() if c[0] == name)
    with pytest.raises((ValueError, TypeError), match=says):
        call(**{**tensors, **wrong})


def test_adamw_state_is_refused_for_what_it_cannot_hold(monkeypatch):
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0)
    with pytest.raises(ValueError, match="bits"):
        jb.adamw_state([_placed(0, 4)], bits=16)
    with pytest.raises(ValueError, match="a tensor"):
        jb.adamw_state([])
    with pytest.raises(TypeError, match="float32, float16 or bfloat16"):
        jb.adamw_state([_placed(0, 4, dtype=torch.float64)])
    with pytest.raises(TypeError, match=r"params\[1\]"):
        jb.adamw_state([_placed(0, 4), _placed(0, 4, dtype=F32)])
    with pytest.raises(ValueError, match="device tensor"):
        jb.adamw_state([torch.zeros(4)])
