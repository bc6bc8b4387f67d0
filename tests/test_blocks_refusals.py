"""What the entry points of the operators that run, train and evaluate refined layers refuse,
beside test_blocks_oracle.py (CPU only: every call fails its checks)."""

import contextlib
import ctypes

import pytest
import torch

from paper_2609_38599_amd import binding as jb

# (with a GPU a check that is lost would let a kernel loose on host memory)
pytestmark = pytest.mark.skipif(torch.cuda.is_available(), reason="host tensors stand in for a GPU's")

FAKE = ctypes.c_void_p(1 << 20)          # aligned, never dereferenced
OFF = ctypes.c_void_p((1 << 20) + 2)     # aligned to two bytes alone


@pytest.fixture(scope="module")
def lib():
    return jb.load_library()


def test_kept_logprob_entry_points_check_arguments(lib):
    need = lib.jarq_token_logprobs_workspace_bytes(4, 100, 5)
    f = lambda **k: lib.jarq_token_logprobs_keep(*[{**dict(  # noqa: E731
        dtype=2, x=FAKE, ld=100, t=4, v=100, tg=FAKE, top=5, lp=FAKE, en=FAKE, lse=FAKE, rest=FAKE,
        ti=FAKE, tl=FAKE, ws=FAKE, n=need, st=None), **k}[n]
        for n in ("dtype", "x", "ld", "t", "v", "tg", "top", "lp", "en", "lse", "rest", "ti", "tl",
                  "ws", "n", "st")])
    for bad in (dict(dtype=4), dict(x=None), dict(ld=99), dict(v=0), dict(top=101), dict(lp=None),
                dict(lse=OFF), dict(rest=OFF), dict(ti=None)):
        assert f(**bad) == jb.JARQ_EINVAL, bad
    assert f(ws=None) == jb.JARQ_EWORKSPACE and f(n=need - 1) == jb.JARQ_EWORKSPACE
    assert f(t=0, x=None, tg=None, lp=None) == jb.JARQ_OK
    b = lambda **k: lib.jarq_token_logprobs_keep_backward(*[{**dict(  # noqa: E731
        dtype=2, x=FAKE, ld=100, t=4, v=100, tg=FAKE, lse=FAKE, rest=FAKE, en=FAKE, dl=FAKE,
        de=None, d=FAKE, ldd=100, st=None), **k}[n]
        for n in ("dtype", "x", "ld", "t", "v", "tg", "lse", "rest", "en", "dl", "de", "d", "ldd",
                  "st")])
    for bad in (dict(lse=None), dict(rest=None), dict(rest=OFF), dict(dl=None), dict(d=None),
                dict(de=FAKE, en=None), dict(ldd=99)):
        assert b(**bad) == jb.JARQ_EINVAL, bad
    assert b(t=0, x=None, rest=None, lse=None, d=None) == jb.JARQ_OK


class _Placed(torch.Tensor):
    """A host tensor that says it is dense on a GPU."""

    at = 0
    is_cuda = property(lambda self: True)

    def get_device(self):
        return self.at


def _placed(at, *shape, dtype=torch.bfloat16):
    t = torch.zeros(*shape, dtype=dtype).as_subclass(_Placed)
    t.at = at
    return t


def _calls():
    """(name, call, its tensors by argument): every entry point on tensors of one GPU."""
    f32, i8 = torch.float32, torch.int8
    x, w, w2 = _placed(0, 4, 64), _placed(0, 8, 64), _placed(0, 8, 64)
    dy, pre = _placed(0, 4, 8), _placed(0, 2, 4, 8, dtype=f32)
    xq, wq = _placed(0, 4, 64, dtype=i8), _placed(0, 8, 64, dtype=i8)
    sx, sw = _placed(0, 4, 1, dtype=f32), _placed(0, 8, 1, dtype=f32)
    t, g = _placed(0, 4, dtype=torch.int64), _placed(0, 4, dtype=f32)
    r = jb.TokenLogprobs(g, g, g, None, None)
    p = jb.make_params(8, 64, 64, 3, 1)
    codes, zeros = _placed(0, 8, 64, dtype=torch.uint8), _placed(0, 8, 1, dtype=torch.int32)
    return [
        ("gated_forward", lambda **k: jb.gated_forward(**k), dict(X=x, Wg=w, Wu=w2)),
        ("gated_backward", lambda **k: jb.gated_backward(**k), dict(X=x, Wg=w, Wu=w2, dY=dy, pre=pre)),
        ("quant_rows_i8", lambda **k: jb.quant_rows_i8(**k), dict(X=x, out=xq, scale=sx)),
        ("codes_i8", lambda **k: jb.codes_i8(p, **k), dict(codes=codes, zeros=zeros, out=wq)),
        ("matmul_i8", lambda **k: jb.matmul_i8(**k), dict(Xq=xq, sx=sx, Wq=wq, sw=sw)),
        ("linear_i8", lambda **k: jb.linear_i8(**k), dict(X=x, Wq=wq, sw=sw)),
        ("token_logprobs", lambda **k: jb.token_logprobs(**k), dict(logits=x, targets=t)),
        ("token_logprobs_backward", lambda **k: jb.token_logprobs_backward(forward=r, **k),
         dict(logits=x, targets=t, d_logprob=g, out=x)),
    ]


NAMES = [c[0] for c in _calls()]


@pytest.mark.parametrize("name", NAMES)
def test_tensors_off_the_current_gpu_are_refused(name, monkeypatch):
    # kernels run on the current device: a tensor of another would be read from there, unordered
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0)
    call, tensors = next(c[1:] for c in _calls() if c[0] == name)
    with pytest.raises(ValueError, match="cuda:1.*cuda:0 is the current"):
        call(**{n: _placed(1, *t.shape, dtype=t.dtype) for n, t in tensors.items()})
    for moved, t in list(tensors.items())[1:]:
        with pytest.raises(ValueError, match=f"{moved} must be on cuda:0"):
            call(**{**tensors, moved: _placed(1, *t.shape, dtype=t.dtype)})


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


@pytest.mark.parametrize("name,shape,dtype", [("codes", (7, 64), torch.uint8),
                                              ("zeros", (7, 1), torch.int32),
                                              ("zeros", (8, 2), torch.int32),
                                              ("out", (8, 63), torch.int8)])
def test_codes_of_another_size_are_refused(name, shape, dtype, monkeypatch):
    # the kernel's grid comes from the parameters: a smaller array would be overrun
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0)
    call, tensors = next(c[1:] for c in _calls() if c[0] == "codes_i8")
    with pytest.raises(ValueError, match="rows, cols"):
        call(**{**tensors, name: _placed(0, *shape, dtype=dtype)})
