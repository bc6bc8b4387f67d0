"""What the entry points of the operators that run, train and evaluate refined layers refuse,
beside test_blocks_oracle.py (CPU only: every call fails its checks)."""

import ctypes

import pytest

from paper_2609_38599_amd import binding as jb

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
