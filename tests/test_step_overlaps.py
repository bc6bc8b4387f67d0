"""What the norm's entry points refuse of arrays that overlap, and what the backward passes' workspaces
take (CPU only: every call fails its checks)."""

import ctypes
import os
import re

import pytest
import torch

from paper_2609_38599_amd import binding as jb

# (with a GPU a check that is lost would let a kernel loose on host memory)
pytestmark = pytest.mark.skipif(torch.cuda.is_available(), reason="made-up addresses stand in for a GPU's")

MB = 1 << 20
T, C = 4, 64
ROWS = T * C * 2     # bytes of bf16 rows
LATE = ROWS - 2      # the last value


@pytest.fixture(scope="module")
def lib():
    return jb.load_library()


def _at(p):
    return None if p is None else ctypes.c_void_p(int(p))


def _norm(lib, x=1 * MB, res=None, g=3 * MB, h=None, y=5 * MB):
    return lib.jarq_rms_norm(2, 2, T, C, _at(x), _at(res), _at(g), ctypes.c_float(1e-6), _at(h), _at(y), None)


def _norm_i8(lib, x=1 * MB, res=None, g=3 * MB, h=None, q=5 * MB, s=6 * MB):
    return lib.jarq_rms_norm_i8(2, 2, T, C, _at(x), _at(res), _at(g), ctypes.c_float(1e-6), _at(h), _at(q),
                                _at(s), None)


def _backward(lib, h=1 * MB, g=2 * MB, dy=3 * MB, dh=4 * MB, dx=5 * MB, dg=6 * MB, ws=7 * MB, cols=C):
    n = int(lib.jarq_rms_norm_workspace_bytes(T, cols))
    return lib.jarq_rms_norm_backward(2, 2, T, cols, _at(h), _at(g), _at(dy), _at(dh), ctypes.c_float(1e-6), _at(dx),
                                      _at(dg), _at(ws), n, None)


def test_norm_refuses_outputs_that_overlap(lib):
    both = dict(x=1 * MB, res=2 * MB, h=4 * MB, y=5 * MB)
    for k in (dict(y=1 * MB + 2), dict(y=1 * MB + LATE), dict(y=1 * MB - LATE), dict(y=3 * MB),
              dict(y=3 * MB + C * 2 - 2), dict(y=3 * MB - LATE),
              dict(both, h=1 * MB + 2), dict(both, h=2 * MB - 2), dict(both, h=3 * MB), dict(both, h=5 * MB + 16),
              dict(both, y=2 * MB + 2), dict(both, y=4 * MB + LATE), dict(both, y=4 * MB),
              dict(both, h=2 * MB, y=2 * MB)):
        assert _norm(lib, **k) == jb.JARQ_EINVAL, k
    both = dict(x=1 * MB, res=2 * MB, h=4 * MB)
    for k in (dict(q=1 * MB), dict(q=1 * MB + 16), dict(q=3 * MB), dict(s=1 * MB + LATE - 2), dict(s=3 * MB),
              dict(s=5 * MB + T * C - 4), dict(q=6 * MB), dict(both, q=2 * MB), dict(both, q=4 * MB),
              dict(both, h=1 * MB + 2), dict(both, h=3 * MB), dict(both, h=5 * MB), dict(both, s=4 * MB)):
        assert _norm_i8(lib, **k) == jb.JARQ_EINVAL, k


def test_norm_gradient_refuses_arrays_that_overlap(lib):
    for cols in (C, 20000):
        rows = T * cols * 2
        for k in (dict(dx=1 * MB), dict(dx=1 * MB + 2), dict(dx=2 * MB), dict(dx=3 * MB + 2), dict(dx=3 * MB - rows + 2),
                  dict(dx=4 * MB + rows - 2), dict(dg=1 * MB + 2), dict(dg=2 * MB), dict(dg=3 * MB), dict(dg=4 * MB),
                  dict(dg=5 * MB + rows - 2), dict(ws=1 * MB), dict(ws=2 * MB), dict(ws=3 * MB), dict(ws=4 * MB),
                  dict(ws=5 * MB), dict(ws=6 * MB)):
            assert _backward(lib, cols=cols, **k) == jb.JARQ_EINVAL, (cols, k)


def test_workspace_of_the_log_probabilities_gradient_is_what_the_header_says(lib):
    with open(os.path.join(os.path.dirname(jb.LIB_PATH), "..", "include", "jarq.h")) as f:
        said = int(re.search(r"tokens (\d+) MiB at most", f.read()).group(1)) * MB
    most = 0
    for t in (1, 5, 300, 511, 1000, 4095, 4096, 4097, 10000, 65536, 100003, 131071, 131072):
        for v in (1, 1000, 8191, 8192, 32001, 128000, 1 << 20, 1 << 22):
            for d in (8, 1024, 4096):
                n = int(lib.jarq_linear_logprobs_backward_workspace_bytes(t, d, v))
                assert 256 <= n <= said + 32 * 4 * t * d + 1024, (t, v, d)
            # (narrow rows: their sums are 4 MiB a share)
            n = int(lib.jarq_linear_logprobs_backward_workspace_bytes(t, 8, v))
            most = max(most, n)
            assert n - 4 * t * 8 <= said + 512
    assert most > said - 8 * MB
