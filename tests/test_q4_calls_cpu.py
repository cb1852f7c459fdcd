"""Calls of the 4-bit product that are refused before anything is launched; no GPU."""
import ctypes

import pytest


@pytest.fixture(scope="module")
def sats():
    from paper_2607_08991_gb300 import build, sats as s
    build.build_library()
    return s


class Handle(ctypes.Structure):
    """As sats_q4 of csrc/q4.cu; what it points to is never looked at, the calls being refused."""
    _fields_ = [("K", ctypes.c_int), ("N", ctypes.c_int), ("G", ctypes.c_int), ("device", ctypes.c_int),
                ("blk", ctypes.c_void_p), ("col_exp", ctypes.c_void_p)]


WS = 0x40000000


def _matmul(s, x, B, y, ld_y, K=64, N=64, f32=True, y_f32=1, ws=WS):
    h = Handle(K, N, 32, 0, None, None)
    n = s.lib().sats_q4_workspace_bytes(K, N, B)
    fn = s.lib().sats_q4_matmul_f32 if f32 else s.lib().sats_q4_matmul
    return fn(ctypes.byref(h), x, B, y, ld_y, y_f32, ws, n, None)


def test_results_over_activations(sats):
    """CTAs write results while others still read activations."""
    s = sats
    x = 0x100000
    assert _matmul(s, x, 4, x, 64) == s.EINVAL                                       # y is x
    assert _matmul(s, x, 4, x, 64, f32=False, y_f32=0) == s.EINVAL
    assert _matmul(s, x, 1, x, 64) == s.EINVAL
    assert _matmul(s, x, 4, x + 4 * 4 * 64 - 4, 64) == s.EINVAL                      # y begins in x's last value
    assert _matmul(s, x, 4, x - (3 * 100 + 64) * 4 + 4, 100) == s.EINVAL             # x begins in y's last value
    assert _matmul(s, x, 1, x + 4 * 63, 64) == s.EINVAL
    assert _matmul(s, x, 4, x - 4 * 80, 100) == s.EINVAL                             # x lies between rows of y, and goes on over them
    assert _matmul(s, x, 1, x - 2 * 64 + 2, 64, y_f32=0) == s.EINVAL
    # apart: not refused for that (without a GPU the call then ends otherwise, with one it must not be made)
    if not _gpu():
        for B, y, ld in ((4, x + 4 * 4 * 64, 64), (4, x - (3 * 100 + 64) * 4, 100), (2, x - 4 * 64, 64 + 2 * 64)):
            assert _matmul(s, x, B, y, ld) not in (s.OK, s.EINVAL)


def test_over_the_workspace(sats):
    s = sats
    n = s.lib().sats_q4_workspace_bytes(64, 64, 4)
    for off in (0, 256, n - 4):
        assert _matmul(s, WS + off, 4, 0x100000, 64) == s.EINVAL
        assert _matmul(s, 0x100000, 4, WS + off, 64) == s.EINVAL
    assert _matmul(s, WS - 4, 4, 0x100000, 64) == s.EINVAL


def _gpu():
    import torch
    return torch.cuda.is_available()
