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


class _Tensor:
    """What the binding asks of a tensor, on a device of one's choice."""

    def __init__(self, shape, dtype, device):
        self.shape, self.dtype, self.device = shape, dtype, device

    def get_device(self):
        return self.device

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return 0x1000


def test_workspace_on_another_device(sats, monkeypatch):
    import torch
    monkeypatch.setattr(sats, "_rows", lambda t, name: (0x2000, 8, 1, 8, True, 0))
    monkeypatch.setattr(sats, "_stream", lambda s: None)
    w, ws = sats.Q4.__new__(sats.Q4), sats.Q4Workspace.__new__(sats.Q4Workspace)
    w.handle, w.K, w.N, w.device = None, 64, 8, 0
    ws.nbytes, ws.buf = 1 << 30, _Tensor((1 << 30,), torch.uint8, 1)
    x = _Tensor((1, 64), torch.float32, 0)
    with pytest.raises(ValueError):
        sats.q4_matmul(w, x, None, ws)
    ws.buf.device = 0
    with pytest.raises(sats.SatsError):      # (then the library refuses the empty handle)
        sats.q4_matmul(w, x, None, ws)


def test_parts_of_other_types(sats, monkeypatch):
    """fp16 scales have bf16's size, int32 values fp32's: not taken for them."""
    import torch
    monkeypatch.setattr(sats, "_ptr", lambda t, name, elem=None: 0x1000)
    monkeypatch.setattr(sats, "_current", lambda p, t: p)
    codes, scales = torch.zeros(32, 8, dtype=torch.uint8), torch.zeros(2, 8, dtype=torch.bfloat16)
    assert sats._q4_parts(codes, scales, 32) == (0x1000, 0x1000, 64, 8)
    assert sats._q4_parts(codes.to(torch.int8), scales.view(torch.int16), 32) == (0x1000, 0x1000, 64, 8)
    for c, s in ((codes, scales.half()), (codes.bool(), scales), (codes, scales.view(torch.int16).to(torch.uint16))):
        with pytest.raises(ValueError):
            sats._q4_parts(c, s, 32)
    with pytest.raises(ValueError):
        sats.q4_dequantize(codes, scales, 32, torch.zeros(64, 8, dtype=torch.int32))
