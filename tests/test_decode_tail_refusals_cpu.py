"""Refusals of the adjusted logits and the 4-bit weights: answered by the host checks, with no CUDA call made."""
import ctypes

import pytest
import torch


@pytest.fixture(scope="module")
def sats():
    from paper_2607_08991_gb300 import build, sats as s
    build.build_library()
    return s


def _adjust(s, z=0x100000, ld=64, B=2, V=64, hist=0x2000, ld_hist=8, L=8, bias=(None, None), M=0, mask=None, ld_mask=0,
            n_masks=0, mask_row=None, out=0x200000, ld_out=64, f32=False, hist_len=None, n_prompt=None):
    fn = s.lib().sats_adjust_logits_f32 if f32 else s.lib().sats_adjust_logits
    return fn(z, ld, B, V, hist, ld_hist, L, hist_len, n_prompt, None, None, None, *bias, M, mask, ld_mask, n_masks,
              mask_row, out, ld_out, None, None)


def _grad(s, z=0x100000, ld=64, B=2, V=64, hist=0x2000, ld_hist=8, L=8, mask=None, ld_mask=0, n_masks=0, mask_row=None,
          dout=0x300000, ld_dout=64, out=0x200000, ld_out=64, f32=False, hist_len=None):
    fn = s.lib().sats_adjust_logits_grad_f32 if f32 else s.lib().sats_adjust_logits_grad
    return fn(z, ld, B, V, hist, ld_hist, L, hist_len, None, mask, ld_mask, n_masks, mask_row, dout, ld_dout, out, ld_out,
              None, None)


def test_adjust(sats):
    s = sats
    for call in (_adjust, _grad):
        assert call(s, z=None) == s.EINVAL and call(s, out=None) == s.EINVAL
        assert call(s, z=0x100001) == s.EINVAL and call(s, z=0x100002, f32=True) == s.EINVAL
        assert call(s, out=0x200001) == s.EINVAL and call(s, out=0x200002, f32=True) == s.EINVAL
        assert call(s, ld=63) == s.EINVAL and call(s, ld_out=63) == s.EINVAL and call(s, B=-1) == s.EINVAL
        assert call(s, V=0) == s.EINVAL and call(s, L=-1) == s.EINVAL and call(s, ld_hist=-1) == s.EINVAL
        assert call(s, hist=None) == s.EINVAL and call(s, hist=None, L=0, hist_len=0x3000, B=0) == s.OK
        assert call(s, B=2**28) == s.ESHAPE and call(s, L=2**30) == s.ESHAPE
        assert call(s, V=2**31 - 64, ld=2**31, ld_out=2**31) == s.ESHAPE and call(s, ld=2**40 + 1) == s.ESHAPE
        # masks: too narrow, too few, rows without masks
        assert call(s, mask=0x4000, ld_mask=1, n_masks=2) == s.EINVAL
        assert call(s, mask=0x4000, ld_mask=2, n_masks=1) == s.EINVAL
        assert call(s, mask_row=0x4000) == s.EINVAL
        # the outputs partly over the logits, from either side, and the same start with other rows
        assert call(s, out=0x100000 + 16) == s.EINVAL and call(s, out=0x100000 - 16) == s.EINVAL
        assert call(s, out=0x100000, ld_out=65) == s.EINVAL
        assert call(s, B=0) == s.OK and call(s, B=0, z=None, out=None) == s.OK
    assert _adjust(s, M=1) == s.EINVAL and _adjust(s, M=-1) == s.EINVAL
    assert _adjust(s, M=1, bias=(0x5000, None)) == s.EINVAL and _adjust(s, M=1025, bias=(0x5000, 0x6000)) == s.ESHAPE
    assert _grad(s, dout=None) == s.EINVAL and _grad(s, ld_dout=63) == s.EINVAL and _grad(s, dout=0x300001) == s.EINVAL
    assert _grad(s, out=0x100000) == s.EINVAL                # over the logits, which the last step reads
    assert _grad(s, out=0x300000 + 16) == s.EINVAL and _grad(s, out=0x300000, ld_out=65) == s.EINVAL


def test_adjust_pointers_of_words(sats):
    """Ids, settings, biases and masks are read in words and vectors of them: none may begin inside a word."""
    s = sats
    for f32 in (False, True):
        for call in (_adjust, _grad):
            assert call(s, hist=0x2002, f32=f32) == s.EINVAL and call(s, hist_len=0x3001, f32=f32) == s.EINVAL
            assert call(s, mask=0x4002, ld_mask=2, n_masks=2, f32=f32) == s.EINVAL
            assert call(s, mask=0x4000, ld_mask=2, n_masks=2, mask_row=0x5001, f32=f32) == s.EINVAL
        assert _adjust(s, n_prompt=0x3002, f32=f32) == s.EINVAL
        assert _adjust(s, M=1, bias=(0x5002, 0x6000), f32=f32) == s.EINVAL
        assert _adjust(s, M=1, bias=(0x5000, 0x6001), f32=f32) == s.EINVAL


def test_q4_shapes(sats):
    L, s = sats.lib(), sats
    out = ctypes.c_void_p()
    for K, N, G in ((7, 8, 32), (12, 8, 32), (0, 8, 32), (65544, 8, 32), (64, 0, 32), (64, 2**24 + 1, 32), (64, 8, 16),
                    (64, 8, 0), (64, 8, 256)):
        assert L.sats_q4_create(0x1000, 0x2000, K, N, G, None, ctypes.byref(out)) == s.ESHAPE
        assert L.sats_q4_quantize(0x1000, 2**25, K, N, G, 0x2000, 0x3000, None) == s.ESHAPE
        assert L.sats_q4_dequantize(0x1000, 0x2000, K, N, G, 0x3000, None) == s.ESHAPE
    assert L.sats_q4_workspace_bytes(12, 8, 1) == 0 and L.sats_q4_workspace_bytes(64, 0, 1) == 0
    assert L.sats_q4_workspace_bytes(64, 8, -1) == 0 and L.sats_q4_workspace_bytes(64, 8, 2**20 + 1) == 0
    assert 0 < L.sats_q4_workspace_bytes(64, 8, 0) <= L.sats_q4_workspace_bytes(64, 8, 1)
    # a larger batch never needs less
    sizes = [L.sats_q4_workspace_bytes(4096, 14336, b) for b in (1, 8, 9, 16, 17, 32, 33, 64, 65, 128, 129, 2048)]
    assert sizes == sorted(sizes)


def test_q4_pointers(sats):
    L, s = sats.lib(), sats
    out = ctypes.c_void_p()
    E = s.EINVAL
    assert L.sats_q4_create(None, 0x2000, 64, 8, 32, None, ctypes.byref(out)) == E
    assert L.sats_q4_create(0x1000, None, 64, 8, 32, None, ctypes.byref(out)) == E
    assert L.sats_q4_create(0x1000, 0x2001, 64, 8, 32, None, ctypes.byref(out)) == E
    assert L.sats_q4_create(0x1000, 0x2000, 64, 8, 32, None, None) == E
    assert L.sats_q4_destroy(None) == E and L.sats_q4_shape(None, None, None, None) == E
    assert L.sats_q4_quantize(None, 8, 64, 8, 32, 0x2000, 0x3000, None) == E
    assert L.sats_q4_quantize(0x1001, 8, 64, 8, 32, 0x2000, 0x3000, None) == E
    assert L.sats_q4_quantize(0x1000, 7, 64, 8, 32, 0x2000, 0x3000, None) == E
    assert L.sats_q4_quantize(0x1000, 8, 64, 8, 32, None, 0x3000, None) == E
    assert L.sats_q4_quantize(0x1000, 8, 64, 8, 32, 0x2000, 0x3001, None) == E
    assert L.sats_q4_dequantize(0x1000, 0x2000, 64, 8, 32, None, None) == E
    assert L.sats_q4_dequantize(0x1000, 0x2000, 64, 8, 32, 0x3002, None) == E
    for fn in (L.sats_q4_matmul, L.sats_q4_matmul_f32):
        assert fn(None, 0x1000, 1, 0x2000, 8, 1, 0x100, 1 << 40, None) == E


def test_binding_refuses_host_tensors(sats):
    z = torch.zeros(2, 64)
    with pytest.raises(ValueError):
        sats.adjust_logits(z, z)
    with pytest.raises(ValueError):
        sats.adjust_logits_grad(z, z, z)
    with pytest.raises(ValueError):
        sats.Q4(torch.zeros(32, 8, dtype=torch.uint8), torch.zeros(2, 8, dtype=torch.bfloat16), 32)
    with pytest.raises(ValueError):
        sats.Q4(torch.zeros(32, 8, dtype=torch.uint8), torch.zeros(3, 8, dtype=torch.bfloat16), 32)
    with pytest.raises(ValueError):
        sats.q4_quantize(torch.zeros(64, 8, dtype=torch.bfloat16), torch.zeros(32, 8, dtype=torch.uint8),
                         torch.zeros(2, 8, dtype=torch.bfloat16), 32)
