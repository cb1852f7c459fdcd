"""Refusals of the vocabulary operators: answered by the host checks, with no CUDA call made."""
import ctypes

import pytest
import torch


@pytest.fixture(scope="module")
def sats():
    from paper_2607_08991_gb300 import build, sats as s
    build.build_library()
    return s


F = ctypes.c_float
ODD = 0x1001   # never dereferenced: the call is refused


def _top(s, z=0x1000, ld=8, T=2, V=8, K=3, v=0x2000, i=0x3000, f32=False):
    return (s.lib().sats_top_logits_f32 if f32 else s.lib().sats_top_logits)(z, ld, T, V, K, v, i, None)


def test_top_logits(sats):
    s = sats
    assert _top(s, z=None) == s.EINVAL and _top(s, v=None) == s.EINVAL and _top(s, i=None) == s.EINVAL
    assert _top(s, ld=7) == s.EINVAL and _top(s, T=-1) == s.EINVAL and _top(s, V=0, ld=0) == s.EINVAL
    assert _top(s, K=0) == s.EINVAL and _top(s, K=9) == s.EINVAL and _top(s, z=ODD) == s.EINVAL
    assert _top(s, z=0x1002, f32=True) == s.EINVAL
    assert _top(s, V=2000, ld=2000, K=1025) == s.ESHAPE
    assert _top(s, V=2**31 - 64, ld=2**31 - 64) == s.ESHAPE and _top(s, T=2**28) == s.ESHAPE
    assert _top(s, ld=2**40 + 1) == s.ESHAPE
    assert _top(s, T=0) == s.OK and _top(s, T=0, z=None, v=None, i=None) == s.OK


def _loss(s, z=0x1000, ld=8, T=2, V=8, idx=0x2000, val=0x3000, K=2, labels=0x4000, tau=1.0, alpha=0.5, loss=0x5000,
          lse=None, f32=False):
    fn = s.lib().sats_distill_loss_f32 if f32 else s.lib().sats_distill_loss
    return fn(z, ld, T, V, idx, val, K, labels, tau, alpha, loss, lse, None, None)


def _grad(s, z=0x100000, ld=8, T=2, V=8, idx=0x2000, val=0x3000, K=2, labels=0x4000, tau=1.0, alpha=0.5, lse=0x5000,
          d=0x200000, ld_d=8, f32=False):
    fn = s.lib().sats_distill_grad_f32 if f32 else s.lib().sats_distill_grad
    return fn(z, ld, T, V, idx, val, K, labels, tau, alpha, lse, None, d, ld_d, None, None)


def _both(s, z=0x100000, ld=8, T=2, V=8, idx=0x2000, val=0x3000, K=2, labels=0x4000, tau=1.0, alpha=0.5, loss=0x5000,
          d=0x200000, ld_d=8, f32=False):
    fn = s.lib().sats_distill_loss_grad_f32 if f32 else s.lib().sats_distill_loss_grad
    return fn(z, ld, T, V, idx, val, K, labels, tau, alpha, None, loss, d, ld_d, None, None)


def test_distill_tau(sats):
    for call in (_loss, _grad, _both):
        for tau in (2.0**-10 * (1 - 2.0**-24), 2.0**10 * (1 + 2.0**-23), 1e-45, 3e38):
            assert call(sats, tau=tau) == sats.EINVAL
        for tau in (2.0**-10, 2.0**10):
            assert call(sats, tau=tau, T=0) == sats.OK


def test_distill(sats):
    s = sats
    for call in (_loss, _grad, _both):
        assert call(s, z=None) == s.EINVAL and call(s, z=ODD) == s.EINVAL and call(s, z=0x1002, f32=True) == s.EINVAL
        assert call(s, ld=7) == s.EINVAL and call(s, T=-1) == s.EINVAL and call(s, V=0) == s.EINVAL
        assert call(s, K=-1) == s.EINVAL and call(s, K=1025) == s.ESHAPE
        assert call(s, idx=None) == s.EINVAL and call(s, val=None) == s.EINVAL
        for tau in (0.0, -1.0, float("inf"), float("nan")):
            assert call(s, tau=tau) == s.EINVAL
        for alpha in (-0.1, 1.1, float("nan")):
            assert call(s, alpha=alpha) == s.EINVAL
        # neither of the two terms
        assert call(s, K=0, idx=None, val=None, labels=None) == s.EINVAL
        assert call(s, K=0, idx=None, val=None, alpha=1.0) == s.EINVAL
        assert call(s, labels=None, alpha=0.0) == s.EINVAL
        assert call(s, T=0) == s.OK
        assert call(s, T=2**28) == s.ESHAPE
    assert _loss(s, loss=None) == s.EINVAL and _both(s, loss=None) == s.EINVAL
    for call in (_grad, _both):
        assert call(s, d=None) == s.EINVAL and call(s, ld_d=7) == s.EINVAL and call(s, d=0x200001) == s.EINVAL
        assert call(s, d=0x200002, f32=True) == s.EINVAL
        # partly over the logits, from either side, and the same start with other rows
        assert call(s, d=0x100000 + 16) == s.EINVAL and call(s, d=0x100000 - 16) == s.EINVAL
        assert call(s, d=0x100000, ld_d=9) == s.EINVAL
    assert _grad(s, lse=None) == s.EINVAL


def _sample(s, z=0x1000, ld=8, B=2, V=8, u=0x2000, ids=0x3000, f32=False):
    fn = s.lib().sats_sample_f32 if f32 else s.lib().sats_sample
    return fn(z, ld, B, V, None, None, None, None, u, ids, None, None, None, None)


def test_sample(sats):
    s = sats
    assert _sample(s, z=None) == s.EINVAL and _sample(s, u=None) == s.EINVAL and _sample(s, ids=None) == s.EINVAL
    assert _sample(s, ld=7) == s.EINVAL and _sample(s, B=-1) == s.EINVAL and _sample(s, V=0, ld=0) == s.EINVAL
    assert _sample(s, z=ODD) == s.EINVAL and _sample(s, z=0x1002, f32=True) == s.EINVAL
    assert _sample(s, B=2**28) == s.ESHAPE and _sample(s, V=2**31 - 1, ld=2**31 - 1) == s.ESHAPE
    assert _sample(s, B=0) == s.OK


def test_binding_refuses_host_tensors(sats):
    z = torch.zeros(2, 8)
    with pytest.raises(ValueError):
        sats.top_logits(z, torch.zeros(2, 2), torch.zeros(2, 2, dtype=torch.int32))
    with pytest.raises(ValueError):
        sats.sample(z, torch.zeros(2), torch.zeros(2, dtype=torch.int32))
    with pytest.raises(ValueError):
        sats.distill_loss(z, None, None, torch.zeros(2, dtype=torch.int32), 1.0, 0.0, torch.zeros(2))
