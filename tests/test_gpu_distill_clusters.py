"""The one-pass distillation where clusters of several CTAs go from row to row: the sums' exchange in its two buffers, the
next row's granules that arrive while this one is stored, and ignored rows, rows without entries and rows with repeated ones
in between, against the 64-bit definition and bit for bit between runs.

228 clusters of two CTAs at most fit on 152 SMs (three CTAs to an SM), 114 of four, 57 of eight.  Tolerances as in
test_gpu_distill.py.
"""
import numpy as np
import pytest
import torch

from tests.test_gpu_distill import case, check, sats, to_dev   # noqa: F401 (sats: the fixture)
from tests.test_gpu_top_logits import rows

pytestmark = pytest.mark.gpu


def mixed(T, V, K, seed):
    z, idx, val, y, up = case(T, V, K, seed, odd=True)
    g = np.random.default_rng([seed, 1])
    y[g.random(T) < 0.3] = -1
    idx[g.random(T) < 0.2] = -1
    rep = g.random(T) < 0.3
    idx[rep, K - 1] = idx[rep, 0]
    up[g.random(T) < 0.1] = 0.0
    y[-3:] = idx[-3:, 0] = 11                     # (live rows at the end)
    return z, idx, val, y, up


@pytest.mark.parametrize("dtype,V,T", [(torch.bfloat16, 50021, 700), (torch.float32, 50021, 300), (torch.bfloat16, 40009, 300),
                                       (torch.bfloat16, 150001, 200), (torch.float32, 150001, 120), (torch.bfloat16, 320001, 90)])
@pytest.mark.parametrize("tau,alpha,d_pad", [(1.0, 0.6, 0), (2.0, 0.5, 1)])
def test_rows_after_rows(sats, dtype, V, T, tau, alpha, d_pad):   # noqa: F811
    z, idx, val, y, up = mixed(T, V, 17, 91)
    same = 16 // torch.empty(0, dtype=dtype).element_size()
    pad = same - V % same                          # the logits' rows all on one boundary; the gradient's on it too, or not
    zd = rows(z, dtype, pad=pad)
    check(sats, zd, idx, val, y, up, tau, alpha, d_pad=pad + d_pad)
    a = [to_dev(x) for x in (idx, val, y)]
    dg = to_dev(up)
    out = []
    for place in ("apart", "apart", "in place"):
        loss = torch.full((T,), 9.0, device="cuda")
        own = rows(z, dtype, pad=pad)
        d = own if place == "in place" else rows(np.zeros_like(z), dtype, pad=pad + d_pad)
        sats.distill_loss_grad(own, *a, tau, alpha, loss, d, g=dg)
        out.append((loss, d))
    assert torch.equal(out[0][0], out[1][0]) and torch.equal(out[0][1], out[1][1])
    if d_pad == 0:                                 # (on other boundaries the sums are added in another order)
        assert torch.equal(out[0][0], out[2][0]) and torch.equal(out[0][1], out[2][1])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_rows_after_rows_on_moving_boundaries(sats, dtype):   # noqa: F811
    # every row on another boundary than the one before it, so that the next row's granules are others than this one's
    V, T = 90011, 250
    z, idx, val, y, up = mixed(T, V, 300, 92)
    check(sats, rows(z, dtype, pad=1, off=1), idx, val, y, up, 1.5, 0.3, d_pad=1, d_off=1)
    check(sats, rows(z, dtype), idx, val, y, up, 1.0, 1.0, d_pad=2, d_off=3)
