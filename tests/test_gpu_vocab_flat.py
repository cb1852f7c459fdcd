"""Flat rows, which show a lost or doubled element: all weights are exactly 1, their sums are whole numbers below 2^24 and
exact in whatever order, and only the roundings at the end are left.  And bf16 given as bit patterns.

With S = V exactly: log2 V <= 20 is off by an ulp (2^-19, 2^-19.5 as a natural logarithm), the log-sum-exp rounded to half an
ulp, at most 2^-20: within LSE = 2^-18 of ln V.  A granule more or less changes ln V by 4 / V in fp32 and 8 / V in bf16, at
least 2^-16.9 here.  The one-pass gradient is 1 / V but for four roundings of 2^-24; one element more or less changes it by 1 / V
of itself, at least 2^-19.
"""
import numpy as np
import pytest
import torch

from tests.test_gpu_distill import sats   # noqa: F401 (the fixture)

pytestmark = pytest.mark.gpu
LSE = 2.0 ** -18


@pytest.mark.parametrize("dtype,V", [(torch.float32, 1003), (torch.float32, 50021), (torch.float32, 128256), (torch.float32, 500003),
                                     (torch.bfloat16, 4097), (torch.bfloat16, 50021), (torch.bfloat16, 151936),
                                     (torch.bfloat16, 900001)])
@pytest.mark.parametrize("T", [1, 40, 160, 330])
@pytest.mark.parametrize("tau,alpha", [(1.0, 0.0), (2.0, 0.5)])
def test_flat_rows(sats, dtype, V, T, tau, alpha):   # noqa: F811
    if T * V > 60_000_000:
        T = 60_000_000 // V
    K = 4                                            # shares of exactly 1/4
    g = np.random.default_rng([101, V, T])
    pad = int(g.integers(0, 8))
    z = torch.full((T, V + pad), float("nan"), dtype=dtype, device="cuda")[:, :V]
    z.fill_(-1.75)
    y = torch.from_numpy(g.integers(0, V, T).astype(np.int32)).cuda()
    idx = torch.from_numpy(np.stack([g.choice(V, K, replace=False) for _ in range(T)]).astype(np.int32)).cuda()
    val = torch.full((T, K), 3.0, device="cuda")
    e = (idx, val) if alpha > 0 else (None, None)
    loss, loss2, lse = torch.zeros(T, device="cuda"), torch.zeros(T, device="cuda"), torch.zeros(T, 2, device="cuda")
    d, d2 = torch.zeros_like(z), torch.zeros_like(z)
    sats.distill_loss(z, *e, y, tau, alpha, loss, lse=lse)
    sats.distill_grad(z, *e, y, tau, alpha, lse, d)
    sats.distill_loss_grad(z, *e, y, tau, alpha, loss2, d2)
    want = np.array([-1.75 / tau, -1.75]) + np.log(V)
    assert np.abs(lse.double().cpu().numpy() - want).max() <= LSE
    # CE = ln V; KD = tau^2 (ln V - ln K); and a rounding to fp32 of each and of their sum
    ce, kd = np.log(V), tau * tau * (np.log(V) - np.log(K))
    right = (1 - alpha) * ce + alpha * kd
    tol = ((1 - alpha) + 2 * alpha * tau * tau) * LSE + 2.0 ** -22 * right
    for got in (loss, loss2):
        assert np.abs(got.double().cpu().numpy() - right).max() <= tol
    p = (1 - alpha + alpha * tau) / V
    own = torch.full((T, V), p, dtype=torch.float64, device="cuda")
    rows_at = torch.arange(T, device="cuda")
    own[rows_at, y.long()] -= 1 - alpha
    if alpha > 0:
        own.scatter_add_(1, idx.long(), torch.full((T, K), -alpha * tau / K, dtype=torch.float64, device="cuda"))
    for got, rel in ((d, LSE), (d2, 2.0 ** -22)):
        # (the places of targets: the difference rounded once more, of terms of at most 1)
        lim = rel * p + (2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -23) * own.abs()
        assert ((got.double() - own).abs() <= lim).all()


def test_bit_patterns_of_bf16(sats):   # noqa: F811
    T, V, K = 9, 5003, 20
    g = torch.Generator().manual_seed(102)
    z = (torch.randn(T, V + 3, generator=g) * 2.5).bfloat16().cuda()[:, 1:V + 1]
    bits = z.view(torch.int16)
    dev = lambda t, dt: t.to(dt).cuda()
    y = dev(torch.randint(-1, V, (T,), generator=g), torch.int32)
    u = dev(torch.rand(T, generator=g), torch.float32)
    f = lambda *s: torch.full(s, 7.0, device="cuda")
    i = lambda *s: torch.full(s, 7, dtype=torch.int32, device="cuda")
    out = []
    for x in (z, bits):
        values, idx, ids, loss, loss2, lse = f(T, K), i(T, K), i(T), f(T), f(T), f(T, 2)
        d, d2 = (torch.full((T, V), 7, dtype=x.dtype, device="cuda") for _ in range(2))
        sats.top_logits(x, values, idx)
        sats.distill_loss(x, idx, values, y, 2.0, 0.5, loss, lse=lse)
        sats.distill_grad(x, idx, values, y, 2.0, 0.5, lse, d)
        sats.distill_loss_grad(x, idx, values, y, 2.0, 0.5, loss2, d2)
        sats.sample(x, u, ids)
        own = x.clone()                              # in place
        sats.distill_loss_grad(own, idx, values, y, 2.0, 0.5, f(T), own)
        out.append([values, idx, ids, loss, loss2, lse] + [t.view(torch.bfloat16) for t in (d, d2, own)])
    for a, b in zip(*out):
        assert torch.equal(a, b) and not (a == 7).all()
    d = torch.zeros_like(z)                          # patterns in, bf16 out
    sats.distill_loss_grad(bits, out[0][1], out[0][0], y, 2.0, 0.5, f(T), d)
    assert torch.equal(d, out[0][7])
    with pytest.raises(ValueError):
        sats.distill_loss_grad(bits, out[0][1], out[0][0], y, 2.0, 0.5, f(T), d.float())
