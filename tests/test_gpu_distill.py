"""Distillation from a teacher's top logits against the 64-bit definition: loss, log-sum-exp and gradient, in one
pass and in two, at odd sizes and strides, with absent, repeated and masked entries and ignored rows.

Tolerances.  With R the largest |z - max z| log2(e) / tau that weighs anything (2^-R V is below a rounding of the sum
from R = 48 on, so R <= 48 counts), a weight 2^x carries the rounding of x (R 2^-24 absolute, of its factor log2(e) /
tau the same again) and 2 ulp of the exponential: relative  ln 2 * 2 R 2^-24 + 2^-22 <= 2^-17.5.  Sums over threads,
warps and CTAs add at most 2^-24 for each of their <= 400 sequential additions: <= 2^-15.3 at the longest row of a
thread, in practice a random walk; the bound used is DELTA = 2^-15 for a weight, a probability or a log-sum-exp (absolute).
Values are rounded to their type at the end, and fp32 outputs once or twice before: 2^-22 relative, bf16 2^-8.
"""
import numpy as np
import pytest
import torch

from oracle import vocab
from tests.test_gpu_top_logits import rows

pytestmark = pytest.mark.gpu
DELTA = 2.0 ** -15


@pytest.fixture(scope="module")
def sats():
    import __graft_entry__
    __graft_entry__.build()
    from paper_2607_08991_gb300 import sats as s
    return s


def case(T, V, K, seed, odd=False):
    """Logits, entries, values, labels, upstream gradients (numpy)."""
    g = np.random.default_rng([seed, T, V, K])
    z = g.normal(0, 2.2, (T, V))
    z[np.arange(T), g.integers(0, V, T)] += g.uniform(0, 14, T)
    idx = np.stack([g.permutation(V)[:K] if K <= V else g.integers(0, V, K) for _ in range(T)]).astype(np.int32) \
        if K else None
    val = g.normal(0, 3, (T, K)).astype(np.float32) if K else None
    y = g.integers(0, V, T).astype(np.int32)
    up = g.normal(0, 1, T).astype(np.float32)
    if K:
        y[::3] = idx[::3, 0]                       # the label among the entries
    if T > 2:
        y[1] = -1
        up[2] = 0.0
    if odd and K > 3:
        idx[0, 1] = idx[0, 0]                      # twice, and three times
        idx[-1, 2] = idx[-1, 3] = idx[-1, 0]
        idx[0, 2] = -1
        val[0, 3] = -np.inf                        # an entry of no weight
        z[0, idx[0, 3]] = -np.inf                  # on a masked logit
        if T > 4:
            idx[3] = -5                            # no entries at all
            val[4] = -np.inf
    return z.astype(np.float32), idx, val, y, up


def to_dev(a):
    return None if a is None else torch.from_numpy(np.ascontiguousarray(a)).cuda()


def run_all(sats, z, idx, val, y, up, tau, alpha, d_pad=0, d_off=0):
    """(loss, lse, gradient of the backward call, loss and gradient of the one-pass call); checks what lies around."""
    T, V = z.shape
    di, dv, dy, dg = to_dev(idx), to_dev(val), to_dev(y), to_dev(up)
    loss, lse = torch.full((T + 1,), 7.0, device="cuda"), torch.full((T + 1, 2), 7.0, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    sats.distill_loss(z, di, dv, dy, tau, alpha, loss[:T], lse=lse[:T], dev_status=status)
    out = []
    for one_pass in (False, True):
        buf = torch.full((T * (V + d_pad) + d_off + 64,), 7.0, dtype=z.dtype, device="cuda")
        d = buf[d_off:d_off + T * (V + d_pad)].view(T, V + d_pad)
        if one_pass:
            loss2 = torch.full((T,), 7.0, device="cuda")
            sats.distill_loss_grad(z, di, dv, dy, tau, alpha, loss2, d[:, :V], g=dg, dev_status=status)
        else:
            sats.distill_grad(z, di, dv, dy, tau, alpha, lse[:T], d[:, :V], g=dg, dev_status=status)
        torch.cuda.synchronize()
        assert (d[:, V:] == 7).all() and (buf[:d_off] == 7).all() and (buf[d_off + T * (V + d_pad):] == 7).all()
        out.append(d[:, :V].double().cpu().numpy())
    assert loss[T] == 7 and (lse[T] == 7).all()
    assert sats.get_status_word(status) == sats.OK
    f = lambda t: t.double().cpu().numpy()
    return f(loss[:T]), f(lse[:T]), out[0], f(loss2), out[1]


def close(got, want, abs_tol, rel):
    """Within the tolerance; where 64 bits give an infinity, the same one."""
    fin = np.isfinite(want)
    assert np.array_equal(got[~fin], want[~fin], equal_nan=True)
    with np.errstate(invalid="ignore"):
        err = np.abs(got - want)
    lim = abs_tol + rel * np.abs(want)
    bad = fin & ~(err <= lim)
    assert not bad.any(), (np.argwhere(bad)[:4], got[bad][:4], want[bad][:4])


def check(sats, z, idx, val, y, up, tau, alpha, **kw):
    bf16 = z.dtype == torch.bfloat16
    z64 = z.double().cpu().numpy()
    loss, lse, grad, loss2, grad2 = run_all(sats, z, idx, val, y, up, tau, alpha, **kw)
    val64 = None if val is None else val.astype(np.float64)
    rl, rs, rd = vocab.distill(z64, idx, val64, y, tau, alpha, np.ones(z.shape[0]) if up is None else up)
    # KD: a weighted mean of log ratios, each off by two DELTA (the entries' own softmax has the same errors)
    tol = alpha * tau * tau * 4 * DELTA + (1 - alpha) * 2 * DELTA
    close(loss, rl, tol, 2.0 ** -20)
    close(loss2, rl, tol, 2.0 ** -20)
    close(lse, rs, DELTA, 2.0 ** -22)
    # gradient: every probability and share within 2 DELTA of itself; both are at most what |d| + share is, and the
    # difference of the two may be small: absolute, by the row's upstream gradient and the share of its terms
    g = np.abs(np.ones(z.shape[0]) if up is None else up)[:, None].astype(np.float64)
    with np.errstate(all="ignore"):
        p = g * (alpha * tau * np.exp(z64 / tau - rs[:, :1]) + (1 - alpha) * np.exp(z64 - rs[:, 1:]))
    q = np.zeros_like(p)
    if idx is not None:
        for r in range(z.shape[0]):
            i, s = vocab.teacher_shares(z.shape[1], idx[r], val64[r], tau)
            np.add.at(q[r], i, g[r, 0] * alpha * tau * s)
    if y is not None:
        for r in range(z.shape[0]):
            if y[r] >= 0:
                q[r, y[r]] += g[r, 0] * (1 - alpha)
    lim = 4 * DELTA * (np.nan_to_num(p) + q) + (2.0 ** -8 if bf16 else 2.0 ** -22) * np.abs(rd) + 2.0 ** -126
    for got in (grad, grad2):
        bad = np.isfinite(rd) & ~(np.abs(got - rd) <= lim)
        assert not bad.any(), (np.argwhere(bad)[:4], got[bad][:4], rd[bad][:4], lim[bad][:4])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T,V,K", [(1, 1, 1), (1, 2, 0), (3, 7, 4), (6, 8, 8), (5, 9, 5), (6, 100, 40), (2, 1000, 1000),
                                   (5, 4099, 64), (6, 50001, 700), (7, 20011, 0)])
def test_sizes(sats, T, V, K, dtype):
    z, idx, val, y, up = case(T, V, K, 21, odd=True)
    for n, (tau, alpha) in enumerate([(1.0, 0.0), (2.0, 0.4), (1.0, 0.7), (0.6, 1.0)]):
        if K == 0 and alpha == 1.0:
            continue
        check(sats, rows(z, dtype, pad=n, off=n), idx, val, y, up, tau, alpha, d_pad=n // 2, d_off=(3 * n) % 4)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T", [1, 9, 330])
def test_vocabulary(sats, T, dtype):
    V = 128256 if T < 300 else 16001
    z, idx, val, y, up = case(T, V, 64, 22)
    check(sats, rows(z, dtype), idx, val, y, up, 2.0, 0.5)
    check(sats, rows(z, dtype, pad=1), idx, val, y, None, 1.0, 0.5, d_pad=2)


@pytest.mark.parametrize("dtype,V", [(torch.float32, 500003), (torch.bfloat16, 900001)])
def test_rows_larger_than_the_cluster_memory(sats, dtype, V):
    z, idx, val, y, up = case(2, V, 1024, 23)
    check(sats, rows(z, dtype, pad=3), idx, val, y, up, 1.5, 0.5, d_pad=2)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_extreme_temperatures(sats, dtype):
    z, idx, val, y, up = case(5, 3001, 9, 37)
    # (the logits and values scaled so that their quotients by tau are ordinary ones)
    for tau, size in ((2.0 ** -10, 2.0 ** -10), (2.0 ** 10, 2.0 ** 5)):
        check(sats, rows(z * np.float32(size), dtype), idx, val * np.float32(size), y, up, tau, 1.0)
        check(sats, rows(z * np.float32(size), dtype), idx, val * np.float32(size), y, up, tau, 0.5)


def test_large_offsets(sats):
    # rows so far apart that their offsets pass 32 bits, of the logits and of the gradient
    V, T, ld = 2003, 3, (1 << 31) + 5
    z, idx, val, y, up = case(T, V, 8, 33)
    buf, out = (torch.empty((T - 1) * ld + V, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    zd, d = (torch.as_strided(b, (T, V), (ld, 1)) for b in (buf, out))
    zd.copy_(torch.from_numpy(z))
    a = (zd, to_dev(idx), to_dev(val), to_dev(y), 2.0, 0.5)
    loss, lse = torch.zeros(T, device="cuda"), torch.zeros(T, 2, device="cuda")
    rl, _, rd = vocab.distill(zd.double().cpu().numpy(), idx, val.astype(np.float64), y, 2.0, 0.5, up)
    for one_pass in (False, True):
        out.zero_()
        if one_pass:
            sats.distill_loss_grad(*a, loss, d, g=to_dev(up))
        else:
            sats.distill_loss(*a, loss, lse=lse)
            sats.distill_grad(*a, lse, d, g=to_dev(up))
        close(loss.double().cpu().numpy(), rl, 12 * DELTA, 2.0 ** -20)
        close(d.double().cpu().numpy(), rd, 16 * DELTA * np.abs(up).max(), 2.0 ** -8)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_every_pair_of_boundaries(sats, dtype):
    # the logits' and the gradient's rows on all combinations of places within 16 bytes, rows of a few granules to many
    E = 4 if dtype == torch.float32 else 8
    for V in (E - 1, 3 * E + 1, 1000):
        z, idx, val, y, up = case(4, V, 3, 34)
        for a in range(E):
            for b in range(0, E, 1 if V < 100 else 3):
                check(sats, rows(z, dtype, pad=(a * 3) % E, off=a), idx, val, y, up, 1.5, 0.5, d_pad=(b * 5) % E, d_off=b)


def test_many_rows_of_one_cluster(sats):
    # clusters go from row to row: live, ignored, without entries, with repeated ones, in every order
    T, V, K = 2500, 500, 5
    g = np.random.default_rng(35)
    z, idx, val, y, up = case(T, V, K, 36)
    y[g.random(T) < 0.4] = -1
    idx[g.random(T) < 0.3] = -1
    rep = g.random(T) < 0.3
    idx[rep, 3] = idx[rep, 0]
    for dtype, pad in ((torch.float32, 0), (torch.bfloat16, 3)):
        check(sats, rows(z, dtype, pad=pad), idx, val, y, up, 2.0, 0.5, d_pad=1)
        check(sats, rows(z, dtype, pad=pad), idx, val, y, up, 1.0, 1.0, d_pad=pad)


def test_without_labels_and_without_entries(sats):
    z, idx, val, y, up = case(5, 3001, 16, 24)
    check(sats, rows(z, torch.float32), idx, val, None, up, 2.0, 0.25)
    check(sats, rows(z, torch.float32), idx, val, None, up, 2.0, 1.0)
    check(sats, rows(z, torch.bfloat16), None, None, y, up, 3.0, 0.25)


def test_masked_logits(sats):
    # most of the vocabulary -inf or the type's lowest value, a row with one place left, one with none
    z, idx, val, y, up = case(6, 5003, 12, 25)
    g = np.random.default_rng(26)
    z[g.random(z.shape) < 0.8] = -np.inf
    z[2, g.random(5003) < 0.5] = np.finfo(np.float32).min
    z[np.arange(6)[:, None], idx] = g.normal(0, 2, idx.shape)
    z[np.arange(6), np.maximum(y, 0)] = 1.0
    z[3] = -np.inf
    z[3, y[3]] = 2.5
    z[3, idx[3]] = 0.5
    for dtype in (torch.float32, torch.bfloat16):
        check(sats, rows(z, dtype, pad=1), idx, val, y, up, 1.3, 0.5)
    # an entry with a share on a masked logit: the loss is +inf, the gradient the formula's
    z[4, idx[4, 0]] = -np.inf
    y[5] = -1
    z[5] = np.nan                                  # an ignored row: not looked at
    check(sats, rows(z, torch.float32), idx, val, y, up, 1.3, 0.5)


def test_nan_and_inf_rows_give_nan(sats):
    z, idx, val, y, up = case(4, 2003, 8, 27)
    y[:] = 5
    z[0, 1000] = np.nan
    z[1, 7] = np.inf
    z[2] = -np.inf
    zd = rows(z, torch.float32)
    loss = torch.zeros(4, device="cuda")
    sats.distill_loss(zd, to_dev(idx), to_dev(val), to_dev(y), 1.0, 0.5, loss)
    assert torch.isnan(loss).tolist() == [True, True, True, False]


def test_bad_indices_and_labels(sats):
    z, idx, val, y, up = case(4, 501, 6, 28)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    zd = rows(z, torch.float32)
    idx_bad = idx.copy()
    idx_bad[0, 2], idx_bad[3, 5] = 501, 2**31 - 1
    y_bad = y.copy()
    y_bad[2] = 501
    y_ref = np.where(y_bad >= 501, -1, y_bad)
    rl, _, rd = vocab.distill(zd.double().cpu().numpy(), idx_bad, val.astype(np.float64), y_ref, 2.0, 0.5, up)
    loss, lse, d = torch.zeros(4, device="cuda"), torch.zeros(4, 2, device="cuda"), torch.zeros(4, 501, device="cuda")
    a = (zd, to_dev(idx_bad), to_dev(val), to_dev(y_bad), 2.0, 0.5)
    for call in range(3):
        if call == 0:
            sats.distill_loss(*a, loss, lse=lse, dev_status=status)
        elif call == 1:
            sats.distill_grad(*a, lse, d, g=to_dev(up), dev_status=status)
        else:
            sats.distill_loss_grad(*a, loss, d, g=to_dev(up), dev_status=status)
        assert sats.get_status_word(status) == sats.EDEVICE and sats.get_status_word(status) == sats.OK
        if call != 1:
            close(loss.double().cpu().numpy(), rl, 12 * DELTA, 2.0 ** -20)
        if call != 0:
            close(d.double().cpu().numpy(), rd, 16 * DELTA * np.abs(up).max(), 2.0 ** -20)
    sats.distill_loss(*a, loss)                     # without a status word: the same results
    close(loss.double().cpu().numpy(), rl, 12 * DELTA, 2.0 ** -20)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [1000, 60001])
def test_in_place(sats, V, dtype):
    z, idx, val, y, up = case(5, V, 30, 29, odd=True)
    di, dv, dy, dg = map(to_dev, (idx, val, y, up))
    zd = rows(z, dtype, pad=3)
    loss, lse, d = torch.zeros(5, device="cuda"), torch.zeros(5, 2, device="cuda"), torch.zeros(5, V, dtype=dtype, device="cuda")
    for tau, alpha, e in ((2.0, 0.5, (di, dv)), (1.0, 0.0, (None, None))):
        sats.distill_loss(zd, *e, dy, tau, alpha, loss, lse=lse)
        sats.distill_grad(zd, *e, dy, tau, alpha, lse, d, g=dg)
        own = rows(z, dtype, pad=3)
        sats.distill_grad(own, *e, dy, tau, alpha, lse, own, g=dg)
        assert torch.equal(own, d)
        sats.distill_loss_grad(zd, *e, dy, tau, alpha, loss, d, g=dg)
        own = rows(z, dtype, pad=3)
        loss2 = torch.zeros(5, device="cuda")
        sats.distill_loss_grad(own, *e, dy, tau, alpha, loss2, own, g=dg)
        # d's rows lie on other boundaries than the logits', and the row's weights are then added in another order: each
        # sum is within DELTA of the true one, so the two probabilities are within 2 DELTA of each other (relative, a
        # probability is at most 1 and g tau times it at most |g| tau), the losses within tau^2 alpha + 1 - alpha times it
        bound = 2 * DELTA * float(dg.abs().max()) * max(tau, 1.0) + (2.0 ** -7 if dtype == torch.bfloat16 else 2.0 ** -22) * d.abs()
        assert ((own.float() - d.float()).abs() <= bound).all()
        assert ((loss - loss2).abs() <= 2 * DELTA * (tau * tau * alpha + 1 - alpha) + 2.0 ** -22 * loss.abs()).all()
        same = torch.zeros(5, V + 3, dtype=dtype, device="cuda")[:, :V]   # on the same boundaries: the same sums
        sats.distill_loss_grad(zd, *e, dy, tau, alpha, loss, same, g=dg)
        assert torch.equal(own, same) and torch.equal(loss, loss2)


def test_gradient_is_the_difference_quotient_of_the_kernel_loss(sats):
    # along a random direction, h = 2^-8: the third derivative (a third moment of the direction, below 10) gives
    # h^2 / 6 of it, 3e-5; losses up to 16, each off by up to 2^-20 relative, give 2^-16 / h / 2 * 2 = 4e-3
    z, idx, val, y, up = case(40, 700, 9, 30)
    g = np.random.default_rng(31)
    v = g.normal(0, 1, z.shape).astype(np.float32)
    a = [to_dev(x) for x in (idx, val, y)]
    h = 2.0 ** -8
    loss = [torch.zeros(40, device="cuda") for _ in range(3)]
    d = torch.zeros(40, 700, device="cuda")
    zd, vd = to_dev(z), to_dev(v)
    sats.distill_loss((zd + h * vd), *a, 1.5, 0.6, loss[0])
    sats.distill_loss((zd - h * vd), *a, 1.5, 0.6, loss[1])
    sats.distill_loss_grad(zd, *a, 1.5, 0.6, loss[2], d)
    quot = ((loss[0] - loss[1]) / (2 * h)).double().cpu().numpy()
    dot = (d.double() * vd.double()).sum(dim=1).cpu().numpy()
    np.testing.assert_allclose(quot, dot, rtol=0, atol=4.1e-3)


def test_same_result_every_time_and_in_a_graph(sats):
    z, idx, val, y, up = case(20, 40009, 50, 32, odd=True)
    zd = rows(z, torch.bfloat16, pad=7)
    a = (zd, to_dev(idx), to_dev(val), to_dev(y), 2.0, 0.5)
    dg = to_dev(up)
    new = lambda: (torch.zeros(20, device="cuda"), torch.zeros(20, 40009, dtype=torch.bfloat16, device="cuda"))
    loss, d = new()
    sats.distill_loss_grad(*a, loss, d, g=dg)
    for _ in range(3):
        l2, d2 = new()
        sats.distill_loss_grad(*a, l2, d2, g=dg)
        assert torch.equal(loss, l2) and torch.equal(d, d2)
    l2, d2 = new()
    lse = torch.zeros(20, 2, device="cuda")
    d3 = torch.zeros_like(d)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        sats.distill_loss_grad(*a, l2, d2, g=dg, stream=s)
        sats.distill_loss(*a, l2, lse=lse, stream=s)
        sats.distill_grad(*a, lse, d3, g=dg, stream=s)
    assert (d2 == 0).all()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(d, d2) and (d3 != 0).any()
    np.testing.assert_allclose(l2.cpu().numpy(), loss.cpu().numpy(), rtol=2.0 ** -20, atol=16 * DELTA)


def test_binding_refusals(sats):
    z = torch.zeros(4, 16, device="cuda")
    y = torch.zeros(4, dtype=torch.int32, device="cuda")
    i, v = torch.zeros(4, 2, dtype=torch.int32, device="cuda"), torch.zeros(4, 2, device="cuda")
    loss, lse = torch.zeros(4, device="cuda"), torch.zeros(4, 2, device="cuda")
    bad = [
        lambda: sats.distill_loss(z.double(), i, v, y, 1.0, 0.5, loss),
        lambda: sats.distill_loss(z, i, None, y, 1.0, 0.5, loss),
        lambda: sats.distill_loss(z, i, v[:, :1], y, 1.0, 0.5, loss),
        lambda: sats.distill_loss(z, i, v, y.long(), 1.0, 0.5, loss),
        lambda: sats.distill_loss(z, i, v, y, 1.0, 0.5, loss[:3]),
        lambda: sats.distill_loss(z, i, v, y, 1.0, 0.5, loss, lse=lse[:, :1]),
        lambda: sats.distill_grad(z, i, v, y, 1.0, 0.5, lse, z.bfloat16()),
        lambda: sats.distill_grad(z, i, v, y, 1.0, 0.5, lse, z[:, :8]),
        lambda: sats.distill_grad(z, i, v, y, 1.0, 0.5, lse, z.clone(), g=loss[:2]),
        lambda: sats.distill_loss_grad(z, i, v, y.cpu(), 1.0, 0.5, loss, z.clone()),
    ]
    for call in bad:
        with pytest.raises(ValueError):
            call()
    buf = torch.zeros(4, 24, device="cuda")
    with pytest.raises(sats.SatsError) as e:
        sats.distill_grad(buf[:, :16], i, v, y, 1.0, 0.5, lse, buf[:, 8:])
    assert e.value.status == sats.EINVAL
