"""Inputs at the edges of what the vocabulary operators allow."""
import numpy as np
import pytest
import torch

from oracle import vocab
from tests.test_gpu_distill import check, to_dev
from tests.test_gpu_top_logits import logits, rows

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def sats():
    import __graft_entry__
    __graft_entry__.build()
    from paper_2607_08991_gb300 import sats as s
    return s


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V,apart", [(1 << 23, 0), ((1 << 23) + 8, 0), (1 << 24, 0), (1 << 24, 30)])
def test_nucleus_of_millions_of_equal_tokens(sats, V, apart, dtype):
    # so many tokens of one weight in each CTA that 32-bit counts of them pass their range, some to exactly 0.  All weigh
    # 1, or every second one next to nothing at all (30 / T is past 62 octaves): the n = ceil(p number) first ones are kept,
    # and of those number floor(u n) is drawn, whatever the way there (u and p are exact in binary)
    u, p = [0.0, 0.25, 0.8125], [0.5, 0.4375, 0.75]
    z = torch.zeros(3, V, dtype=dtype, device="cuda")
    T = 100.0
    if apart:
        z[:, 1::2] = -float(apart) * T * 2
    ids, n = (torch.full((3,), 77, dtype=torch.int32, device="cuda") for _ in range(2))
    lp = torch.full((3,), 7.0, device="cuda")
    dev = lambda a: torch.tensor(a, device="cuda")
    sats.sample(z, dev(u), ids, temperature=dev([T] * 3), top_p=dev(p), logprob=lp, n_kept=n)
    number, step = (V // 2, 2) if apart else (V, 1)
    kept = [int(np.ceil(x * number)) for x in p]
    assert n.tolist() == kept
    assert ids.tolist() == [int(np.floor(x * m)) * step for x, m in zip(u, kept)]
    # the logarithm of a whole number, rounded a few times
    np.testing.assert_allclose(lp.cpu().numpy(), -np.log(np.array(kept, np.float64)), rtol=2.0 ** -21)


@pytest.mark.parametrize("dtype,V", [(torch.float32, 5), (torch.float32, 1000), (torch.bfloat16, 5003), (torch.float32, 100003)])
@pytest.mark.parametrize("kw", [dict(), dict(top_k=20), dict(top_k=700), dict(top_p=0.5), dict(min_p=0.1), dict(temperature=-0.0)])
def test_negative_zeros_are_zeros(sats, dtype, V, kw):
    # a random number of -0 lies in [0, 1): the first kept token
    z = rows(logits("normal", 4, V, 93), dtype, pad=1)
    dev = lambda a, t: torch.tensor(a, dtype=t, device="cuda")
    args = {k: dev([v] * 4, torch.int32 if k == "top_k" else torch.float32) for k, v in kw.items()}
    got = []
    for u in ([-0.0, 0.0, -0.0, 0.25], [0.0, 0.0, 0.0, 0.25]):
        ids = torch.full((4,), -7, dtype=torch.int32, device="cuda")
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        sats.sample(z, dev(u, torch.float32), ids, dev_status=status, **args)
        assert sats.get_status_word(status) == sats.OK
        got.append(ids.tolist())
    ref = {k: [v] * 4 for k, v in kw.items()}
    ri = vocab.sample(z.double().cpu().numpy(), np.array([0.0, 0.0, 0.0, 0.25]), **ref)[0]
    assert got[0] == got[1] == ri.tolist()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T,V,gap", [(5, 900, 0), (400, 900, 7), (30, 60001, 3)])
def test_gradient_between_the_rows_of_the_logits(sats, T, V, gap, dtype):
    # one buffer, in turn a row of logits and a row for its gradient, either of them first
    g = np.random.default_rng([94, T])
    values = logits("normal", T, V, 95)
    y = torch.from_numpy(g.integers(-1, V, T).astype(np.int32)).cuda()
    z = rows(values, dtype)
    loss, lse, d = torch.zeros(T, device="cuda"), torch.zeros(T, 2, device="cuda"), torch.zeros_like(z)
    sats.distill_loss(z, None, None, y, 1.0, 0.0, loss, lse=lse)
    sats.distill_grad(z, None, None, y, 1.0, 0.0, lse, d)
    for first in (True, False):
        for one_pass in (False, True):
            buf = torch.full((T, 2 * V + 2 * gap), 9.0, dtype=dtype, device="cuda")
            own, out = buf[:, :V], buf[:, V + gap:2 * V + gap]
            if not first:
                own, out = out, own
            own.copy_(z)
            l2 = torch.zeros(T, device="cuda")
            if one_pass:
                sats.distill_loss_grad(own, None, None, y, 1.0, 0.0, l2, out)
            else:
                sats.distill_loss(own, None, None, y, 1.0, 0.0, l2)
                sats.distill_grad(own, None, None, y, 1.0, 0.0, lse, out)
            torch.cuda.synchronize()
            assert torch.equal(own, z) and (buf[:, V:V + gap] == 9).all() and (buf[:, 2 * V + gap:] == 9).all()
            # the sums in another order: within 2^-15 of one another (absolute, of a loss and of a probability; the
            # gradient's rounding to its type on top)
            assert ((l2 - loss).abs() <= 2.0 ** -14).all()
            eps = 2.0 ** -7 if dtype == torch.bfloat16 else 2.0 ** -22
            assert ((out.float() - d.float()).abs() <= 2.0 ** -14 + eps * d.float().abs()).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T,V", [(12, 500), (12, 60001), (700, 500), (260, 60001)])
@pytest.mark.parametrize("tau,alpha,labels,entries", [(1.0, 0.0, True, False), (1.0, 0.5, True, True), (2.0, 0.5, True, True),
                                                      (2.0, 1.0, False, True), (2.0, 0.5, False, True), (1.0, 1.0, True, True)])
def test_rows_without_a_finite_sum(sats, T, V, tau, alpha, labels, entries, dtype):
    # all three calls, one row a cluster and many, one CTA a row and several: the rows that are not ordinary ones have NaN
    # where the header says so, the others are what they would be without them
    K, n = 6, 9
    g = np.random.default_rng([96, T, V])
    z = logits("normal", T, V, 97)
    idx = np.stack([g.permutation(V)[:K] for _ in range(T)]).astype(np.int32)
    val = g.normal(0, 2, (T, K)).astype(np.float32)
    y = g.integers(0, V, T).astype(np.int32)
    up = g.uniform(0.5, 1.5, T).astype(np.float32)
    at = g.permutation(T)[:n]                        # where the special rows are
    nan_at, inf_at = int(g.integers(0, V)), int(g.integers(0, V))
    for r in at[[0, 4, 6]]:
        z[r, nan_at] = np.nan
    for r in at[[1, 7]]:
        z[r, inf_at] = np.inf
    z[at[[2, 8]]] = -np.inf
    up[at[[4, 8]]] = 0.0                             # of which one has no weight ...
    idx[at[[6, 7]]] = -1                             # ... or no entries
    val[at[3], 2], val[at[5], 0] = np.nan, np.inf    # a teacher's value that is none
    zd = rows(z, dtype, pad=1)
    a = (to_dev(idx) if entries else None, to_dev(val) if entries else None, to_dev(y) if labels else None)
    loss, loss2, lse = torch.zeros(T, device="cuda"), torch.zeros(T, device="cuda"), torch.zeros(T, 2, device="cuda")
    d, d2 = torch.zeros_like(zd), torch.zeros_like(zd)
    sats.distill_loss(zd, *a, tau, alpha, loss, lse=lse)
    sats.distill_grad(zd, *a, tau, alpha, lse, d, g=to_dev(up))
    sats.distill_loss_grad(zd, *a, tau, alpha, loss2, d2, g=to_dev(up))
    soft, hard = entries and alpha > 0, labels and alpha < 1
    nan_loss = np.zeros(T, bool)
    nan_grad = np.zeros((T, V), bool)
    for r in at:
        counts = hard or (soft and (idx[r] >= 0).any())
        numbers = np.isfinite(z[r]) | (z[r] == -np.inf)
        odd_row = not numbers.all() or not np.isfinite(z[r]).any()
        odd_val = soft and not np.isfinite(val[r]).all()
        nan_loss[r] = odd_row and counts or odd_val
        if odd_row:
            nan_grad[r] = ~numbers if up[r] == 0 or not counts else True
        elif odd_val:
            nan_grad[r, idx[r]] = True
    for got, name in ((loss, "loss"), (loss2, "one-pass loss")):
        assert np.array_equal(torch.isnan(got).cpu().numpy(), nan_loss), name
    for got, name in ((d, "gradient"), (d2, "one-pass gradient")):
        got = got.float().cpu().numpy()
        assert np.array_equal(np.isnan(got), nan_grad), (name, np.argwhere(np.isnan(got) != nan_grad)[:5], at)
        gone = at[[r for r in range(n) if nan_grad[at[r]].any() and not nan_grad[at[r]].all() and r not in (3, 5)]]
        assert (np.nan_to_num(got[gone]) == 0).all()
    rest = np.setdiff1d(np.arange(T), at)[:40]
    pick = lambda x: None if x is None else x[rest]
    check(sats, rows(z[rest], dtype, pad=1), pick(idx) if entries else None, pick(val) if entries else None,
          pick(y) if labels else None, pick(up), tau, alpha, d_pad=1)


def test_calls_at_once_on_two_streams(sats):
    # eager calls on one stream while another replays a captured one: nothing is shared between them
    V, T, K = 60001, 300, 16
    z = [rows(logits("normal", T, V, 98 + i), torch.bfloat16, pad=i) for i in range(2)]
    y = torch.arange(T, dtype=torch.int32, device="cuda")
    u = torch.linspace(0, 0.999, T, device="cuda")

    def outputs():
        return (torch.zeros(T, K, device="cuda"), torch.zeros(T, K, dtype=torch.int32, device="cuda"),
                torch.zeros(T, device="cuda"), torch.zeros(T, V, dtype=torch.bfloat16, device="cuda"),
                torch.zeros(T, dtype=torch.int32, device="cuda"))

    def calls(x, o, stream=None):
        sats.top_logits(x, o[0], o[1], stream=stream)
        sats.distill_loss_grad(x, o[1], o[0], y, 2.0, 0.5, o[2], o[3], stream=stream)
        sats.sample(x, u, o[4], stream=stream)

    alone = [outputs() for _ in range(2)]
    for x, o in zip(z, alone):
        calls(x, o)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [outputs() for _ in range(2)]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=streams[0]):
        calls(z[0], got[0], streams[0])
    for _ in range(4):
        for o in got:
            for t in o:
                t.zero_()
        torch.cuda.synchronize()
        with torch.cuda.stream(streams[0]):
            graph.replay()
        calls(z[1], got[1], streams[1])
        torch.cuda.synchronize()
        for a, b in zip(alone, got):
            assert all(torch.equal(s, t) for s, t in zip(a, b))
