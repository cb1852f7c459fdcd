"""Drawing a token against the 64-bit definition: the id and the number of kept tokens exactly, wherever no decision
lies within 2^-32 of going the other way (weights carry 35 bits); the log probability to fp32: a quotient and a
difference rounded to 2^-24 each and log1p to 2^-22, relative to the terms, which are at most |logprob| + log V + 1.
"""
import numpy as np
import pytest
import torch

from oracle import vocab
from tests.test_gpu_top_logits import logits, rows

pytestmark = pytest.mark.gpu
NEAR = 2.0 ** -32


@pytest.fixture(scope="module")
def sats():
    import __graft_entry__
    __graft_entry__.build()
    from paper_2607_08991_gb300 import sats as s
    return s


def dev(a, dtype=torch.float32):
    return None if a is None else torch.as_tensor(np.asarray(a)).to(dtype).cuda()


def draw(sats, z, u, T=None, k=None, p=None, mp=None, status=None):
    B = z.shape[0]
    ids = torch.full((B + 1,), 77, dtype=torch.int32, device="cuda")
    lp = torch.full((B + 1,), 7.0, device="cuda")
    n = torch.full((B + 1,), 77, dtype=torch.int32, device="cuda")
    sats.sample(z, dev(u), ids[:B], temperature=dev(T), top_k=dev(k, torch.int32), top_p=dev(p), min_p=dev(mp),
                logprob=lp[:B], n_kept=n[:B], dev_status=status)
    torch.cuda.synchronize()
    assert ids[B] == 77 and lp[B] == 7 and n[B] == 77
    return ids[:B].cpu().numpy(), lp[:B].double().cpu().numpy(), n[:B].cpu().numpy()


def check(sats, z, u, T=None, k=None, p=None, mp=None, unsure=1):
    f32 = lambda a: None if a is None else np.asarray(a, np.float32).astype(np.float64)
    u, T, p, mp = f32(u), f32(T), f32(p), f32(mp)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    ids, lp, n = draw(sats, z, u, T, k, p, mp, status)
    assert sats.get_status_word(status) == sats.OK
    ri, rl, rn, margin = vocab.sample(z.double().cpu().numpy(), u, T, k, p, mp)
    sure = margin > NEAR
    assert sure.sum() >= len(sure) - unsure
    assert np.array_equal(ids[sure], ri[sure]), (ids, ri, margin)
    assert np.array_equal(n[sure], rn[sure]), (n, rn, margin)
    fin = sure & np.isfinite(rl)
    assert np.array_equal(lp[sure & ~fin], rl[sure & ~fin])
    assert np.all(np.abs(lp[fin] - rl[fin]) <= 2.0 ** -21 * (np.abs(rl[fin]) + np.log(z.shape[1]) + 1)), (lp[fin], rl[fin])


def settings(B, V, seed):
    """Every combination of the cuts turns up over a few rows."""
    g = np.random.default_rng([seed, B, V])
    T = g.uniform(0.3, 1.5, B)
    k = np.where(g.random(B) < 0.5, 0, g.integers(1, max(2, min(V, 3000)), B))
    p = np.where(g.random(B) < 0.5, 1.0, g.uniform(0.05, 0.999, B))
    mp = np.where(g.random(B) < 0.5, 0.0, g.uniform(0.0, 0.5, B) ** 3)
    T[g.random(B) < 0.1] = 0.0
    return g.random(B), T, k, p, mp


KINDS = ["normal", "ties", "equal", "ascending", "masked", "half"]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [1, 2, 7, 8, 9, 100, 1000, 4099, 20011])
def test_sizes(sats, V, dtype):
    for n, kind in enumerate(KINDS):
        B = 12
        check(sats, rows(logits(kind, B, V, 41), dtype, pad=n, off=n), *settings(B, V, n))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("kind", KINDS)
def test_vocabulary(sats, kind, dtype):
    B, V = 16, 128256
    check(sats, rows(logits(kind, B, V, 42), dtype, pad=5, off=3), *settings(B, V, 43))


@pytest.mark.parametrize("mode", ["free", "top_p", "top_k", "large_k", "min_p", "greedy", "one", "all"])
def test_one_cut_at_a_time(sats, mode):
    B, V = 24, 30011
    g = np.random.default_rng(44)
    z = logits("normal", B, V, 45)
    z[np.arange(B), g.integers(0, V, B)] += np.linspace(0, 15, B).astype(np.float32)
    kw = dict(free=dict(), top_p=dict(p=g.uniform(0.01, 0.9999, B)), top_k=dict(k=g.integers(2, 1025, B)),
              large_k=dict(k=g.integers(1025, V, B)), min_p=dict(mp=g.uniform(0, 1, B) ** 4),
              greedy=dict(T=np.zeros(B)), one=dict(k=np.ones(B, int)),
              all=dict(k=np.full(B, V), p=np.full(B, 1.0), mp=np.zeros(B)))[mode]
    kw.setdefault("T", g.uniform(0.4, 2, B))
    for dtype in (torch.float32, torch.bfloat16):
        check(sats, rows(z, dtype, pad=1), g.random(B), **kw)


def test_edges_of_the_settings(sats):
    B, V = 9, 5003
    z = rows(logits("ties", B, V, 46), torch.float32)
    u = np.linspace(0, 1 - 2.0 ** -24, B)
    for kw in (dict(T=np.full(B, 1e-3)), dict(T=np.full(B, 1e-20)), dict(T=np.full(B, 1e-38)), dict(T=np.full(B, 1e6)),
               dict(mp=np.ones(B)), dict(p=np.zeros(B)), dict(p=np.full(B, -1.0)), dict(p=np.full(B, 1e-30)),
               dict(p=np.full(B, 1 - 2.0 ** -24)), dict(k=np.full(B, -3)), dict(k=np.full(B, V + 5)),
               dict(p=np.full(B, 7.0)), dict(mp=np.full(B, -1.0)), dict(mp=np.full(B, 1e-30)), dict()):
        check(sats, z, u, **kw)
    check(sats, rows(1e30 * logits("normal", B, V, 47), torch.float32), u, T=np.full(B, 1e30), p=np.full(B, 0.8))


def test_rows_with_infinities_and_nan(sats):
    B, V = 8, 3001
    z = logits("odd", B, V, 48)
    u = np.linspace(0, 0.999, B)
    for dtype in (torch.float32, torch.bfloat16):
        check(sats, rows(z, dtype), u)
        check(sats, rows(z, dtype), u, p=np.full(B, 0.5), k=np.full(B, 40))
    z[np.isinf(z)] = 0.25
    z[1] = -np.inf
    z[2] = np.nan
    z[3, 1:] = -np.inf
    zd = rows(z, torch.float32)
    check(sats, zd, u, p=np.full(B, 0.9))
    check(sats, zd, u, T=np.zeros(B))
    check(sats, zd, u, k=np.full(B, 7), mp=np.full(B, 0.1))


def test_equal_logits_are_exact(sats):
    # all weights alike: the token is floor(u V), the nucleus ceil(p V) tokens, in whatever way they are found
    V = 4096
    z = torch.full((64, V), -2.5, device="cuda")
    u = (np.arange(64) + 0.5) / 64
    ids, lp, n = draw(sats, z, u)
    assert np.array_equal(ids, np.floor(u * V)) and (n == V).all() and np.allclose(lp, -np.log(V), rtol=1e-6)
    p = np.full(64, 0.25)
    ids, lp, n = draw(sats, z, u, p=p)
    assert (n == V // 4).all() and np.array_equal(ids, np.floor(u * V / 4))
    ids, lp, n = draw(sats, z, u, k=np.full(64, 100))
    assert (n == 100).all() and np.array_equal(ids, np.floor(u * 100))


def test_many_draws_near_their_borders(sats):
    # a flat vocabulary, borders 1e-5 apart, and numbers next to them
    V, B = 100003, 64
    z1 = logits("normal", 1, V, 49) * 0.1
    z = rows(np.repeat(z1, B, axis=0), torch.float32)
    g = np.random.default_rng(50)
    w = np.exp(z1[0].astype(np.float64) - z1.max())
    cum = np.cumsum(w) / w.sum()
    u = (cum[g.integers(0, V - 1, B)] + g.choice([-1, 1], B) * 1e-7).astype(np.float32)
    check(sats, z, u)
    check(sats, z, u, p=np.full(B, 0.7))


@pytest.mark.parametrize("dtype,V", [(torch.float32, 400003), (torch.bfloat16, 800001)])
def test_rows_larger_than_the_cluster_memory(sats, dtype, V):
    B = 6
    check(sats, rows(logits("normal", B, V, 51), dtype, pad=3), *settings(B, V, 52))
    check(sats, rows(logits("ties", B, V, 51), dtype), np.linspace(0, 0.9, B), p=np.full(B, 0.9))


@pytest.mark.parametrize("B", [1, 40, 500])
def test_batches(sats, B):
    V = 16001
    check(sats, rows(logits("normal", B, V, 53), torch.bfloat16, pad=1), *settings(B, V, 54))


def test_large_offsets(sats):
    # rows so far apart that their offsets pass 32 bits
    V, B, ld = 4099, 3, (1 << 31) + 5
    buf = torch.empty((B - 1) * ld + V, dtype=torch.bfloat16, device="cuda")
    z = torch.as_strided(buf, (B, V), (ld, 1))
    z.copy_(torch.from_numpy(logits("normal", B, V, 60)))
    check(sats, z, [0.1, 0.5, 0.9], p=[0.9, 1.0, 0.3], k=[0, 0, 100])


def test_long_lists(sats):
    # sets that are sorted: a top-k near the list's limit, nuclei whose border lies among many equal tokens
    B, V = 6, 40009
    u = np.linspace(0.05, 0.95, B)
    for dtype in (torch.float32, torch.bfloat16):
        z = rows(logits("normal", B, V, 61), dtype)
        check(sats, z, u, k=[1024, 1000, 700, 512, 300, 257], p=[0.99, 1.0, 0.5, 0.999, 0.7, 1.0], mp=[0, 0.01, 0, 0, 0.2, 0])
        ties = logits("ties", B, V, 62)
        ties[3:] = np.round(ties[3:] / 3) * 3      # thousands of tokens share a value
        check(sats, rows(ties, dtype), u, p=[0.2, 0.6, 0.95, 0.2, 0.6, 0.95])
        check(sats, rows(ties, dtype), u, p=[0.2, 0.6, 0.95, 0.2, 0.6, 0.95], k=[2000, 5000, 1500, 2000, 5000, 1500])
    # a few hundred different values within one step of the weight
    near = np.full((B, V), -30.0, np.float32)
    near[:, ::50] = 1.0 + np.arange(near[:, ::50].shape[1], dtype=np.float32) * 1e-6
    check(sats, rows(near, torch.float32), u, p=[0.1, 0.3, 0.5, 0.7, 0.9, 0.99])


@pytest.mark.parametrize("T", [4.0, 20.0, 300.0])
def test_high_temperatures(sats, T):
    # weights so alike that many steps of the weight are within a logit of each other
    B, V = 5, 30011
    z = rows(logits("normal", B, V, 63), torch.float32)
    check(sats, z, np.linspace(0.01, 0.99, B), T=np.full(B, T), p=[0.05, 0.3, 0.7, 0.95, 0.9999])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("large", [None, 70.0, 300.0])
def test_flat_nuclei(sats, large, dtype):
    # thousands of tokens in every step of the weight, one far above them, few rows to many, with and without a top-k
    for B, V in ((4, 100003), (320, 20011)):
        g = np.random.default_rng([74, B])
        z = logits("normal", B, V, 75)
        if large:
            z[:, 11] = large
        z = rows(z, dtype, pad=1)
        T = np.resize([2.0, 4.0, 8.0, 20.0, 60.0], B)
        p = g.uniform(0.05, 0.999, B)
        check(sats, z, g.random(B), T=T, p=p, unsure=3)
        check(sats, z, g.random(B), T=T, p=p, k=g.integers(1025, V, B), unsure=3)


def few_values(kind, B, V, seed):
    """Rows that a count of their values serves badly, or not at all (bf16 numbers)."""
    g = np.random.default_rng([seed, B, V])
    z = g.normal(0, 2.2, (B, V))
    if kind == "large":            # many above 64
        z *= 30
    elif kind == "one_large":
        z[:, V // 3] = 64.0
    elif kind == "just_below":     # the largest that counts, and its neighbours
        z[:, ::7] = 63.75
        z[:, 1::7] = 63.5
    elif kind == "tiny":           # all next to nothing
        z *= 1e-4
    elif kind == "zeros":
        z[:, : V // 2] = 0.0
        z[:, 1:V // 2:2] = -0.0
    elif kind == "few_tiny":       # a border among them
        z = np.full((B, V), -6.0)
        z[:, ::61] = 2.0 ** -11 * g.integers(-2, 3, z[:, ::61].shape)
        z[:, ::1009] = 0.5
    elif kind == "far_below":      # most below -64
        z[:, g.permutation(V)[: V - V // 10]] = -200.0
        z[:, V // 2] = -64.0
    elif kind == "masked":
        z[:, g.permutation(V)[: V - V // 8]] = -np.inf
        z[:, 5::11] = np.nan
    elif kind == "negative":
        z -= 30.0
    elif kind == "negative_tiny":
        z = -np.abs(z)
        z[:, 17] = -1e-5
    elif kind == "top_zero":
        z = -np.abs(z) - 0.01
        z[:, [7, V - 3]] = 0.0
    elif kind == "equal":
        z[:] = 1.0
    elif kind == "two":
        z = np.where(g.random((B, V)) < 0.5, 1.0, 0.984375)
    return torch.from_numpy(z.astype(np.float32)).to(torch.bfloat16).float().numpy()


@pytest.mark.parametrize("kind", ["large", "one_large", "just_below", "tiny", "zeros", "few_tiny", "far_below", "masked",
                                  "negative", "negative_tiny", "top_zero", "equal", "two"])
@pytest.mark.parametrize("V", [4096, 33333])
def test_values(sats, kind, V):
    B = 6
    z = rows(few_values(kind, B, V, 70), torch.bfloat16, pad=3, off=1)
    u = np.array([0.001, 0.2, 0.45, 0.6, 0.85, 0.999])
    one = lambda u, **kw: check(sats, z, u, unsure=3, **kw)   # (equal tokens: shares that a border divides exactly)
    p = [0.2, 0.53, 0.8, 0.95, 0.999, 0.9999]
    one(u)
    one(u, p=p)
    one(u, p=p[::-1], T=[0.3, 0.7, 1.0, 1.5, 3.0, 30.0])
    one(u, mp=[0.5, 0.1, 0.01, 1e-4, 1e-9, 1e-14])
    one(u, p=p, mp=[1e-14, 1e-9, 1e-4, 0.01, 0.1, 0.5])
    for k in ([1, 2, 50, 192, 193, 1000], [V // 10, V // 10 + 1, V // 8, V // 2, V - 1, 1024], [400, 401, 402, 403, 404, 405]):
        one(u, k=k)
        one(u, k=k, p=p, T=[0.5, 1.0, 2.0, 0.8, 1.0, 40.0])
        one(u, k=k, p=p[::-1], mp=[0, 0.02, 0.3, 0, 1e-5, 0.1])


def test_values_of_long_rows(sats):
    # as many tokens of one value in a CTA as its counts hold, and more than that
    for V in (8 * 65408 - 1, 8 * 65408 + 9):
        for kind in ("equal", "two", "far_below"):
            z = rows(few_values(kind, 2, V, 71), torch.bfloat16)
            check(sats, z, [0.3, 0.99], p=[0.7, 1.0], k=[0, 70000])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [700, 2500, 6001])
def test_top_k_of_short_rows(sats, V, dtype):
    # as many rows as share the GPU out to one CTA each, top-k with more entries than groups
    B = 310
    g = np.random.default_rng([72, V])
    for kind in ("normal", "ties", "masked"):
        check(sats, rows(logits(kind, B, V, 73), dtype, pad=1), g.random(B), k=g.integers(1, 1100, B),
              p=np.where(g.random(B) < 0.5, 1.0, g.uniform(0.1, 0.99, B)), unsure=3)


def test_first_call_captured(sats):
    # a shape that no call has had before, captured at once
    B, V = 3, 77777
    z = rows(logits("normal", B, V, 64), torch.float32)
    ud, ids = dev([0.2, 0.5, 0.8]), torch.zeros(B, dtype=torch.int32, device="cuda")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        sats.sample(z, ud, ids, stream=s)
    g.replay()
    torch.cuda.synchronize()
    ri, _, _, margin = vocab.sample(z.double().cpu().numpy(), ud.double().cpu().numpy())
    assert (margin > NEAR).all() and np.array_equal(ids.cpu().numpy(), ri)


def test_bad_settings(sats):
    V = 1000
    z = rows(logits("normal", 8, V, 55), torch.float32)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    nan = float("nan")
    T = [1, -1, nan, np.inf, 1, 1, 1, 1]
    p = [1, 1, 1, 1, nan, 1, 1, 1]
    mp = [0, 0, 0, 0, 0, nan, 1.5, 0]
    u = [0.5, 0.5, 0.5, 0.5, 0.5, 0.5, 0.5, 1.0]
    ids, lp, n = draw(sats, z, u, T, None, p, mp, status)
    assert sats.get_status_word(status) == sats.EDEVICE and sats.get_status_word(status) == sats.OK
    assert ids[0] >= 0 and (ids[1:] == -1).all() and np.isnan(lp[1:]).all() and (n[1:] == 0).all() and n[0] == V
    ids2, _, _ = draw(sats, z, u, T, None, p, mp)
    assert np.array_equal(ids, ids2)


def test_streams_and_graphs(sats):
    B, V = 7, 50021
    u, T, k, p, mp = settings(B, V, 56)
    z = rows(logits("normal", B, V, 57), torch.bfloat16, pad=1)
    ud, ids, status = dev(u), torch.zeros(B, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    kw = dict(temperature=dev(T), top_k=dev(k, torch.int32), top_p=dev(p), min_p=dev(mp), dev_status=status)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        sats.sample(z, ud, ids, stream=s, **kw)
    f = lambda a: np.asarray(a, np.float32).astype(np.float64)
    for seed in (58, 59):
        z.copy_(torch.from_numpy(logits("normal", B, V, seed)))
        g.replay()
        torch.cuda.synchronize()
        ri, _, _, margin = vocab.sample(z.double().cpu().numpy(), f(u), f(T), k, f(p), f(mp))
        sure = margin > NEAR
        assert sure.sum() >= B - 1 and np.array_equal(ids.cpu().numpy()[sure], ri[sure])


def test_binding_refusals(sats):
    z = torch.zeros(4, 16, device="cuda")
    u, ids = torch.zeros(4, device="cuda"), torch.zeros(4, dtype=torch.int32, device="cuda")
    bad = [
        lambda: sats.sample(z.half(), u, ids),
        lambda: sats.sample(z, u.double(), ids),
        lambda: sats.sample(z, u, ids.long()),
        lambda: sats.sample(z, u[:3], ids),
        lambda: sats.sample(z, u, ids, temperature=u[:1]),
        lambda: sats.sample(z, u, ids, top_k=u),
        lambda: sats.sample(z, u, ids, top_p=u.cpu()),
        lambda: sats.sample(z, u, ids, n_kept=u),
        lambda: sats.sample(z, torch.zeros(8, device="cuda")[::2], ids),
    ]
    for call in bad:
        with pytest.raises(ValueError):
            call()
