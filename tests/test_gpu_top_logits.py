"""The top logits of a row against a sort: values and indices exactly, at sizes around the vector and the cluster
width, on rows that start anywhere, with ties, masked places, NaN, infinities and both zeros."""
import numpy as np
import pytest
import torch

from oracle import vocab

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def sats():
    import __graft_entry__
    __graft_entry__.build()
    from paper_2607_08991_gb300 import sats as s
    return s


def rows(values, dtype, pad=0, off=0, fill=float("nan")):
    """A device tensor [T][V] of these values, its rows `pad` elements apart and `off` elements into an allocation;
    what lies around them is `fill`."""
    T, V = values.shape
    buf = torch.full((T * (V + pad) + off + 64,), fill, dtype=dtype, device="cuda")
    z = buf[off:off + T * (V + pad)].view(T, V + pad)[:, :V]
    z.copy_(torch.from_numpy(np.ascontiguousarray(values)))
    return z


def logits(kind, T, V, seed):
    g = np.random.default_rng([seed, T, V, len(kind)])
    z = g.normal(0, 2.5, (T, V))
    if kind == "ties":
        z = np.round(z)
    elif kind == "equal":
        z[:] = 1.25
    elif kind == "ascending":          # the largest all in the last CTA
        z = np.sort(z, axis=1)
    elif kind == "masked":             # most places, whole stretches among them
        z[g.random((T, V)) < 0.9] = -np.inf
        z[:, : V // 2] = -np.inf
        z[0] = -np.inf
    elif kind == "half":               # a stretch that leaves more than the list holds
        z[:, : V // 2] = -np.inf
    elif kind == "odd":
        z[g.random((T, V)) < 0.2] = np.nan
        z[g.random((T, V)) < 0.1] = np.inf
        z[g.random((T, V)) < 0.2] = 0.0
        z[g.random((T, V)) < 0.2] = -0.0
        z[g.random((T, V)) < 0.1] = np.finfo(np.float32).min
        z[g.random((T, V)) < 0.1] = 1e-42
    return z.astype(np.float32)


def check(sats, z, K):
    T = z.shape[0]
    v = torch.full((T + 1, K), 7.0, device="cuda")
    i = torch.full((T + 1, K), 7, dtype=torch.int32, device="cuda")
    sats.top_logits(z, v[:T], i[:T])
    torch.cuda.synchronize()
    rv, ri = vocab.top_logits(z.double().cpu().numpy(), K)
    assert np.array_equal(i[:T].cpu().numpy(), ri)
    assert np.array_equal(v[:T].cpu().numpy().astype(np.float64), rv)
    assert (v[T:] == 7).all() and (i[T:] == 7).all()       # what lies behind the last row


KINDS = ["normal", "ties", "equal", "ascending", "masked", "half", "odd"]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V,K", [(1, 1), (2, 2), (7, 3), (8, 8), (9, 1), (33, 33), (1000, 50), (1024, 1024), (4099, 600),
                                 (50001, 64)])
def test_sizes(sats, V, K, dtype):
    for n, kind in enumerate(KINDS):
        T = 3
        check(sats, rows(logits(kind, T, V, 11), dtype, pad=n, off=n), K)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("kind", KINDS)
def test_vocabulary(sats, kind, dtype):
    for K in (1, 20, 1024):
        check(sats, rows(logits(kind, 2, 128256, 12), dtype, pad=5, off=1), K)


@pytest.mark.parametrize("T", [1, 2, 40, 400])
def test_rows(sats, T):
    # from rows that share the GPU out among clusters to more of them than fit
    check(sats, rows(logits("ties", T, 20011, 13), torch.bfloat16, pad=3), 17)


@pytest.mark.parametrize("dtype,V", [(torch.float32, 400003), (torch.bfloat16, 800001)])
def test_rows_larger_than_the_cluster_memory(sats, dtype, V):
    for kind in ("normal", "equal", "half"):
        check(sats, rows(logits(kind, 2, V, 14), dtype, pad=1), 100)


def long_lists(kind, T, V, seed):
    """Rows whose long lists are unevenly spread."""
    g = np.random.default_rng([seed, T, V])
    if kind == "outliers":             # nearly all of the list within one step of it
        z = g.normal(0, 1e-3, (T, V))
        z[:, V // 3] = 50.0
        z[:, 0] = np.finfo(np.float32).min
    elif kind == "narrow":             # neighbouring numbers
        z = 1.0 + g.integers(0, 300, (T, V)) * 2.0 ** -23
    elif kind == "bounded":            # the K-th largest among hundreds of equal ones
        z = np.where(g.random((T, V)) < 0.1, 2.0, g.normal(-3, 1, (T, V)))
    else:
        return logits(kind, T, V, seed)
    return z.astype(np.float32)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("kind", KINDS + ["outliers", "narrow", "bounded"])
def test_long_lists(sats, kind, dtype):
    # few rows to many (one CTA a row), rows of fewer groups than entries to long ones
    for T, V in ((2, 1500), (3, 30011), (160, 2003), (320, 5003)):
        z = rows(long_lists(kind, T, V, 16), dtype, pad=1, off=1)
        for K in (130, 257, 1000, 1024):
            check(sats, z, K)


def test_large_offsets(sats):
    # rows so far apart that their offsets pass 32 bits
    V, T = 4099, 3
    ld = (1 << 31) + 5
    buf = torch.empty((T - 1) * ld + V, dtype=torch.bfloat16, device="cuda")
    z = torch.as_strided(buf, (T, V), (ld, 1))
    z.copy_(torch.from_numpy(logits("normal", T, V, 15)))
    check(sats, z, 9)


def test_streams_and_graphs(sats):
    z = rows(logits("ties", 5, 30011, 16), torch.bfloat16)
    v, i = torch.zeros(5, 40, device="cuda"), torch.zeros(5, 40, dtype=torch.int32, device="cuda")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        sats.top_logits(z, v, i, stream=s)
    assert (v == 0).all()
    for seed in (17, 18):
        z.copy_(torch.from_numpy(logits("ties", 5, 30011, seed)))
        g.replay()
        torch.cuda.synchronize()
        rv, ri = vocab.top_logits(z.double().cpu().numpy(), 40)
        assert np.array_equal(i.cpu().numpy(), ri) and np.array_equal(v.cpu().numpy(), rv)


def test_binding_refusals(sats):
    z = torch.zeros(4, 16, device="cuda")
    v, i = torch.zeros(4, 3, device="cuda"), torch.zeros(4, 3, dtype=torch.int32, device="cuda")
    with pytest.raises(ValueError):
        sats.top_logits(z.half(), v, i)
    with pytest.raises(ValueError):
        sats.top_logits(z.t(), v, i)
    with pytest.raises(ValueError):
        sats.top_logits(z[:1].expand(4, 16), v, i)
    with pytest.raises(ValueError):
        sats.top_logits(z, v, i.long())
    with pytest.raises(ValueError):
        sats.top_logits(z, v[:3], i)
    with pytest.raises(sats.SatsError) as e:
        sats.top_logits(z, torch.zeros(4, 17, device="cuda"), torch.zeros(4, 17, dtype=torch.int32, device="cuda"))
    assert e.value.status == sats.EINVAL
