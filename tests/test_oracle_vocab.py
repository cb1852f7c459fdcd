"""The 64-bit vocabulary operators that the kernels are tested against: hand-computed values, gradients against
differences, and the frequencies of drawn tokens against their probabilities."""
import numpy as np
import pytest

from oracle import vocab


def test_top_logits_orders_ties_by_index_and_skips_masked():
    z = np.array([[1.0, 3.0, -np.inf, 3.0, np.nan, 2.0], [-np.inf] * 6])
    v, i = vocab.top_logits(z, 5)
    assert i[0].tolist() == [1, 3, 5, 0, -1] and v[0, :4].tolist() == [3, 3, 2, 1] and v[0, 4] == -np.inf
    assert i[1].tolist() == [-1] * 5


def test_distill_by_hand():
    z = np.log(np.array([[0.5, 0.25, 0.25]]))
    idx, val = np.array([[0, 1]]), np.log(np.array([[0.75, 0.25]]))
    loss, lse, d = vocab.distill(z, idx, val, None, 1.0, 1.0)
    assert np.isclose(loss[0], 0.75 * np.log(0.75 / 0.5) + 0.0)
    assert np.allclose(d[0], [0.5 - 0.75, 0.0, 0.25]) and np.allclose(lse, 0.0)
    loss, _, d = vocab.distill(z, None, None, np.array([2]), 1.0, 0.0)
    assert np.isclose(loss[0], np.log(4.0)) and np.allclose(d[0], [0.5, 0.25, -0.75])
    assert vocab.distill(z, idx, val, np.array([-1]), 1.0, 0.5)[0][0] == 0


@pytest.mark.parametrize("tau,alpha", [(1.0, 1.0), (2.5, 1.0), (0.7, 0.3), (1.0, 0.0)])
def test_distill_gradient_is_the_difference_quotient(tau, alpha):
    g = np.random.default_rng(5)
    z, g_out = g.normal(0, 2, (3, 11)), g.normal(0, 1, 3)
    idx = np.array([[0, 5, 5, -1], [10, 2, 3, 4], [-1, -1, -1, -1]])
    val, y = g.normal(0, 2, (3, 4)), np.array([5, -1, 7])
    _, _, d = vocab.distill(z, idx, val, y, tau, alpha, g_out)
    h = 1e-5
    for r in range(3):
        for j in range(11):
            up, dn = z.copy(), z.copy()
            up[r, j] += h
            dn[r, j] -= h
            lu, ld = (vocab.distill(x, idx, val, y, tau, alpha)[0][r] for x in (up, dn))
            assert abs(g_out[r] * (lu - ld) / (2 * h) - d[r, j]) < 1e-8


def test_sample_cuts_by_hand():
    z = np.log(np.array([[4.0, 1.0, 2.0, 2.0, 1.0]]))
    f = lambda u, **kw: tuple(a[0] for a in vocab.sample(z, np.array([u]), **{k: [v] for k, v in kw.items()}))[:3]
    assert f(0.0)[0] == 0 and f(0.45)[0] == 1 and f(0.55)[0] == 2 and f(0.99)[0] == 4 and f(0.5)[2] == 5
    assert f(0.6, top_k=3)[0] == 2 and f(0.6, top_k=3)[2] == 3      # ties: 2 and 3 both, 1 and 4 not
    assert f(0.99, top_k=2)[0] == 2 and f(0.1, top_k=2)[2] == 2     # of the tied ones the lower index
    assert f(0.9, top_p=0.59)[2] == 2 and f(0.9, top_p=0.61)[2] == 3 and f(0.9, top_p=0.0)[2] == 1
    assert f(0.9, min_p=0.5)[2] == 3 and f(0.9, min_p=0.51)[2] == 1 and f(0.9, min_p=1.0)[0] == 0
    assert f(0.9, temperature=0.0)[:2] == (0, 0.0)
    assert np.isclose(f(0.9, top_k=3)[1], np.log(2 / 8))


def test_sample_frequencies():
    g = np.random.default_rng(3)
    z = np.tile(g.normal(0, 1, 12), (4000, 1))
    ids = vocab.sample(z, (np.arange(4000) + 0.5) / 4000, [0.8] * 4000)[0]
    w = np.exp((z[0] - z[0].max()) / 0.8)
    assert np.all(np.abs(np.bincount(ids, minlength=12) / 4000 - w / w.sum()) <= 2 / 4000)


def test_sample_of_masked_rows():
    z = np.array([[-np.inf, np.nan, -np.inf], [-np.inf, 0.0, -np.inf], [np.inf, 0.0, np.inf]])
    ids, lp, n, _ = vocab.sample(z, np.array([0.5, 0.5, 0.75]))
    assert ids.tolist() == [-1, 1, 2] and n.tolist() == [0, 1, 3] and lp[0] == -np.inf and np.isclose(lp[2], -np.log(2))
