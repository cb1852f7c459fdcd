"""The bounded waits of the one-pass distillation, run out without a fault: a CTA does not get another's sums of one row.
The status says so, every place is either right or NaN, and the stream serves the next call."""
import time

import numpy as np
import pytest
import torch

from tests.test_gpu_top_logits import logits, rows

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def sats():
    import __graft_entry__
    __graft_entry__.build()
    from paper_2607_08991_gb300 import sats as s
    return s


@pytest.mark.parametrize("V,T,row,pad", [(50021, 1000, 5, 0), (50021, 1000, 999, 3), (320001, 300, 0, 7)])
def test_a_cta_that_gives_up_leaves_nan(sats, V, T, row, pad):
    # rows of two CTAs and of eight, many rows for each cluster (228 at most fit on 152 SMs)
    z = rows(logits("normal", 50, V, 81), torch.bfloat16)
    z = z.repeat(T // 50, 1)
    g = np.random.default_rng(82)
    y = g.integers(0, V, T).astype(np.int32)
    y[g.random(T) < 0.1] = -1
    y[row] = 7
    y = torch.from_numpy(y).cuda()
    new = lambda: (torch.full((T,), 9.0, device="cuda"),
                   torch.full((T, V + pad), 9.0, dtype=torch.bfloat16, device="cuda")[:, :V])
    loss, d = new()
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    sats.distill_loss_grad(z, None, None, y, 1.0, 0.0, loss, d, dev_status=status)
    assert sats.get_status_word(status) == sats.OK and torch.isfinite(loss).all()
    loss2, d2 = new()
    t0 = time.perf_counter()
    sats.selftest_distill_timeout(z, y, loss2, d2, row, status)
    assert sats.get_status_word(status) == sats.ETIMEOUT
    assert 1.9 < time.perf_counter() - t0 < 8           # one limit, and one more of those that depend on it
    wrong = torch.isnan(loss2)
    same = d2 == d
    assert torch.equal(loss2[~wrong], loss[~wrong]) and (same | torch.isnan(d2)).all()
    live = (y >= 0).cpu().numpy()
    rows_off = torch.nonzero(~same.all(dim=1)).flatten().cpu().numpy()
    assert wrong[row] and rows_off.min() == row         # the first CTA has the loss
    # the rows that this cluster serves from there on, evenly apart, all of them and no others
    assert np.array_equal(rows_off, torch.nonzero(wrong).flatten().cpu().numpy())
    if row + 1 < T // 2:
        hop = np.gcd.reduce(rows_off - row)
        assert rows_off.size > 1 and hop > 1
        mine = np.arange(row, T, hop)
        assert np.array_equal(rows_off, mine[live[mine]])
        # after the first row no CTA of the cluster has all sums
        later = rows_off[1:]
        assert torch.isnan(d2[later]).all()
    else:
        assert rows_off.size == 1
    loss3, d3 = new()
    sats.distill_loss_grad(z, None, None, y, 1.0, 0.0, loss3, d3, dev_status=status)
    assert sats.get_status_word(status) == sats.OK
    assert torch.equal(loss3, loss) and torch.equal(d3, d)
