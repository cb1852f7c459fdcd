"""The vocabulary operators as they are used together with the token routing: a teacher's top logits feed the
distillation of the sparse path, its label losses feed the routing calibration, and drawn tokens are routed by the
table that comes out."""
import numpy as np
import pytest
import torch

from oracle import vocab
from tests.test_gpu_distill import DELTA, close
from tests.test_gpu_sample import NEAR
from tests.test_gpu_top_logits import logits, rows

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def sats():
    import __graft_entry__
    __graft_entry__.build()
    from paper_2607_08991_gb300 import sats as s
    return s


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_teacher_to_routed_tokens(sats, oracle, dtype):
    T, V, K = 60, 2003, 24
    base = logits("normal", T, V, 61)
    g = np.random.default_rng(62)
    sparse = base + g.normal(0, 0.5, base.shape).astype(np.float32)
    zb, zs = rows(base, dtype, pad=5), rows(sparse, dtype, pad=5)
    b64, s64 = zb.double().cpu().numpy(), zs.double().cpu().numpy()
    new = lambda *shape, t=torch.float32: torch.zeros(shape, dtype=t, device="cuda")
    status = new(1, t=torch.int32)

    # the base model's top logits, and a step of the sparse model towards them
    val, idx = new(T, K), new(T, K, t=torch.int32)
    sats.top_logits(zb, val, idx)
    labels = torch.from_numpy(g.integers(0, V, T).astype(np.int32)).cuda()
    loss, d = new(T), torch.zeros(T, V, dtype=dtype, device="cuda")
    sats.distill_loss_grad(zs, idx, val, labels, 2.0, 0.5, loss, d, dev_status=status)
    rv, ri = vocab.top_logits(b64, K)
    y = labels.cpu().numpy()
    rl, _, rd = vocab.distill(s64, ri, rv, y, 2.0, 0.5, np.ones(T))
    close(loss.double().cpu().numpy(), rl, 12 * DELTA, 2.0 ** -20)
    close(d.double().cpu().numpy(), rd, 16 * DELTA, 2.0 ** -8)
    moved = rows((s64 - 0.1 * d.double().cpu().numpy()).astype(np.float32), torch.float32)
    after = new(T)
    sats.distill_loss(moved, idx, val, labels, 2.0, 0.5, after)
    r_after, _, _ = vocab.distill(moved.double().cpu().numpy(), ri, rv, y, 2.0, 0.5)
    close(after.double().cpu().numpy(), r_after, 12 * DELTA, 2.0 ** -20)

    # both paths' label losses to the routing table
    ids = torch.from_numpy(g.integers(0, 40, T).astype(np.int32)).cuda()
    l_base, l_sparse = new(T), new(T)
    sats.distill_loss(zb, None, None, labels, 1.0, 0.0, l_base, dev_status=status)
    sats.distill_loss(zs, None, None, labels, 1.0, 0.0, l_sparse, dev_status=status)
    rb, rs = vocab.distill(b64, None, None, y, 1.0, 0.0)[0], vocab.distill(s64, None, None, y, 1.0, 0.0)[0]
    close(l_base.double().cpu().numpy(), rb, 2 * DELTA, 2.0 ** -20)
    score = sats.token_scores(ids, l_base, l_sparse, V)
    r_score = oracle.token_scores(ids.cpu().numpy(), rb.astype(np.float32), rs.astype(np.float32), V)
    seen = np.isfinite(r_score)
    assert np.array_equal(np.isfinite(score.cpu().numpy()), seen)
    assert np.abs(score.cpu().numpy()[seen] - r_score[seen]).max() <= 6 * DELTA
    _, _, lut = sats.route_calibrate(score, ids, 0.5)

    # the next tokens, and where they go
    nxt, u = new(T, t=torch.int32), torch.from_numpy(g.random(T).astype(np.float32)).cuda()
    sats.sample(zs, u, nxt, top_k=torch.full((T,), 50, dtype=torch.int32, device="cuda"),
                top_p=torch.full((T,), 0.9, device="cuda"), dev_status=status)
    p9 = np.full(T, np.float64(np.float32(0.9)))
    r_ids, _, _, margin = vocab.sample(s64, u.double().cpu().numpy(), None, np.full(T, 50), p9)
    sure = margin > NEAR
    assert sure.sum() >= T - 1 and np.array_equal(nxt.cpu().numpy()[sure], r_ids[sure])
    perm, n_dense = new(T, t=torch.int32), new(1, t=torch.int32)
    sats.route(nxt, lut, perm, n_dense, dev_status=status)
    flags = lut.cpu().numpy()[nxt.cpu().numpy()] != 0
    want = np.concatenate([np.flatnonzero(flags), np.flatnonzero(~flags)])
    assert np.array_equal(perm.cpu().numpy(), want) and int(n_dense) == flags.sum()
    assert sats.get_status_word(status) == sats.OK


def test_same_stream_order_without_waits(sats):
    # two streams with their own rows at the same time; each call's results are its own
    V, B = 40009, 30
    a, b = (rows(logits("normal", B, V, s), torch.bfloat16) for s in (63, 64))
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = []
    u = torch.rand(B, generator=torch.Generator().manual_seed(65)).cuda()
    p = torch.full((B,), 0.95, device="cuda")
    alone = []
    for z in (a, b):
        ids = torch.zeros(B, dtype=torch.int32, device="cuda")
        sats.sample(z, u, ids, top_p=p)
        alone.append(ids)
    torch.cuda.synchronize()
    for rep in range(4):
        for z, s in zip((a, b), streams):
            ids = torch.zeros(B, dtype=torch.int32, device="cuda")
            s.wait_stream(torch.cuda.current_stream())
            sats.sample(z, u, ids, top_p=p, stream=s)
            outs.append(ids)
    torch.cuda.synchronize()
    for n, ids in enumerate(outs):
        assert torch.equal(ids, alone[n % 2])
