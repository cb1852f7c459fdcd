"""The tail of a decode step as it is used: the stack's output normalised, the 4-bit head, penalties and masks on its logits, a
token drawn and routed, by itself and as one graph; and the way back from a loss of the adjusted logits.

Each stage is held against 64 bits on what the stage before it gave.  Tolerances: RMSNorm's own (2^-21 of the value, the
mean of H squares and a root in fp32); the others' as in the tests of the single operators.
"""
import numpy as np
import pytest
import torch

from oracle import adjust as ref_adjust
from oracle import q4, vocab
from tests.test_gpu_adjust import case, close, expected
from tests.test_gpu_q4 import check
from tests.test_gpu_sample import NEAR

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def sats():
    import __graft_entry__
    __graft_entry__.build()
    from paper_2607_08991_gb300 import sats as s
    return s


class Tail:
    """Buffers, weights and settings of a server's decode step; go() makes the calls."""

    def __init__(self, sats, B, H, V, dtype, seed):
        g = np.random.default_rng(seed)
        cuda = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()
        self.sats, self.B, self.V, self.G = sats, B, V, 64
        W = torch.from_numpy(g.normal(size=(H, V)) * 2.0 * H ** -0.5).to(torch.bfloat16).cuda()
        self.codes = torch.empty(H // 2, V, dtype=torch.uint8, device="cuda")
        self.scales = torch.empty((H + 63) // 64, V, dtype=torch.bfloat16, device="cuda")
        sats.q4_quantize(W, self.codes, self.scales, self.G)
        self.head = sats.Q4(self.codes, self.scales, self.G)
        self.ws = sats.Q4Workspace(self.head, B)
        self.x, self.norm_w = cuda(g.normal(size=(B, H)).astype(np.float32)), cuda((1 + 0.1 * g.normal(size=H)).astype(np.float32))
        self.n = torch.empty(B, H, device="cuda")
        self.logits = torch.empty(B, V, dtype=dtype, device="cuda")
        self.a = case(B, V, 90, seed + 1, M=6, masks=2)
        self.a["mask"][:] |= 255          # (something is always allowed)
        self.a["bias_val"] = np.where(np.isinf(self.a["bias_val"]), -4.0, self.a["bias_val"]).astype(np.float32)
        self.args = {k: cuda(v) for k, v in self.a.items()}
        self.adjusted = torch.empty_like(self.logits)
        self.u = cuda(g.random(B).astype(np.float32))
        self.temperature = cuda(g.uniform(0.5, 1.5, B).astype(np.float32))
        self.top_p = cuda(np.full(B, 0.9, np.float32))
        self.lut = cuda((g.random(V) < 0.5).astype(np.uint8))
        i32 = lambda n: torch.zeros(n, dtype=torch.int32, device="cuda")
        self.ids, self.perm, self.n_dense, self.status = i32(B), i32(B), i32(1), i32(1)

    def go(self):
        s = self.sats
        s.rmsnorm(self.x, self.norm_w, 1e-6, self.n)
        s.q4_matmul(self.head, self.n, self.logits, self.ws)
        s.adjust_logits(self.logits, self.adjusted, dev_status=self.status, **self.args)
        s.sample(self.adjusted, self.u, self.ids, temperature=self.temperature, top_p=self.top_p, dev_status=self.status)
        s.route(self.ids, self.lut, self.perm, self.n_dense, dev_status=self.status)

    def look(self):
        f64 = lambda t: t.double().cpu().numpy()
        x = f64(self.x)
        n = x / np.sqrt((x ** 2).mean(axis=1, keepdims=True) + 1e-6) * f64(self.norm_w)
        assert np.abs(f64(self.n) - n).max() <= 2.0 ** -21 * np.abs(n).max()
        check(self.logits, self.n, q4.unpack(self.codes.cpu().numpy()), f64(self.scales), self.G)
        z = f64(self.logits)
        close(f64(self.adjusted), expected(z, self.a), z, self.a, self.logits.dtype)
        ids, _, _, margin = vocab.sample(f64(self.adjusted), f64(self.u), f64(self.temperature), None, f64(self.top_p))
        sure = margin > NEAR
        assert sure.sum() >= self.B - 1 and np.array_equal(self.ids.cpu().numpy()[sure], ids[sure])
        flags = self.lut.cpu().numpy()[self.ids.cpu().numpy()] != 0
        assert np.array_equal(self.perm.cpu().numpy(), np.concatenate([np.flatnonzero(flags), np.flatnonzero(~flags)]))
        assert int(self.n_dense) == flags.sum()
        assert self.sats.get_status_word(self.status) == self.sats.OK
        assert self.sats.get_error(self.ws) == self.sats.OK


@pytest.mark.parametrize("B,H,V,dtype", [(1, 512, 4099, torch.float32), (7, 1024, 8000, torch.bfloat16),
                                         (40, 256, 12001, torch.bfloat16), (70, 512, 3001, torch.float32)])
def test_decode_step(sats, B, H, V, dtype):
    t = Tail(sats, B, H, V, dtype, B + V)
    t.go()
    t.look()


@pytest.mark.parametrize("B", [1, 24])
def test_decode_step_as_a_graph(sats, B):
    t = Tail(sats, B, 512, 5003, torch.bfloat16, 70 + B)
    t.go()
    t.look()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        t.go()
        t.go()
    for seed in range(3):
        gen = torch.Generator().manual_seed(seed)
        t.x.copy_(torch.randn(t.x.shape, generator=gen))
        t.u.copy_(torch.rand(B, generator=gen))
        t.ids.fill_(-1)
        t.logits.zero_()
        g.replay()
        torch.cuda.synchronize()
        t.look()


def test_two_graphs_with_their_own_workspaces(sats):
    """Two captured steps on two streams at once, the same head."""
    a, b = (Tail(sats, 6, 512, 5003, torch.float32, s) for s in (80, 81))
    b.head, b.codes, b.scales = a.head, a.codes, a.scales
    b.ws = sats.Q4Workspace(a.head, 6)
    graphs, streams = [], [torch.cuda.Stream() for _ in range(2)]
    for t in (a, b):
        t.go()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            t.go()
        graphs.append(g)
    torch.cuda.synchronize()
    for t in (a, b):
        t.logits.zero_()
        t.ids.fill_(-1)
    torch.cuda.synchronize()
    for _ in range(10):
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
    torch.cuda.synchronize()
    a.look()
    b.look()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_loss_of_adjusted_logits(sats, dtype):
    """Cross entropy of the adjusted logits and its gradient with respect to the model's, in place all the way."""
    T, V = 50, 3001
    g = np.random.default_rng(91)
    seq = g.integers(0, V, T).astype(np.int32)
    z = torch.from_numpy(g.normal(size=(T, V)) * 2).to(dtype).cuda()
    a = dict(hist=np.broadcast_to(seq, (T, T)), hist_len=np.arange(T, dtype=np.int32),
             repetition=g.uniform(1.0, 1.5, T).astype(np.float32))
    hist = torch.from_numpy(seq).cuda()[None].expand(T, T)
    args = dict(hist=hist, hist_len=torch.from_numpy(a["hist_len"]).cuda(), repetition=torch.from_numpy(a["repetition"]).cuda())
    labels = torch.from_numpy(g.integers(0, V, T).astype(np.int32)).cuda()
    adjusted, loss = torch.empty_like(z), torch.empty(T, device="cuda")
    sats.adjust_logits(z, adjusted, **args)
    z64 = z.double().cpu().numpy()
    close(adjusted.double().cpu().numpy(), expected(z64, a), z64, a, dtype)
    a64, y = adjusted.double().cpu().numpy(), labels.cpu().numpy()
    sats.distill_loss_grad(adjusted, None, None, labels, 1.0, 0.0, loss, adjusted)
    d_in = adjusted.double().cpu().numpy()
    sats.adjust_logits_grad(z, adjusted, adjusted, **args)
    want_loss, _, want_d = vocab.distill(a64, None, None, y, 1.0, 0.0, np.ones(T))
    assert np.abs(loss.double().cpu().numpy() - want_loss).max() <= 2.0 ** -18 * max(1, np.abs(want_loss).max())
    half = 2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -20
    assert (np.abs(d_in - want_d) <= half * np.abs(want_d) + 2.0 ** -20).all()
    got, want = adjusted.double().cpu().numpy(), ref_adjust.grad(z64, d_in, **a)
    assert (np.abs(got - want) <= (2.0 ** -24 + (2.0 ** -8 if dtype == torch.bfloat16 else 0)) * np.abs(want)).all()
