"""Every kernel of the 4-bit product, with whole and with divided tiles, at the sizes that choose it (152 SMs); quantising where one side
is aligned and the other is not.

Tolerance: as test_gpu_q4.check, against 64 bits on the GPU.  What a case is for stands beside it: direct (the product's CTAs stage the
activations) or staged, columns of a tile, whole tiles or stages divided among CTAs.
"""
import numpy as np
import pytest
import torch

from oracle import q4
from tests.test_gpu_q4 import sats  # noqa: F401

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


def made(K, N, G, seed):
    """codes, scales, W in 64 bits, made on the GPU."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    codes = torch.randint(0, 256, (K // 2, N), generator=g, device="cuda", dtype=torch.int16).to(torch.uint8)
    s = torch.exp(0.5 * torch.randn((K + G - 1) // G, N, generator=g, device="cuda")) * 0.05
    s = (s * torch.where(torch.rand(s.shape, generator=g, device="cuda") < 0.1, -1.0, 1.0)).to(BF)
    q = torch.stack((codes & 15, codes >> 4), 1).view(K, N).double()
    W = torch.where(q > 7, q - 16, q) * s.double().repeat_interleave(G, 0)[:K]
    return codes, s, W


def held(y, x, W):
    """y against x W."""
    x64 = x.double()
    ref, A = x64 @ W, x64.abs() @ W.abs()
    tol = A * (2.0 ** -22 + 8 * 2.0 ** -21 + ((W.shape[0] + 127) // 128 + 1) * 2.0 ** -24)
    if y.dtype == BF:
        tol = tol + ref.abs() * 2.0 ** -8 + 2.0 ** -133
    err = (y.double() - ref).abs()
    assert (err <= tol).all(), float((err / tol).max())


# What a workspace holds behind its counters (256 bytes and 2 * 16 * 320 of them) is scratch: whatever earlier calls of other
# sizes left there, a call must not see it.
SCRATCH = 256 + 2 * 16 * 320 * 4


def scribble(ws, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    part = ws.buf[SCRATCH:SCRATCH + (ws.nbytes - SCRATCH) // 4 * 4].view(torch.int32)
    part.copy_(torch.randint(-2 ** 31, 2 ** 31 - 1, part.shape, generator=g, device="cuda", dtype=torch.int32))


def same(got, want):
    if not torch.equal(got, want):
        rows, cols = torch.nonzero(got != want, as_tuple=True)
        raise AssertionError("%d differ: rows %d..%d, columns %d..%d, largest %g" % (
            rows.numel(), rows.min(), rows.max(), cols.min(), cols.max(), float((got - want).abs().max())))


CASES = [
    (1, 8192, 38912, 64, F32),      # staged 8, whole
    (1, 8192, 128256, 128, F32),    # .. divided, a head
    (8, 8192, 40000, 32, BF),
    (7, 8192, 20000, 32, BF),       # direct 8, divided
    (4, 12296, 9000, 64, F32),      # .. K that ends inside a stage
    (16, 4096, 38912, 32, BF),      # staged 16, whole
    (8, 4096, 128256, 64, F32),     # .. divided, a head
    (16, 4096, 128256, 64, BF),
    (6, 14336, 7001, 128, F32),
    (13, 16384, 5000, 32, BF),      # direct 16, divided
    (20, 14336, 1000, 64, BF),      # staged 32, divided; more of a token than a CTA's registers hold
    (16, 14336, 1300, 32, F32),
    (31, 9000, 12000, 128, BF),
    (64, 14336, 4096, 64, BF),      # staged 64, divided
    (32, 14336, 4096, 128, F32),
    (50, 16392, 1000, 32, BF),
    (128, 9000, 700, 64, BF),       # staged 128, divided: two warpgroups to a tile's exchange
    (64, 9000, 700, 32, F32),
    (256, 14336, 4096, 64, BF),     # .. two tiles of tokens
    (200, 14336, 4095, 128, F32),   # staged 128, whole
    (3, 65536, 300, 64, F32),       # the longest K: direct 8,
    (8, 65536, 200, 32, BF),
    (12, 65536, 30000, 128, BF),    # staged 16,
    (40, 65536, 300, 128, BF),      # 64,
    (100, 65536, 260, 64, F32),     # 128
]


@pytest.mark.parametrize("B,K,N,G,x_dtype", CASES)
def test_variant(sats, B, K, N, G, x_dtype):  # noqa: F811
    codes, scales, W = made(K, N, G, B + K + N)
    g = torch.Generator(device="cuda").manual_seed(N)
    x = (torch.randn(B, K, generator=g, device="cuda") * torch.exp(0.7 * torch.randn(1, K, generator=g, device="cuda"))).to(x_dtype)
    w = sats.Q4(codes, scales, G)
    ws = sats.Q4Workspace(w, B)
    first = None
    for turn in range(20):                                  # the counters are left as they were, the rest may hold anything
        scribble(ws, turn)
        y = torch.full((B, N + 1), 7.0, device="cuda")[:, :N]
        sats.q4_matmul(w, x, y, ws)
        if first is None:
            first = y.clone()
            held(first, x, W)
        same(y, first)
    half = torch.full((B, N), 7.0, dtype=BF, device="cuda")
    scribble(ws, 30)
    sats.q4_matmul(w, x, half, ws)
    held(half, x, W)
    sats.q4_matmul(w, x[:1], half[:1], ws)                  # .. also to another variant
    held(half[:1], x[:1], W)
    sats.q4_matmul(w, x, y, ws)
    same(y, first)
    assert sats.get_error(ws) == sats.OK


@pytest.mark.parametrize("B,K,N,x_dtype,y_dtype", [(256, 14336, 4096, BF, F32), (100, 4096, 14336, F32, F32), (2048, 1024, 4096, BF, F32),
                                                   (128, 2048, 2000, BF, BF), (1000, 2048, 5000, BF, BF), (60, 14336, 4096, BF, F32),
                                                   (19, 2048, 40003, BF, F32), (14, 4096, 20000, BF, F32), (1, 4096, 40000, F32, F32),
                                                   (3, 14336, 4096, F32, F32)])
def test_the_same_bits_a_thousand_times(sats, B, K, N, x_dtype, y_dtype):  # noqa: F811
    """Waits that are right only as long as loads arrive in their order would show in one call of some hundreds."""
    codes, scales, W = made(K, N, 64, B)
    g = torch.Generator(device="cuda").manual_seed(B)
    x = torch.randn(B, K, generator=g, device="cuda").to(x_dtype)
    w = sats.Q4(codes, scales, 64)
    ws = sats.Q4Workspace(w, B)
    y, first = (torch.empty(B, N, dtype=y_dtype, device="cuda") for _ in range(2))
    sats.q4_matmul(w, x, first, ws)
    held(first, x, W)
    other = torch.zeros((), dtype=torch.int64, device="cuda")
    flush = torch.empty(1 << 27, dtype=torch.int16, device="cuda")
    for turn in range(1000):
        if turn % 20 == 0:
            flush.fill_(turn)                               # weights and activations from memory, not from the L2
        sats.q4_matmul(w, x, y, ws)
        other += (y != first).any()
    assert other.item() == 0
    assert sats.get_error(ws) == sats.OK


@pytest.mark.parametrize("B,K,N,x_dtype", [(64, 14336, 4096, BF), (128, 9000, 700, F32), (13, 16384, 5000, BF)])
def test_divided_tiles_in_a_graph(sats, B, K, N, x_dtype):  # noqa: F811
    """Captured calls, replayed on other activations, beside another stream's with a workspace of its own."""
    codes, scales, W = made(K, N, 64, 3 * B)
    w = sats.Q4(codes, scales, 64)
    g = torch.Generator(device="cuda").manual_seed(K)
    xs = [torch.randn(B, K, generator=g, device="cuda").to(x_dtype) for _ in range(2)]
    ws = [sats.Q4Workspace(w, B) for _ in range(2)]
    ys = [torch.empty(B, N, device="cuda") for _ in range(2)]
    want = []
    for x, y, s in zip(xs, ys, ws):
        sats.q4_matmul(w, x, y, s)
        held(y, x, W)
        want.append(y.clone())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        sats.q4_matmul(w, xs[0], ys[0], ws[0])
        sats.q4_matmul(w, xs[0], ys[0], ws[0])
    side = torch.cuda.Stream()
    for turn in range(5):
        ys[0].zero_()
        ys[1].zero_()
        torch.cuda.synchronize()
        graph.replay()
        with torch.cuda.stream(side):
            sats.q4_matmul(w, xs[1], ys[1], ws[1])
        torch.cuda.synchronize()
        same(ys[0], want[0])
        same(ys[1], want[1])
    xs[0].mul_(0.5)
    graph.replay()
    torch.cuda.synchronize()
    same(ys[0], want[0] * 0.5)
    assert sats.get_error(ws[0]) == sats.OK and sats.get_error(ws[1]) == sats.OK


@pytest.mark.parametrize("K,N,ld,G", [(256, 1001, 1004, 32),     # vectors in, bytes out
                                      (256, 1000, 1001, 64),     # elements in, vectors out
                                      (264, 1003, 1003, 128), (1024, 5002, 5004, 128), (128, 130, 132, 32)])
def test_quantising_with_one_side_aligned(sats, K, N, ld, G):  # noqa: F811
    g = np.random.default_rng(K + N)
    W = g.normal(size=(K, N))
    W[:, N // 2:] = g.integers(-14, 15, (K, N - N // 2)) / 2.0
    W = q4.bf16(W)
    W[:40, 5], W[:, 140 % N], W[3, 7] = 0.0, q4.bf16(W[:, 140 % N] * 2.0 ** -130), np.inf
    buf = torch.full((K, ld), float("nan"), dtype=BF, device="cuda")
    buf[:, :N] = torch.from_numpy(W).cuda()
    codes = torch.full((K // 2 * N + 64,), 0x5a, dtype=torch.uint8, device="cuda")
    scales = torch.full(((K + G - 1) // G * N + 64,), 7.0, dtype=BF, device="cuda")
    values = torch.empty(K, N, device="cuda")
    c, s = codes[:K // 2 * N].view(K // 2, N), scales[:(K + G - 1) // G * N].view(-1, N)
    sats.q4_quantize(buf[:, :N], c, s, G)
    sats.q4_dequantize(c, s, G, values)
    q_ref, s_ref = q4.quantize(W, G)
    assert np.array_equal(s.double().cpu().numpy(), s_ref, equal_nan=True)
    assert np.array_equal(q4.unpack(c.cpu().numpy()), q_ref)
    assert np.array_equal(values.double().cpu().numpy(), q4.values(q_ref, s_ref, G), equal_nan=True)
    assert (codes[K // 2 * N:] == 0x5a).all() and (scales[s.numel():] == 7.0).all()
