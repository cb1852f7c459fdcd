"""4-bit weights with group scales against their definition in 64 bits: quantising, reading back, the product.

Tolerances.  Quantising and reading back are exact (a value is a product of 8 and 4 bits).  A product's error, relative
to A = sum |x| |W| of the element: activations of 22 bits (fp32) or exact (bf16), 2^-22; the 128 products of a stage in
8 steps of the tensor core, each of which cuts sums and products to no fewer than 22 bits of the largest, 8 * 2^-21; the
fp32 sums of the stages, (stages + 1) 2^-24; a bf16 result's own half step, 2^-8 of the value.
"""
import numpy as np
import pytest
import torch

from oracle import q4

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def sats():
    import __graft_entry__
    __graft_entry__.build()
    from paper_2607_08991_gb300 import sats as s
    return s


def weights(K, N, G, seed, spread=0.5):
    """(q, scales float64 bf16 values): all codes occur, scales of both signs and some zero."""
    g = np.random.default_rng(seed)
    q = g.integers(-8, 8, (K, N))
    s = np.exp(spread * g.normal(size=((K + G - 1) // G, N))) * 0.05 * np.where(g.random(((K + G - 1) // G, N)) < 0.1, -1, 1)
    s[g.random(s.shape) < 0.02] = 0.0
    return q, q4.bf16(s)


def to_bf16(a):
    return torch.from_numpy(np.asarray(a)).to(torch.bfloat16).cuda()


def activations(B, K, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(B, K, generator=g, dtype=torch.float64) * torch.exp(0.7 * torch.randn(1, K, generator=g, dtype=torch.float64))
    return x.to(dtype).cuda()


def product(sats, q, s, G, x, y_dtype, pad=0):
    codes, scales = torch.from_numpy(q4.pack(q)).cuda(), to_bf16(s)
    w = sats.Q4(codes, scales, G)
    ws = sats.Q4Workspace(w, x.shape[0])
    buf = torch.full((x.shape[0], w.N + pad), 7.0, dtype=y_dtype, device="cuda")
    y = buf[:, : w.N]
    sats.q4_matmul(w, x, y, ws)
    assert sats.get_error(ws) == sats.OK
    assert pad == 0 or (buf[:, w.N:] == 7.0).all()
    return y, (w, ws, buf)


def check(y, x, q, s, G):
    W = q4.values(q, s, G)
    x64 = x.double().cpu().numpy()
    ref, A = x64 @ W, np.abs(x64) @ np.abs(W)
    K = W.shape[0]
    tol = A * (2.0 ** -22 + 8 * 2.0 ** -21 + ((K + 127) // 128 + 1) * 2.0 ** -24)
    if y.dtype == torch.bfloat16:
        tol = tol + np.abs(ref) * 2.0 ** -8 + 2.0 ** -133
    err = np.abs(y.double().cpu().numpy() - ref)
    assert np.isfinite(err).all()
    assert (err <= tol + 2.0 ** -149).all(), float((err / (tol + 1e-300)).max())


SHAPES = [(1, 8, 1, 32), (1, 128, 128, 32), (2, 40, 129, 64), (1, 512, 1408, 32), (3, 1000, 300, 128), (5, 136, 127, 64),
          (8, 4096, 257, 64), (9, 1024, 640, 32), (16, 14336, 130, 128), (17, 264, 1000, 64), (32, 640, 128, 32),
          (33, 384, 513, 128), (64, 2048, 300, 64), (65, 520, 200, 32), (128, 256, 129, 64), (129, 1032, 400, 128),
          (300, 776, 1300, 64)]


@pytest.mark.parametrize("B,K,N,G", SHAPES)
@pytest.mark.parametrize("x_dtype,y_dtype", [(torch.bfloat16, torch.float32), (torch.float32, torch.float32),
                                             (torch.float32, torch.bfloat16)])
def test_product(sats, B, K, N, G, x_dtype, y_dtype):
    q, s = weights(K, N, G, 11 * B + K + N)
    x = activations(B, K, x_dtype, B + N)
    y, _ = product(sats, q, s, G, x, y_dtype, pad=N % 3)
    check(y, x, q, s, G)


@pytest.mark.parametrize("B,N", [(1, 40000), (4, 130000), (200, 20000), (1000, 5000)])
def test_many_columns(sats, B, N):
    """More tiles than CTAs: shares that begin and end inside tiles, and whole ones."""
    K, G = 384, 64
    q, s = weights(K, N, G, N)
    x = activations(B, K, torch.bfloat16, N)
    y, _ = product(sats, q, s, G, x, torch.float32)
    check(y, x, q, s, G)


@pytest.mark.parametrize("B,K,N,G,x_dtype", [(1000, 384, 4400, 64, torch.bfloat16), (1000, 200, 4600, 32, torch.bfloat16),
                                             (513, 520, 4001, 128, torch.float32), (2000, 256, 9000, 64, torch.bfloat16),
                                             (1025, 4096, 4097, 64, torch.float32)])
def test_many_tokens(sats, B, K, N, G, x_dtype):
    """bf16 results whose sums stay in the tensor cores' accumulators for all of K: K / 16 steps, each of which cuts no more than
    2^-21 of the largest (check() allows 8 of them); against 64 bits on the GPU."""
    q, s = weights(K, N, G, B + N)
    x = activations(B, K, x_dtype, B)
    y, _ = product(sats, q, s, G, x, torch.bfloat16, pad=1)
    W = torch.from_numpy(q4.values(q, s, G)).cuda()
    x64 = x.double()
    ref, A = x64 @ W, x64.abs() @ W.abs()
    tol = A * (2.0 ** -22 + (K // 16 + 1) * 2.0 ** -21) + ref.abs() * 2.0 ** -8 + 2.0 ** -133
    err = (y.double() - ref).abs()
    assert (err <= tol).all(), float((err / tol).max())
    # and on the whole no further off than rounding to bf16 puts it (half a step uniformly: 2^-9 / sqrt(3) at most)
    assert float(err.norm() / ref.norm()) <= 2.0 ** -9


def test_one_product_each(sats):
    """Single activations: every weight comes out as it is."""
    K, N, G = 264, 200, 32
    q, s = weights(K, N, G, 5)
    W = q4.values(q, s, G)
    x = torch.eye(K, dtype=torch.bfloat16, device="cuda")
    y, _ = product(sats, q, s, G, x, torch.float32)
    assert np.array_equal(y.double().cpu().numpy(), W)


@pytest.mark.parametrize("x_dtype", [torch.bfloat16, torch.float32])
def test_far_values(sats, x_dtype):
    """Tokens of very different size beside one another, zero tokens, outliers, scales far apart."""
    K, N, G = 512, 150, 32
    q, s = weights(K, N, G, 6, spread=2.0)
    s[:, 3] = q4.bf16(s[:, 3] * 2.0 ** -100)
    s[:, 4] = q4.bf16(s[:, 4] * 2.0 ** 100)
    s[:, 5] = 0.0
    s[1, 6] = q4.bf16(s[1, 6] * 2.0 ** -12)
    x = activations(12, K, x_dtype, 7)
    x[1] *= 2.0 ** -90
    x[2] *= 2.0 ** 20
    x[3] = 0
    x[4, 7] *= 2.0 ** 15
    x[5] = 0
    x[5, 9] = 2.0 ** -126
    y, _ = product(sats, q, s, G, x, torch.float32)
    W = q4.values(q, s, G)
    x64 = x.double().cpu().numpy()
    ref, A = x64 @ W, np.abs(x64) @ np.abs(W)
    # what fp32 does not hold, and the absolute steps of small activations beside an outlier (see the header)
    fine = (A < 2.0 ** 126)
    top = np.abs(x64).max(axis=1, keepdims=True) * np.abs(W).sum(axis=0)
    tol = A * (2.0 ** -22 + 8 * 2.0 ** -21 + 6 * 2.0 ** -24) + top * 2.0 ** -38 + 2.0 ** -148
    got = y.double().cpu().numpy()
    assert (np.abs(got - ref)[fine] <= tol[fine]).all()


def test_not_finite(sats):
    """An infinity or NaN in a token or a column's scales stays with it."""
    K, N, G = 256, 140, 64
    q, s = weights(K, N, G, 8)
    q[q == 0] = 1
    s[s == 0] = 0.05
    x = activations(6, K, torch.float32, 9)
    clean, _ = product(sats, q, s, G, x, torch.float32)
    bad = x.clone()
    bad[1, 5] = float("nan")
    bad[2, 6] = float("inf")
    s2 = s.copy()
    s2[1, 17], s2[2, 18] = np.nan, np.inf
    y, _ = product(sats, q, s2, G, bad, torch.float32)
    assert y[:, 17].isnan().all() and y[:, 18].isnan().all()
    keep = [c for c in range(N) if c not in (17, 18)]
    assert y[1].isnan().all()
    W6 = torch.from_numpy(q4.values(q, s, G)[6]).cuda()
    assert torch.equal(y[2, keep], (float("inf") * W6[keep]).float())
    for b in (0, 3, 4, 5):
        assert torch.equal(y[b, keep], clean[b, keep])


@pytest.mark.parametrize("B,K,N", [(1, 4096, 300), (3, 14336, 512), (40, 2048, 700), (130, 512, 1000)])
def test_again_and_in_a_graph(sats, B, K, N):
    """The same bits every time; a captured call takes what its buffers hold at the replay."""
    G = 64
    q, s = weights(K, N, G, 10)
    x = activations(B, K, torch.float32, 11)
    y, (w, ws, _) = product(sats, q, s, G, x, torch.float32)
    first = y.clone()
    for _ in range(5):
        y.zero_()
        sats.q4_matmul(w, x, y, ws)
        assert torch.equal(y, first)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        sats.q4_matmul(w, x, y, ws)
        sats.q4_matmul(w, x, y, ws)
    x.mul_(0.5)
    y.zero_()
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(y, first * 0.5)
    assert sats.get_error(ws) == sats.OK


def test_two_streams(sats):
    K, N, G = 1024, 3000, 64
    q, s = weights(K, N, G, 12)
    x = [activations(4, K, torch.float32, 13 + i) for i in range(2)]
    kept = [product(sats, q, s, G, x[i], torch.float32) for i in range(2)]
    want = [k[0].clone() for k in kept]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(20):
        for i, st in enumerate(streams):
            w, ws, _ = kept[i][1]
            sats.q4_matmul(w, x[i], kept[i][0], ws, stream=st)
    torch.cuda.synchronize()
    for i in range(2):
        assert torch.equal(kept[i][0], want[i])


def test_unaligned_activations_and_no_tokens(sats):
    K, N, G = 200, 70, 32
    q, s = weights(K, N, G, 14)
    for dtype in (torch.bfloat16, torch.float32):
        x = activations(3, K, dtype, 15)
        off = torch.empty(3 * K + 1, dtype=dtype, device="cuda")[1:].view(3, K)
        off.copy_(x)
        y, (w, ws, _) = product(sats, q, s, G, off, torch.float32)
        check(y, x, q, s, G)
        sats.q4_matmul(w, x[:0], y[:0], ws)


def test_one_workspace_for_all_batches(sats):
    """A workspace of the largest batch serves smaller ones and other weights in any order."""
    made = []
    for K, N, G, seed in ((2048, 700, 64, 20), (512, 5000, 32, 21)):
        q, s = weights(K, N, G, seed)
        made.append((q, s, G, sats.Q4(torch.from_numpy(q4.pack(q)).cuda(), to_bf16(s), G)))
    big = max((sats.Q4Workspace(w[3], 300) for w in made), key=lambda ws: ws.nbytes)
    for turn, (B, which) in enumerate([(300, 0), (1, 0), (40, 1), (3, 1), (300, 1), (17, 0), (70, 0), (1, 1), (200, 1), (5, 0)] * 2):
        q, s, G, w = made[which]
        x = activations(B, w.K, torch.float32 if turn % 3 else torch.bfloat16, turn)
        y = torch.full((B, w.N), float("nan"), device="cuda")
        sats.q4_matmul(w, x, y, big)
        check(y, x, q, s, G)
    assert sats.get_error(big) == sats.OK


def test_workspace_too_small(sats):
    q, s = weights(64, 40, 32, 16)
    w = sats.Q4(torch.from_numpy(q4.pack(q)).cuda(), to_bf16(s), 32)
    ws = sats.Q4Workspace(w, 1)
    with pytest.raises(sats.SatsError) as e:
        sats.q4_matmul(w, activations(200, 64, torch.float32, 1), torch.empty(200, 40, device="cuda"), ws)
    assert e.value.status == sats.ENOSPACE
    with pytest.raises(sats.SatsError) as e:
        n = ws.nbytes
        sats._check(sats.lib().sats_q4_matmul(w.handle, 0x1000, 1, 0x2000, 40, 1, ws.buf.data_ptr() + 16, n - 16, None), "x")
    assert e.value.status == sats.EINVAL
    for x, y in ((torch.zeros(1, 63, device="cuda"), torch.zeros(1, 40, device="cuda")),
                 (torch.zeros(1, 64, device="cuda"), torch.zeros(1, 41, device="cuda")),
                 (torch.zeros(1, 64, dtype=torch.float64, device="cuda"), torch.zeros(1, 40, device="cuda")),
                 (torch.zeros(2, 64, device="cuda"), torch.zeros(1, 40, device="cuda"))):
        with pytest.raises(ValueError):
            sats.q4_matmul(w, x, y, ws)


# ---------------------------------------------------------------------- quantising
def matrix(K, N, seed):
    """bf16 weights with exact ties (ratios of whole numbers), zero groups, subnormal and large ones."""
    g = np.random.default_rng(seed)
    W = g.normal(size=(K, N))
    W[:, N // 3:] = g.integers(-14, 15, (K, N - N // 3)) / 2.0      # amax 7: steps of 1, ties at the halves
    W = q4.bf16(W)
    W[:, -1] *= 2.0 ** -120
    W[:, -1] = q4.bf16(W[:, -1])
    W[:, 0] = 0.0
    return W


@pytest.mark.parametrize("K,N,G,pad", [(8, 1, 32, 0), (40, 3, 32, 5), (128, 257, 64, 0), (1000, 130, 128, 1), (520, 1000, 32, 24),
                                       (256, 4096, 64, 64)])
def test_quantize(sats, K, N, G, pad):
    W = matrix(K, N, K + N)
    buf = torch.full((K, N + pad), float("nan"), dtype=torch.bfloat16, device="cuda")
    buf[:, :N] = torch.from_numpy(W).cuda()
    codes = torch.empty(K // 2, N, dtype=torch.uint8, device="cuda")
    scales = torch.empty((K + G - 1) // G, N, dtype=torch.bfloat16, device="cuda")
    values = torch.empty(K, N, device="cuda")
    sats.q4_quantize(buf[:, :N], codes, scales, G)
    sats.q4_dequantize(codes, scales, G, values)
    q, s = q4.quantize(W, G)
    assert np.array_equal(scales.double().cpu().numpy(), s)
    assert np.array_equal(q4.unpack(codes.cpu().numpy()), q)
    assert np.array_equal(values.double().cpu().numpy(), q4.values(q, s, G))


def test_quantize_extremes(sats):
    """Subnormal groups, the largest values, infinities and NaN."""
    K, G = 64, 32
    W = np.zeros((K, 8))
    W[:32, 0] = 2.0 ** -133 * np.arange(-16, 16)
    W[:32, 1] = 2.0 ** -126 * np.arange(-16, 16) / 16
    W[:32, 2] = 2.0 ** 127 * (1 + 127 / 128) * np.sign(np.arange(-16, 16))
    W[3, 3], W[35, 4], W[:, 5] = np.inf, np.nan, 1.0
    W[5, 6] = 2.0 ** -133
    t = to_bf16(W)
    codes = torch.empty(K // 2, 8, dtype=torch.uint8, device="cuda")
    scales = torch.empty(2, 8, dtype=torch.bfloat16, device="cuda")
    sats.q4_quantize(t, codes, scales, G)
    q, s = q4.quantize(W, G)
    assert np.array_equal(scales.double().cpu().numpy(), s, equal_nan=True)
    assert np.array_equal(q4.unpack(codes.cpu().numpy()), q)


def test_all_codes_read_back(sats):
    codes = torch.arange(256, dtype=torch.uint8, device="cuda").repeat(16, 1).contiguous()
    scales = to_bf16(q4.bf16(np.random.default_rng(3).normal(size=(1, 256))))
    values = torch.empty(32, 256, device="cuda")
    sats.q4_dequantize(codes, scales, 32, values)
    ref = q4.values(q4.unpack(codes.cpu().numpy()), scales.double().cpu().numpy(), 32)
    assert np.array_equal(values.double().cpu().numpy(), ref)
