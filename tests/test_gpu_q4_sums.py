"""bf16 results of many tokens are the fp32 results rounded once.

Both kinds of results add 128 products up in the tensor cores and the stages in fp32, in the order of k, where each takes
whole tiles: the same numbers, so no tolerance.  Sums that stayed in the accumulators for all of K would be cut K / 16 times.
"""
import pytest
import torch

from tests.test_gpu_q4 import activations, product, sats, weights  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("x_dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("positive", [False, True])
@pytest.mark.parametrize("B,K,N", [(1024, 4096, 9728), (512, 1000, 9728), (500, 136, 9700), (512, 392, 9601)])
def test_bf16_results_are_the_fp32_ones_rounded(sats, B, K, N, positive, x_dtype):  # noqa: F811
    """Sizes that are whole waves of tiles for both kinds (two columns of activations to an fp32 token)."""
    B = B // 2 if x_dtype == torch.float32 else B
    q, s = weights(K, N, 64, B + K)
    x = activations(B, K, x_dtype, K)
    if positive:
        q, s, x = abs(q), abs(s), x.abs()
    q[q == 8] = 7
    exact, _ = product(sats, q, s, 64, x, torch.float32)
    got, _ = product(sats, q, s, 64, x, torch.bfloat16, pad=N % 2)
    assert torch.equal(got, exact.to(torch.bfloat16))


@pytest.mark.parametrize("spread", [0, 60])
def test_far_powers_of_two(sats, spread):  # noqa: F811
    """Columns and tokens of very different size: results from subnormal ones to those past bf16's range."""
    B, K, N = 512, 264, 9728
    q, s = weights(K, N, 64, 5)
    g = torch.Generator().manual_seed(6)
    s = s * 2.0 ** torch.randint(-spread, spread + 1, (1, N), generator=g).double().numpy()
    x = activations(B, K, torch.bfloat16, 7) * (2.0 ** torch.randint(-spread, spread + 1, (B, 1), generator=g).float().cuda()).bfloat16()
    exact, _ = product(sats, q, s, 64, x, torch.float32)
    got, _ = product(sats, q, s, 64, x, torch.bfloat16)
    assert torch.equal(got, exact.to(torch.bfloat16))
    if spread:
        assert (exact.abs() < 2.0 ** -100).any() and (exact.abs() > 2.0 ** 100).any()


@pytest.mark.parametrize("x_dtype", [torch.bfloat16, torch.float32])
def test_long_sums(sats, x_dtype):  # noqa: F811
    """The longest K, positive numbers: a result is its own sum of magnitudes, of which the tensor cores cut no more than 2^-21 in
    each of the 8 steps of 128 products, and 512 parts are added up in fp32 (and the activations have 22 bits)."""
    K, N, G = 65536, 4864, 128
    B = 1024 if x_dtype == torch.bfloat16 else 512
    g = torch.Generator(device="cuda").manual_seed(3)
    low, high = (torch.randint(1, 8, (K // 2, N), generator=g, device="cuda", dtype=torch.uint8) for _ in range(2))
    codes = low | high << 4
    scales = (torch.rand(K // G, N, generator=g, device="cuda") + 0.5).to(torch.bfloat16)
    x = torch.randn(B, K, generator=g, device="cuda").abs().to(x_dtype)
    w = sats.Q4(codes, scales, G)
    ws = sats.Q4Workspace(w, B)
    exact, got = torch.empty(B, N, device="cuda"), torch.empty(B, N, dtype=torch.bfloat16, device="cuda")
    sats.q4_matmul(w, x, exact, ws)
    sats.q4_matmul(w, x, got, ws)
    assert sats.get_error(ws) == sats.OK
    assert torch.equal(got, exact.to(torch.bfloat16))
    cols = torch.arange(0, N, 97, device="cuda")
    W = torch.stack((low[:, cols], high[:, cols]), 1).view(K, -1).double() * scales[:, cols].double().repeat_interleave(G, 0)
    ref = x.double() @ W
    assert ((exact[:, cols].double() - ref).abs() <= ref * (2.0 ** -22 + 2.0 ** -18 + 513 * 2.0 ** -24)).all()
