"""Adjusted logits and their gradient against the definition in 64 bits.

Tolerance: the fp32 chain rounds at most five times (quotient or product, frequency times count, two differences, a
sum), each by 2^-24 of a value no larger than the sum S of all terms' magnitudes: 5 * 2^-24 S; a bf16 result is rounded
once more, 2^-8 of the value.
"""
import numpy as np
import pytest
import torch

from oracle import adjust as ref

pytestmark = pytest.mark.gpu
DTYPES = [torch.float32, torch.bfloat16]


@pytest.fixture(scope="module")
def sats():
    import __graft_entry__
    __graft_entry__.build()
    from paper_2607_08991_gb300 import sats as s
    return s


def rows(B, V, dtype, seed, pad=0, first=0):
    g = torch.Generator().manual_seed(seed)
    z = (torch.randn(B, V, generator=g) * 3).to(dtype).cuda()
    buf = torch.full((B * (V + pad) + first,), 99.0, dtype=dtype, device="cuda")[first:].view(B, V + pad)
    buf[:, :V] = z
    return buf[:, :V]


def case(B, V, L, seed, M=0, masks=0, share=0.3):
    """Arguments as numpy: histories with repetitions and absent ids, settings on and off."""
    g = np.random.default_rng(seed)
    few = g.integers(0, V, max(1, L // 3))
    hist = np.where(g.random((B, L)) < 0.7, few[g.integers(0, few.size, (B, L))], g.integers(0, V, (B, L)))
    hist[g.random((B, L)) < 0.05] = -1
    a = dict(hist=hist.astype(np.int32), hist_len=g.integers(0, L + 1, B).astype(np.int32))
    a["hist_len"][0] = L
    a["n_prompt"] = (a["hist_len"] * g.random(B)).astype(np.int32)
    on = lambda v, off: np.where(g.random(B) < 0.8, v, off).astype(np.float32)
    a["repetition"] = on(g.uniform(0.5, 1.8, B), 1.0)
    a["presence"], a["frequency"] = on(g.uniform(-1, 1, B), 0.0), on(g.uniform(-0.3, 0.5, B), 0.0)
    if M:
        a["bias_idx"] = g.integers(-1, V, (B, M)).astype(np.int32)
        a["bias_val"] = (g.normal(size=(B, M)) * 5).astype(np.float32)
        a["bias_val"][g.random((B, M)) < 0.1] = -np.inf
    if masks:
        W = (V + 31) // 32
        a["mask"] = g.integers(-2 ** 31, 2 ** 31, (masks, W)).astype(np.int32)
        a["mask"][0] = 0                                      # nothing is allowed
        a["mask_row"] = g.integers(-1, masks, B).astype(np.int32)
        a["mask_row"][-1] = 0
    return a


def on_gpu(a):
    return {k: torch.from_numpy(v).cuda() for k, v in a.items()}


def expected(z, a):
    b = None
    if "bias_idx" in a:
        b = [{int(i): float(v) for i, v in zip(ii, vv) if i >= 0} for ii, vv in zip(a["bias_idx"], a["bias_val"])]
    keep = {k: a[k] for k in a if not k.startswith("bias")}
    return ref.adjust(z, bias=b, **keep)


def close(got, want, z, a, dtype):
    """z: the logits in 64 bits."""
    B, V = z.shape
    r = np.maximum(a.get("repetition", np.ones(B)), 1 / a.get("repetition", np.ones(B)))
    S = np.abs(z) * r[:, None].astype(np.float64)
    L = a["hist"].shape[1] if "hist" in a else 0
    S = S + (np.abs(a.get("presence", np.zeros(B))) + np.abs(a.get("frequency", np.zeros(B))) * L)[:, None]
    if "bias_val" in a:
        S = S + np.abs(np.where(np.isfinite(a["bias_val"]), a["bias_val"], 0)).max(axis=1)[:, None]
    same = np.isneginf(want)
    assert np.array_equal(np.isneginf(got), same)
    tol = 5 * 2.0 ** -24 * S + (2.0 ** -8 * np.abs(np.where(same, 0, want)) if dtype == torch.bfloat16 else 0)
    err = np.abs(np.where(same, 0, got) - np.where(same, 0, want))
    assert np.isfinite(err).all() and (err <= tol).all(), float((err - tol).max())


SHAPES = [(1, 1, 1, 0, 0), (1, 31, 5, 3, 1), (3, 33, 40, 7, 2), (2, 300, 0, 20, 2), (5, 1000, 100, 0, 3), (1, 128256, 2000, 50, 1),
          (7, 5003, 700, 300, 4), (40, 20011, 333, 30, 5), (2, 70001, 40000, 1024, 2), (150, 4099, 64, 5, 150),
          # more rows than are slices at once
          (310, 33, 20, 3, 4), (333, 1000, 300, 17, 9), (320, 4099, 0, 9, 320), (45, 130001, 700, 100, 6),
          (64, 70001, 60000, 5, 2), (305, 515, 17000, 2, 1)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("B,V,L,M,masks", SHAPES)
@pytest.mark.parametrize("place", ["apart", "aligned_alike", "in_place", "between"])
def test_adjust(sats, B, V, L, M, masks, dtype, place):
    a = case(B, V, L, 3 * B + V + L, M, masks)
    args = on_gpu(a)
    if place == "between":
        buf = torch.full((B, 2 * V + 9), 99.0, dtype=dtype, device="cuda")
        z, out = buf[:, :V], buf[:, V + 4:2 * V + 4]
        z.copy_(rows(B, V, dtype, V))
    else:
        z = rows(B, V, dtype, V, pad=3, first=1)
        out = z if place == "in_place" else rows(B, V, dtype, 1, pad=0 if place == "apart" else 3, first=1)
    z64 = z.double().cpu().numpy()
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    sats.adjust_logits(z, out, dev_status=status, **args)
    assert sats.get_status_word(status) == sats.OK
    close(out.double().cpu().numpy(), expected(z64, a), z64, a, dtype)
    if place == "between":
        assert np.array_equal(z.double().cpu().numpy(), z64)
        assert (buf[:, V:V + 4] == 99).all() and (buf[:, 2 * V + 4:] == 99).all()
    elif place != "in_place":
        assert np.array_equal(z.double().cpu().numpy(), z64)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("B,V,L,M,masks", [s for s in SHAPES if s[2] > 0])
@pytest.mark.parametrize("place", ["apart", "dout", "between"])
def test_grad(sats, B, V, L, M, masks, dtype, place):
    a = case(B, V, L, 5 * B + V + L, 0, masks)
    a = {k: a[k] for k in ("hist", "hist_len", "repetition", "mask", "mask_row") if k in a}
    z, d = rows(B, V, dtype, 1, pad=5, first=1), rows(B, V, dtype, 2, pad=0 if place == "apart" else 5, first=1)
    z[:, ::7] = 0.0
    if masks:
        d[-1, 0], d[-1, V // 2] = float("nan"), float("inf")     # where nothing is allowed
    out = {"apart": rows(B, V, dtype, 3, pad=2), "dout": d, "between": None}[place]
    if place == "between":
        buf = torch.full((B, 2 * V + 9), 99.0, dtype=dtype, device="cuda")
        buf[:, V + 4:2 * V + 4] = d
        out, d = buf[:, :V], buf[:, V + 4:2 * V + 4]
    z64, d64 = z.double().cpu().numpy(), d.double().cpu().numpy()
    sats.adjust_logits_grad(z, d, out, **on_gpu(a))
    want = ref.grad(z64, d64, **a)
    got = out.double().cpu().numpy()
    assert np.array_equal(np.isfinite(got), np.isfinite(want))
    tol = np.abs(want) * (2.0 ** -24 + (2.0 ** -8 if dtype == torch.bfloat16 else 0))
    assert (np.abs(got - want) <= tol).all()


def test_grad_by_differences(sats):
    """The gradient of sum(g adjusted) against differences of the call itself (fp32; steps of 2^-6 are exact on values
    below 16 but for two roundings, 2 * 2^-24 * 32 / 2^-6 = 2.5e-4)."""
    B, V, L = 3, 50, 30
    a = case(B, V, L, 77, M=4, masks=3)
    args = on_gpu(a)
    z = torch.round(rows(B, V, torch.float32, 5) * 64) / 64
    z[z == 0] = 1.0
    z = torch.where(z.abs() < 0.25, z + 0.5, z)                # no step crosses 0
    z = z.contiguous()
    d = torch.empty_like(z)
    sats.adjust_logits_grad(z, torch.ones_like(z), d, **{k: args[k] for k in ("hist", "hist_len", "repetition", "mask", "mask_row")})
    h = 2.0 ** -6
    up, down = torch.empty_like(z), torch.empty_like(z)
    sats.adjust_logits(z + h, up, **args)
    sats.adjust_logits(z - h, down, **args)
    slope = (up.double() - down.double()) / (2 * h)
    slope[torch.isneginf(up)] = 0.0
    biased_out = torch.zeros_like(z, dtype=torch.bool)         # a bias of -inf is a constant of the forward alone
    for b in range(B):
        for i, v in zip(a["bias_idx"][b], a["bias_val"][b]):
            if i >= 0:
                biased_out[b, int(i)] = bool(v == -np.inf)
    assert (slope - d.double())[~biased_out].abs().max() <= 2.5e-4


@pytest.mark.parametrize("dtype", DTYPES)
def test_special_logits(sats, dtype):
    """NaN stays, infinities stay, and a banned token is -inf whatever it was."""
    V = 64
    z = rows(1, V, dtype, 4)
    z[0, 0], z[0, 1], z[0, 2], z[0, 3], z[0, 4] = float("nan"), float("inf"), -float("inf"), 0.0, -0.0
    z[0, 32], z[0, 33] = float("nan"), float("inf")
    hist = torch.arange(V, dtype=torch.int32, device="cuda")[None].contiguous()
    mask = torch.tensor([[-1, ~3]], dtype=torch.int32, device="cuda")
    bias_idx = torch.tensor([[5, 6, 6]], dtype=torch.int32, device="cuda")
    bias_val = torch.tensor([[-float("inf"), 3.0, 2.0]], device="cuda")
    v = lambda x: torch.tensor([x], device="cuda")
    out = torch.empty_like(z)
    sats.adjust_logits(z, out, hist=hist, repetition=v(2.0), presence=v(0.5), bias_idx=bias_idx, bias_val=bias_val, mask=mask)
    assert out[0, 0].isnan() and out[0, 1] == float("inf") and out[0, 2] == -float("inf")
    assert out[0, 3] == -0.5 and out[0, 4] == -0.5 and out[0, 5] == -float("inf")
    x = z[0, 6].float()
    assert out[0, 6] == ((x / 2 if x > 0 else x * 2) - 0.5 + 2.0).to(dtype)
    assert out[0, 32] == -float("inf") and out[0, 33] == -float("inf")


def test_settings_outside_their_range(sats):
    """Off, absent or cut, and noted."""
    B, V, L = 8, 100, 10
    z = rows(B, V, torch.float32, 6)
    hist = torch.randint(0, V, (B, L), dtype=torch.int32, device="cuda")
    ones = lambda x: torch.full((B,), x, device="cuda")
    good = dict(hist=hist, repetition=ones(1.5), presence=ones(0.5), frequency=ones(0.25))
    want = torch.empty_like(z)
    sats.adjust_logits(z, want, **good)

    def run(**more):
        out, status = torch.empty_like(z), torch.zeros(1, dtype=torch.int32, device="cuda")
        sats.adjust_logits(z, out, dev_status=status, **{**good, **more})
        assert sats.get_status_word(status) == sats.EDEVICE
        return out

    for bad in (0.0, -1.0, float("nan"), float("inf")):
        r = ones(1.5)
        r[2] = bad
        out = run(repetition=r)
        base = torch.empty_like(z)
        r[2] = 1.0
        sats.adjust_logits(z, base, **{**good, "repetition": r})
        assert torch.equal(out, base)
    for name in ("presence", "frequency"):
        p = good[name].clone()
        p[3] = float("nan")
        out = run(**{name: p})
        p[3] = 0.0
        base = torch.empty_like(z)
        sats.adjust_logits(z, base, **{**good, name: p})
        assert torch.equal(out, base)
    n = torch.full((B,), L, dtype=torch.int32, device="cuda")
    n[1] = L + 1
    assert torch.equal(run(hist_len=n), want)
    n[1] = -1
    assert torch.equal(run(hist_len=n)[1], z[1])
    h = torch.cat([hist, torch.full((B, 1), V, dtype=torch.int32, device="cuda")], dim=1)
    assert torch.equal(run(hist=h), want)
    i = torch.tensor([[5, V]] * B, dtype=torch.int32, device="cuda")
    v = torch.tensor([[float("nan"), 1.0]] * B, device="cuda")
    assert torch.equal(run(bias_idx=i, bias_val=v), want)
    v[:, 0] = float("inf")
    assert torch.equal(run(bias_idx=i, bias_val=v), want)
    m = torch.zeros(1, 4, dtype=torch.int32, device="cuda")
    row = torch.full((B,), -1, dtype=torch.int32, device="cuda")
    row[4] = 1
    assert torch.equal(run(mask=m, mask_row=row), want)


@pytest.mark.parametrize("dtype", DTYPES)
def test_shared_and_overlapping_histories(sats, dtype):
    """Row t has seen the first t ids of one sequence; windows of one sequence."""
    T, V = 37, 257
    g = np.random.default_rng(8)
    seq = g.integers(0, V, 200).astype(np.int32)
    z, out = rows(T, V, dtype, 9), rows(T, V, dtype, 10)
    z64 = z.double().cpu().numpy()
    rep = np.full(T, 1.7, np.float32)
    dev = torch.from_numpy(seq).cuda()
    lens = np.arange(T, dtype=np.int32)
    sats.adjust_logits(z, out, hist=dev[None].expand(T, 200), hist_len=torch.from_numpy(lens).cuda(),
                       repetition=torch.from_numpy(rep).cuda())
    a = dict(hist=np.broadcast_to(seq, (T, 200)), hist_len=lens, repetition=rep)
    close(out.double().cpu().numpy(), expected(z64, a), z64, a, dtype)
    win = dev.as_strided((T, 30), (3, 1))
    sats.adjust_logits(z, out, hist=win, repetition=torch.from_numpy(rep).cuda())
    a = dict(hist=win.cpu().numpy(), repetition=rep)
    close(out.double().cpu().numpy(), expected(z64, a), z64, a, dtype)


def test_far_rows(sats):
    """Rows beyond 2^31 elements, bf16, one of them in place."""
    V, ld = 1000, (1 << 31) + 8
    buf = torch.empty(ld + V, dtype=torch.bfloat16, device="cuda")
    z = buf.as_strided((2, V), (ld, 1))
    z.copy_(rows(2, V, torch.bfloat16, 11))
    a = case(2, V, 50, 12, M=4, masks=2)
    z64 = z.double().cpu().numpy()
    sats.adjust_logits(z, z, **on_gpu(a))
    close(z.double().cpu().numpy(), expected(z64, a), z64, a, torch.bfloat16)


@pytest.mark.parametrize("dtype", DTYPES)
def test_graph_and_streams(sats, dtype):
    """A captured call takes what its buffers hold at the replay; two streams at once; the same bits every time."""
    B, V, L = 20, 30000, 500
    a = on_gpu(case(B, V, L, 13, M=9, masks=3))
    z, out = rows(B, V, dtype, 14), rows(B, V, dtype, 15)
    sats.adjust_logits(z, out, **a)
    first = out.clone()
    st = [torch.cuda.Stream() for _ in range(2)]
    outs = [torch.empty_like(out) for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(10):
        for s, o in zip(st, outs):
            sats.adjust_logits(z, o, **a, stream=s)
    torch.cuda.synchronize()
    assert torch.equal(outs[0], first) and torch.equal(outs[1], first)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        sats.adjust_logits(z, out, **a)
    a["repetition"].fill_(1.0)
    a["presence"].zero_()
    a["frequency"].zero_()
    a["bias_idx"].fill_(-1)
    a["mask_row"].fill_(-1)
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, z)


def test_binding_refusals(sats):
    z = rows(2, 64, torch.float32, 1)
    out = torch.empty_like(z)
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")
    f32 = lambda *s: torch.zeros(s, device="cuda")
    for bad in (dict(hist=i32(1, 4)), dict(hist=f32(2, 4)), dict(hist=i32(2, 8)[:, ::2]), dict(hist=i32(2, 4), hist_len=i32(3)),
                dict(mask=i32(2, 1)), dict(mask=f32(2, 2)), dict(bias_idx=i32(2, 3)), dict(bias_idx=i32(2, 3), bias_val=f32(2, 4)),
                dict(repetition=f32(3)), dict(hist=i32(2, 4).cpu())):
        with pytest.raises(ValueError):
            sats.adjust_logits(z, out, **bad)
    with pytest.raises(ValueError):
        sats.adjust_logits(z, out[:, :63])
    with pytest.raises(ValueError):
        sats.adjust_logits(z, out.to(torch.bfloat16))
    with pytest.raises(sats.SatsError):
        sats.adjust_logits(z, out, mask=i32(1, 2))           # two rows, one mask, no mask_row
