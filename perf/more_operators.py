"""The operators between the MLP stack and the sampled token, as cases that can be timed.

What turns a hidden state into the logits that are sampled, and back:

- ``product``: rows of activations times a matrix of 4-bit weights with group scales (the vocabulary head, or any
  projection), from one token to a prompt of thousands;
- ``quantise``: bf16 weights to that form and back to the values they stand for, as a calibration of it looks at them;
- ``adjust``: penalties for repeated tokens, biases and grammar masks on rows of logits, before the next token is drawn;
- ``grad``: the gradient of that with respect to the model's logits, for training through the adjusted ones.

``run`` computes a case in plain torch operations, or with ``own`` set through ``paper_2607_08991_gb300.sats``.
``exact`` evaluates the definitions in 64 bits.
"""
import math

import torch

own = False

LLAMA_H, LLAMA_N, LLAMA_V = 4096, 14336, 128256
QWEN_V = 151936
MOST_FLOPS = 2 * 2048 * LLAMA_H * LLAMA_N
MOST_WEIGHTS = LLAMA_H * LLAMA_V


# ---------------------------------------------------------------------- the cases
def listed():
    return [
        # one token through the gate of the small layer: the smallest call, latency only
        dict(name="product_1_small", kind="product", B=1, K=512, N=1408, G=32, x="bf16", y="f32"),
        # the vocabulary head of one decode step: the normalised fp32 stream in, bf16 logits out
        dict(name="product_1_head", kind="product", B=1, K=LLAMA_H, N=LLAMA_V, G=64, x="f32", y="bf16"),
        # a down projection for three requests: a long sum with few columns
        dict(name="product_3_down", kind="product", B=3, K=LLAMA_N, N=LLAMA_H, G=128, x="bf16", y="f32"),
        # the head of a busy server, a ragged number of requests and an odd vocabulary
        dict(name="product_19_head", kind="product", B=19, K=2048, N=100003, G=64, x="bf16", y="bf16"),
        # a prompt through the up projection: the largest work
        dict(name="product_2048_up", kind="product", B=2048, K=LLAMA_H, N=LLAMA_N, G=64, x="bf16", y="bf16"),
        # a layer's weights quantised and looked at again
        dict(name="quantise_layer", kind="quantise", K=LLAMA_H, N=LLAMA_N, G=64, pad=0),
        # a head with an odd vocabulary, small groups, a slice of a wider matrix
        dict(name="quantise_odd", kind="quantise", K=1000, N=100003, G=32, pad=61),
        # one chat request: everything it said so far is penalised
        dict(name="adjust_1", kind="adjust", B=1, V=LLAMA_V, x="bf16", L=2000, M=0, masks=0, pad=0),
        # a busy server: settings of each request, biases, a third of the requests under one of few grammars
        dict(name="adjust_256_mixed", kind="adjust", B=256, V=QWEN_V, x="bf16", L=4096, M=100, masks=8, pad=0),
        # fp32 logits of an odd vocabulary in padded rows, long histories
        dict(name="adjust_77_long_f32", kind="adjust", B=77, V=50001, x="f32", L=30000, M=300, masks=77, pad=61),
        # training on a whole answer: row t has seen the tokens before it
        dict(name="grad_1024_sequence", kind="grad", B=1024, V=LLAMA_V, x="bf16", L=1024, masks=4, pad=0, shared=True),
        # gradients of a few steps of different requests, fp32
        dict(name="grad_33_f32", kind="grad", B=33, V=32000, x="f32", L=900, masks=0, pad=7, shared=False),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["product"] * 5 + ["quantise", "adjust", "adjust", "adjust", "grad"])
    if kind in ("product", "quantise"):
        K = max(8, _log(rng, 64, LLAMA_N) // 8 * 8)
        N = min(_log(rng, 64, 152000), MOST_WEIGHTS // K)
        G = rng.choice([32, 64, 128])
        if kind == "quantise":
            N = min(N, 100003 * 1000 // K)
            return dict(kind=kind, K=K, N=N, G=G, pad=rng.choice([0, 0, rng.randint(1, 200)]))
        B = max(1, min(rng.choice([_log(rng, 1, 16), _log(rng, 1, 2048)]), MOST_FLOPS // (2 * K * N)))
        return dict(kind=kind, B=B, K=K, N=N, G=G, x=rng.choice(["bf16", "f32"]), y=rng.choice(["bf16", "f32"]))
    V = _log(rng, 300, 200000)
    x = rng.choice(["bf16", "f32"])
    pad = rng.choice([0, 0, rng.randint(1, 200)])
    L = _log(rng, 1, 16384)
    if kind == "adjust":
        B = min(_log(rng, 1, 256), (256 * QWEN_V if x == "bf16" else 128 * QWEN_V) // V)
        return dict(kind=kind, B=B, V=V, x=x, L=L, M=rng.choice([0, rng.randint(1, 300)]),
                    masks=rng.choice([0, 0, 1, max(1, B // 3), B]), pad=pad)
    B = min(_log(rng, 1, 1024), (1024 * LLAMA_V if x == "bf16" else 512 * LLAMA_V) // V)
    return dict(kind=kind, B=B, V=V, x=x, L=min(L, 4096), masks=rng.choice([0, 0, 1, max(1, B // 3)]), pad=pad,
                shared=rng.random() < 0.5)


# ---------------------------------------------------------------------- inputs
def _gen(seed, *tags):
    g = torch.Generator(device="cuda")
    v = int(seed) & 0x7FFFFFFF
    for t in tags:
        v = (v * 1000003 + int(t) + 17) & 0x7FFFFFFFFFFF
    g.manual_seed(v)
    return g


def _dtype(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


def _weights(K, N, seed, pad=0):
    """bf16 weights of a trained layer: a bell, some columns and some rows stronger than the others."""
    g = _gen(seed, 1)
    row = torch.exp(0.3 * torch.randn(K, 1, generator=g, device="cuda"))
    col = torch.exp(0.3 * torch.randn(1, N + pad, generator=g, device="cuda")) * K ** -0.5
    W = torch.empty(K, N + pad, dtype=torch.bfloat16, device="cuda")
    for k0 in range(0, K, 512):
        k1 = min(K, k0 + 512)
        W[k0:k1] = torch.randn(k1 - k0, N + pad, generator=g, device="cuda") * row[k0:k1] * col
    return W[:, :N]


def _codes(K, N, G, seed):
    """4-bit weights as they are stored: uint8 [K / 2][N], the even row of a pair in the low half of the byte (two's
    complement), and bf16 scales [ceil(K / G)][N]; most codes small, as quantised bells are."""
    g = _gen(seed, 2)
    codes = torch.empty(K // 2, N, dtype=torch.uint8, device="cuda")
    for k0 in range(0, K // 2, 512):
        k1 = min(K // 2, k0 + 512)
        q = (torch.randn(2, k1 - k0, N, generator=g, device="cuda") * 2.6).round_().clamp_(-8, 7).to(torch.int32) & 15
        codes[k0:k1] = (q[0] | (q[1] << 4)).to(torch.uint8)
    scales = torch.exp(0.4 * torch.randn((K + G - 1) // G, N, generator=g, device="cuda")) * (0.4 * K ** -0.5)
    return codes, scales.to(torch.bfloat16)


def _logits(B, V, pad, dtype, seed, tag):
    buf = torch.empty(B, V + pad, device="cuda", dtype=dtype)
    for r0 in range(0, B, 256):
        r1 = min(B, r0 + 256)
        buf[r0:r1] = torch.randn(r1 - r0, V + pad, generator=_gen(seed, tag, r0), device="cuda").mul_(2.5)
    return buf[:, :V]


def _text(rows, L, V, seed):
    """Token ids as text has them: few tokens make up most of it."""
    u = torch.rand(rows, L, generator=_gen(seed, 5), device="cuda")
    rank = torch.exp(u * math.log(V)).to(torch.int64)          # densities fall like 1 / rank
    return ((rank * 2654435761) % V).to(torch.int32)


def _masks(n, V, seed):
    """Bits of the allowed tokens, 32 to a word: a grammar that leaves few tokens, or one that forbids few."""
    W = (V + 31) // 32
    g = _gen(seed, 6)
    words = torch.randint(-2 ** 31, 2 ** 31, (6, n, W), generator=g, device="cuda", dtype=torch.int64).to(torch.int32)
    few = words[0] & words[1] & words[2] & words[3] & words[4]
    most = words[0] | words[1] | words[2] | words[3] | words[5]
    strict = torch.rand(n, 1, generator=g, device="cuda") < 0.5
    return torch.where(strict, few, most).contiguous()


def prepare(case, seed):
    s = dict(case=case)
    g = _gen(seed, 7)
    kind = case["kind"]
    if kind == "product":
        B, K, N = case["B"], case["K"], case["N"]
        s["codes"], s["scales"] = _codes(K, N, case["G"], seed)
        x = torch.randn(B, K, generator=g, device="cuda")
        x *= torch.exp(0.5 * torch.randn(1, K, generator=g, device="cuda"))   # channels differ in strength
        x[:, :: max(8, K // 4)] *= 20.0                                       # and a few are far above the others
        s["x"] = x.to(_dtype(case["x"]))
        s["y"] = torch.empty(B, N, device="cuda", dtype=_dtype(case["y"]))
        if own:
            from paper_2607_08991_gb300 import sats
            s["w"] = sats.Q4(s["codes"], s["scales"], case["G"])
            s["ws"] = sats.Q4Workspace(s["w"], B)
        return s
    if kind == "quantise":
        K, N, G = case["K"], case["N"], case["G"]
        s["W"] = _weights(K, N, seed, case["pad"])
        s["codes"] = torch.empty(K // 2, N, dtype=torch.uint8, device="cuda")
        s["scales"] = torch.empty((K + G - 1) // G, N, dtype=torch.bfloat16, device="cuda")
        s["values"] = torch.empty(K, N, device="cuda")
        return s
    B, V, L = case["B"], case["V"], case["L"]
    dtype = _dtype(case["x"])
    s["logits"] = _logits(B, V, case["pad"], dtype, seed, 3)
    s["out"] = torch.empty(B, V, device="cuda", dtype=dtype)
    s["status"] = torch.zeros(1, dtype=torch.int32, device="cuda")
    rnd = lambda lo, hi: torch.rand(B, generator=g, device="cuda") * (hi - lo) + lo
    off = lambda t, share, value: torch.where(torch.rand(B, generator=g, device="cuda") < share, value, t)
    s["repetition"] = off(rnd(1.0, 1.4), 0.2, 1.0)
    if kind == "grad":
        if case["shared"]:
            s["hist"] = _text(1, L, V, seed).expand(B, L)
            s["hist_len"] = (torch.arange(B, device="cuda") % (L + 1)).to(torch.int32)
        else:
            s["hist"] = _text(B, L, V, seed)
            s["hist_len"] = rnd(0, L + 0.999).to(torch.int32)
        s["dout"] = _logits(B, V, case["pad"], dtype, seed, 4)
    else:
        s["hist"] = _text(B, L, V, seed)
        s["hist_len"] = rnd(L // 4, L + 0.999).to(torch.int32)
        s["n_prompt"] = (s["hist_len"] * rnd(0.0, 0.9)).to(torch.int32)
        s["presence"] = off(rnd(0.0, 1.0), 0.3, 0.0)
        s["frequency"] = off(rnd(0.0, 0.3), 0.3, 0.0)
        s["bias_idx"] = s["bias_val"] = None
        if case["M"]:
            i = torch.randint(0, V, (B, case["M"]), generator=g, device="cuda").sort(dim=1)[0]
            i[:, 1:][i[:, 1:] == i[:, :-1]] = -1                              # each token once; the others are absent
            ban = torch.rand(B, case["M"], generator=g, device="cuda") < 0.3
            s["bias_idx"] = i.to(torch.int32)
            s["bias_val"] = torch.where(ban, -100.0, 4.0 * torch.randn(B, case["M"], generator=g, device="cuda"))
    n = case["masks"]
    s["mask"] = s["mask_row"] = None
    if n:
        s["mask"] = _masks(n, V, seed)
        s["mask_row"] = torch.randint(0, n, (B,), generator=g, device="cuda").to(torch.int32)
        if n < B:                                                             # the others write freely
            s["mask_row"][torch.rand(B, generator=g, device="cuda") < 0.67] = -1
    return s


# ---------------------------------------------------------------------- one pass
def run(state):
    kind = state["case"]["kind"]
    if kind == "product":
        return (_own_product if own else _plain_product)(state)
    if kind == "quantise":
        return (_own_quantise if own else _plain_quantise)(state)
    if kind == "adjust":
        return (_own_adjust if own else _plain_adjust)(state)
    return (_own_grad if own else _plain_grad)(state)


def _own_product(s):
    from paper_2607_08991_gb300 import sats
    sats.q4_matmul(s["w"], s["x"], s["y"], s["ws"])
    return s["y"]


def _own_quantise(s):
    from paper_2607_08991_gb300 import sats
    G = s["case"]["G"]
    sats.q4_quantize(s["W"], s["codes"], s["scales"], G)
    sats.q4_dequantize(s["codes"], s["scales"], G, s["values"])
    return s["values"], s["scales"]


def _own_adjust(s):
    from paper_2607_08991_gb300 import sats
    sats.adjust_logits(s["logits"], s["out"], hist=s["hist"], hist_len=s["hist_len"], n_prompt=s["n_prompt"],
                       repetition=s["repetition"], presence=s["presence"], frequency=s["frequency"],
                       bias_idx=s["bias_idx"], bias_val=s["bias_val"], mask=s["mask"], mask_row=s["mask_row"],
                       dev_status=s["status"])
    return s["out"]


def _own_grad(s):
    from paper_2607_08991_gb300 import sats
    sats.adjust_logits_grad(s["logits"], s["dout"], s["out"], hist=s["hist"], hist_len=s["hist_len"],
                            repetition=s["repetition"], mask=s["mask"], mask_row=s["mask_row"],
                            dev_status=s["status"])
    return s["out"]


def _values(codes, scales, G, dtype):
    """What codes and scales stand for."""
    both = codes.to(torch.int32)
    q = torch.stack([both & 15, both >> 4], dim=1).reshape(-1, codes.shape[1])
    q = torch.where(q >= 8, q - 16, q)
    return q.to(dtype) * scales.to(dtype).repeat_interleave(G, dim=0)[: q.shape[0]]


def _plain_product(s):
    x, N = s["x"].float(), s["case"]["N"]
    for n0 in range(0, N, 16384):
        cut = slice(n0, min(N, n0 + 16384))
        s["y"][:, cut] = x @ _values(s["codes"][:, cut], s["scales"][:, cut], s["case"]["G"], torch.float32)
    return s["y"]


def _plain_quantise(s):
    G = s["case"]["G"]
    K, N = s["W"].shape
    W = torch.zeros((K + G - 1) // G * G, N, device="cuda")
    W[:K] = s["W"]
    W = W.view(-1, G, N)
    scale = (W.abs().amax(dim=1) / 7).to(torch.bfloat16)
    q = W / scale.float().clamp(min=1e-38)[:, None]
    q = q.round().clamp(-7, 7).view(-1, N)[:K].to(torch.int32) & 15
    codes = (q[0::2] | (q[1::2] << 4)).to(torch.uint8)
    return _values(codes, scale, G, torch.float32), scale


def _plain_allowed(s):
    if s["mask"] is None:
        return None
    V = s["case"]["V"]
    v = torch.arange(V, device="cuda")
    bits = ((s["mask"][:, v >> 5] >> (v & 31)) & 1).bool()
    row = s["mask_row"].long()
    return bits[row.clamp(min=0)] | (row < 0)[:, None]


def _plain_counts(s, first):
    """How often each token stands in each row's history from position `first` on."""
    B, V = s["logits"].shape
    at = torch.arange(s["case"]["L"], device="cuda")[None, :]
    there = (at < s["hist_len"][:, None]) & (at >= first)
    n = torch.zeros(B, V, device="cuda")
    return n.scatter_add_(1, s["hist"].long(), there.float())


def _plain_adjust(s):
    z = s["logits"].float()
    r = s["repetition"][:, None]
    seen = _plain_counts(s, torch.zeros_like(s["n_prompt"])[:, None]) > 0
    count = _plain_counts(s, s["n_prompt"][:, None])
    z = torch.where(seen, torch.where(z > 0, z / r, z * r), z)
    z = z - s["frequency"][:, None] * count - s["presence"][:, None] * (count > 0)
    if s["bias_idx"] is not None:
        here = s["bias_idx"] >= 0
        z.scatter_add_(1, s["bias_idx"].clamp(min=0).long(), torch.where(here, s["bias_val"], 0.0))
    allowed = _plain_allowed(s)
    if allowed is not None:
        z = torch.where(allowed, z, -math.inf)
    return z.to(s["logits"].dtype)


def _plain_grad(s):
    z, d = s["logits"].float(), s["dout"].float()
    r = s["repetition"][:, None]
    seen = _plain_counts(s, torch.zeros_like(s["hist_len"])[:, None]) > 0
    d = torch.where(seen, torch.where(z > 0, d / r, d * r), d)
    allowed = _plain_allowed(s)
    if allowed is not None:
        d = torch.where(allowed, d, 0.0)
    return d.to(s["logits"].dtype)


# ---------------------------------------------------------------------- work
def work(case):
    kind = case["kind"]
    if kind in ("product", "quantise"):
        K, N, G = case["K"], case["N"], case["G"]
        packed = K * N // 2 + 2 * N * ((K + G - 1) // G)
        if kind == "quantise":
            return {"bytes": 2 * K * N + 2 * packed + 4 * K * N, "flops": 4 * K * N}
        B = case["B"]
        es = {"bf16": 2, "f32": 4}
        return {"bytes": packed + B * K * es[case["x"]] + B * N * es[case["y"]], "flops": 2 * B * K * N}
    B, V, L = case["B"], case["V"], case["L"]
    es = 2 if case["x"] == "bf16" else 4
    bits = case["masks"] * V // 8
    if kind == "adjust":
        return {"bytes": 2 * B * V * es + int(0.6 * 4 * B * L) + 8 * B * case["M"] + bits + 24 * B, "flops": B * V}
    ids = 4 * L if case["shared"] else 2 * B * L
    return {"bytes": 2 * B * V * es + ids + bits + 12 * B, "flops": B * V}


# ---------------------------------------------------------------------- 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "product":
        return _exact_product(s)
    if kind == "quantise":
        return _exact_quantise(s)
    return _exact_rows(s)


def _exact_product(s):
    """Group by group: whole-number codes times activations, weighted with the group's scales."""
    c = s["case"]
    K, N, G = c["K"], c["N"], c["G"]
    x = s["x"].double()
    if G * c["B"] < 16384:
        y = torch.zeros(c["B"], N, dtype=torch.float64, device="cuda")
        for k0 in range(0, K, G):
            k1 = min(K, k0 + G)
            b = s["codes"][k0 // 2:k1 // 2].to(torch.int16)
            lo, hi = (b % 16 + 8) % 16 - 8, (b // 16 + 8) % 16 - 8
            y += (x[:, k0:k1:2] @ lo.double() + x[:, k0 + 1:k1:2] @ hi.double()) * s["scales"][k0 // G].double()
        return y
    out = []
    group = torch.arange(K, device="cuda") // G
    for n0 in range(0, N, 4096):
        b = s["codes"][:, n0:n0 + 4096].to(torch.int16)
        w = torch.empty(K, b.shape[1], dtype=torch.float64, device="cuda")
        w[0::2], w[1::2] = (b % 16 + 8) % 16 - 8, (b // 16 + 8) % 16 - 8
        out.append(x @ (w * s["scales"][:, n0:n0 + 4096].double()[group]))
    return torch.cat(out, dim=1)


def _exact_quantise(s):
    G = s["case"]["G"]
    K = s["W"].shape[0]
    values, scales = [], []
    for k0 in range(0, K, G):
        w = s["W"][k0:min(K, k0 + G)].double()
        step = (w.abs().max(dim=0)[0] / 7).to(torch.bfloat16)
        wide = step.double()
        q = torch.round(w / torch.where(wide > 0, wide, torch.ones_like(wide)))
        values.append(torch.minimum(torch.maximum(q, q.new_tensor(-7.0)), q.new_tensor(7.0)) * wide)
        scales.append(step)
    return torch.cat(values), torch.stack(scales).double()


def _exact_rows(s):
    """Row by row, from the tokens that its history names."""
    c = s["case"]
    V = c["V"]
    rows = []
    shift = torch.arange(32, device="cuda", dtype=torch.int64)
    bits = None
    if s["mask"] is not None:
        bits = (((s["mask"].long() & 0xFFFFFFFF)[:, :, None] >> shift) & 1).reshape(c["masks"], -1)[:, :V] == 0
    lens, mrow = s["hist_len"].tolist(), s["mask_row"].tolist() if bits is not None else None
    if c["kind"] == "adjust":
        starts = s["n_prompt"].tolist()
    for b in range(c["B"]):
        z = s["logits"][b].double()
        r = float(s["repetition"][b])
        text = s["hist"][b, :lens[b]].long()
        named = torch.unique(text)
        if c["kind"] == "adjust":
            o = z.clone()
            o[named] = torch.where(z[named] > 0, z[named] / r, z[named] * r)
            made, times = torch.unique(text[starts[b]:], return_counts=True)
            o[made] -= float(s["frequency"][b]) * times.double() + float(s["presence"][b])
            if s["bias_idx"] is not None:
                i = s["bias_idx"][b]
                o[i[i >= 0].long()] += s["bias_val"][b][i >= 0].double()
            banned = -math.inf
        else:
            o = s["dout"][b].double()
            o[named] *= torch.where(z[named] > 0, 1.0 / r, r)
            banned = 0.0
        if bits is not None and mrow[b] >= 0:
            o[bits[mrow[b]]] = banned
        rows.append(o)
    return torch.stack(rows)
