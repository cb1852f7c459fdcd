"""The operators on rows of vocabulary logits, as cases that can be timed.

Three operators that stand on either side of the library's token routing:

- ``top``: the K largest logits of each row with their indices, as a teacher model hands them over;
- ``loss`` / ``grad`` / ``step``: distillation from a teacher's top logits mixed with the next-token
  cross entropy, forward, backward, and both in one pass.  With no teacher entries the forward is the
  per-token loss that the routing calibration takes for its base and sparse paths;
- ``sample``: the next token ids of a batch, by temperature, top-k, top-p and min-p from given random
  numbers; the ids are what the routing table is looked up with.

``run`` computes a case in plain torch operations, or with ``own`` set through
``paper_2607_08991_gb300.sats``.  ``exact`` evaluates the definitions in 64 bits.
"""
import math

import torch

own = False

LLAMA_V = 128256
QWEN_V = 151936


# ---------------------------------------------------------------------- the cases
def listed():
    return [
        # one decode step of one request, the usual chat settings: latency only
        dict(name="sample_1", kind="sample", B=1, V=LLAMA_V, x="bf16", mode="chat", pad=0),
        # a few requests of a small-vocabulary draft model, fp32 logits: the smallest call
        dict(name="sample_4_tiny_f32", kind="sample", B=4, V=1000, x="f32", mode="chat", pad=0),
        # one decode step of a busy server, every request with settings of its own
        dict(name="sample_256_mixed", kind="sample", B=256, V=QWEN_V, x="bf16", mode="mixed", pad=0),
        # nucleus sampling over the whole vocabulary (roll-outs for training), an odd vocabulary in padded rows
        dict(name="sample_300_top_p_f32", kind="sample", B=300, V=100003, x="f32", mode="top_p", pad=61),
        # roll-outs with temperature alone: nothing is cut, every token's mass counts
        dict(name="sample_512_free", kind="sample", B=512, V=LLAMA_V, x="bf16", mode="free", pad=0),
        # alternatives shown beside one generated token
        dict(name="top_1", kind="top", T=1, V=QWEN_V, x="bf16", K=20, pad=0),
        # a teacher's top logits over a long document, written out for a later distillation
        dict(name="top_2048", kind="top", T=2048, V=LLAMA_V, x="bf16", K=64, pad=0),
        # many logits of a ragged number of odd fp32 rows
        dict(name="top_77_many_f32", kind="top", T=77, V=50001, x="f32", K=1000, pad=0),
        # per-token losses of a corpus piece for the routing calibration: no teacher, labels only
        dict(name="loss_8192_labels", kind="loss", T=8192, V=QWEN_V, x="bf16", K=0, tau=1.0, alpha=0.0, pad=0),
        # validation loss of a short prompt against stored teacher logits
        dict(name="loss_37_f32", kind="loss", T=37, V=LLAMA_V, x="f32", K=32, tau=2.0, alpha=0.5, pad=0),
        # backward of that loss for a micro-batch whose upstream gradients come from another program part
        dict(name="grad_1000_f32", kind="grad", T=1000, V=QWEN_V, x="f32", K=50, tau=2.0, alpha=0.7, pad=0),
        # a training step of the adapted sparse model: loss and gradient of 4096 tokens
        dict(name="step_4096", kind="step", T=4096, V=LLAMA_V, x="bf16", K=64, tau=1.0, alpha=0.8, pad=0),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["sample", "sample", "sample", "top", "top", "loss", "grad", "step"])
    V = _log(rng, 300, 200000)
    x = rng.choice(["bf16", "f32"])
    pad = rng.choice([0, 0, rng.randint(1, 200)])
    es = 2 if x == "bf16" else 4
    if kind == "sample":
        return dict(kind=kind, B=min(_log(rng, 1, 512), 512 * LLAMA_V // V), V=V, x=x, pad=pad,
                    mode=rng.choice(["chat", "mixed", "mixed", "top_p", "top_k", "min_p", "free", "greedy"]))
    if kind == "top":
        T = min(_log(rng, 1, 2048), 2048 * LLAMA_V * 2 // (V * es))
        return dict(kind=kind, T=T, V=V, x=x, K=min(_log(rng, 1, 1024), V), pad=pad)
    T = min(_log(rng, 1, 8192), 4096 * LLAMA_V * 2 // (V * es))
    K = rng.choice([0, min(_log(rng, 1, 1024), V), min(_log(rng, 1, 256), V)])
    alpha = 0.0 if K == 0 else rng.choice([1.0, 0.5, round(rng.uniform(0.1, 0.9), 2)])
    return dict(kind=kind, T=T, V=V, x=x, K=K, tau=rng.choice([1.0, 2.0, round(rng.uniform(0.7, 5.0), 2)]),
                alpha=alpha, pad=pad)


# ---------------------------------------------------------------------- inputs
def _gen(seed, *tags):
    g = torch.Generator(device="cuda")
    v = int(seed) & 0x7FFFFFFF
    for t in tags:
        v = (v * 1000003 + int(t) + 17) & 0x7FFFFFFFFFFF
    g.manual_seed(v)
    return g


def _rows(case):
    return case["B"] if case["kind"] == "sample" else case["T"]


def _logits(case, seed):
    """Rows of a language model's logits: a bell of all tokens and in each row a few tokens above it, by an amount
    that goes from nothing (the model does not know) to a lot (one token is certain).  A view of padded rows where
    the case has padding; what lies in the padding is never part of a row."""
    R, V = _rows(case), case["V"]
    dtype = torch.bfloat16 if case["x"] == "bf16" else torch.float32
    buf = torch.empty(R, V + case["pad"], device="cuda", dtype=dtype)
    for r0 in range(0, R, 1024):
        r1 = min(R, r0 + 1024)
        n = r1 - r0
        z = torch.randn(n, V + case["pad"], generator=_gen(seed, 1, r0), device="cuda").mul_(2.2)
        g = _gen(seed, 2, r0)
        few = min(V, 6)
        at = torch.randint(0, V, (n, few), generator=g, device="cuda")
        up = torch.rand(n, 1, generator=g, device="cuda") * 14.0 * torch.rand(n, few, generator=g, device="cuda")
        z.scatter_add_(1, at, up)
        buf[r0:r1] = z
    return buf[:, :V]


def _settings(case, seed):
    """temperature, top_k, top_p, min_p of each request (None: nobody sets it) and the random numbers."""
    B, V, mode = case["B"], case["V"], case["mode"]
    g = _gen(seed, 3)
    rnd = lambda lo, hi: torch.rand(B, generator=g, device="cuda") * (hi - lo) + lo
    u = torch.rand(B, generator=g, device="cuda")
    temp, top_k, top_p, min_p = rnd(0.5, 1.2), None, None, None
    if mode == "chat":
        top_k = torch.full((B,), min(50, V), dtype=torch.int32, device="cuda")
        top_p = torch.full((B,), 0.9, device="cuda")
    elif mode == "top_k":
        top_k = torch.randint(1, min(V, 1000) + 1, (B,), generator=g, device="cuda").to(torch.int32)
    elif mode == "top_p":
        top_p = rnd(0.5, 0.99)
    elif mode == "min_p":
        min_p = rnd(0.01, 0.2)
    elif mode == "greedy":
        temp = torch.zeros(B, device="cuda")
    elif mode == "mixed":
        off = lambda share: torch.rand(B, generator=g, device="cuda") < share
        top_k = torch.randint(1, min(V, 200) + 1, (B,), generator=g, device="cuda").to(torch.int32)
        top_k[off(0.4)] = 0
        top_p = rnd(0.6, 1.0)
        top_p[off(0.4)] = 1.0
        min_p = rnd(0.0, 0.1)
        min_p[off(0.6)] = 0.0
        temp[off(0.1)] = 0.0
    return temp, top_k, top_p, min_p, u


def _teacher(case, seed, logits):
    """K entries of each row: mostly tokens that the student ranks high too, with the teacher's own logits."""
    T, V, K = case["T"], case["V"], case["K"]
    if K == 0:
        return None, None
    idx = torch.empty(T, K, dtype=torch.int32, device="cuda")
    val = torch.empty(T, K, device="cuda")
    for r0 in range(0, T, 1024):
        r1 = min(T, r0 + 1024)
        z = logits[r0:r1].float()
        z = z + torch.randn(z.shape, generator=_gen(seed, 4, r0), device="cuda")
        v, i = torch.topk(z, K, dim=1)
        val[r0:r1], idx[r0:r1] = v, i.to(torch.int32)
    return idx, val


def prepare(case, seed):
    R, V = _rows(case), case["V"]
    z = _logits(case, seed)
    s = dict(case=case, logits=z, status=torch.zeros(1, dtype=torch.int32, device="cuda"))
    f32 = lambda *shape: torch.empty(shape, device="cuda")
    i32 = lambda *shape: torch.empty(shape, dtype=torch.int32, device="cuda")
    if case["kind"] == "sample":
        s["temperature"], s["top_k"], s["top_p"], s["min_p"], s["u"] = _settings(case, seed)
        s.update(ids=i32(R), logprob=f32(R), n_kept=i32(R))
    elif case["kind"] == "top":
        s.update(values=f32(R, case["K"]), idx=i32(R, case["K"]))
    else:
        s["top_idx"], s["top_val"] = _teacher(case, seed, z)
        g = _gen(seed, 5)
        labels = z.argmax(dim=1).to(torch.int32)   # right for half of the tokens, anything for the others
        other = torch.randint(0, V, (R,), generator=g, device="cuda").to(torch.int32)
        coin = torch.rand(R, generator=g, device="cuda")
        labels = torch.where(coin < 0.5, labels, other)
        if R > 1:
            labels[coin > 0.95] = -1               # padding of the batch: ignored rows, of which nothing is read
        s["labels"] = labels
        s["g"] = torch.full((R,), 1.0 / max(1, int((labels >= 0).sum())), device="cuda")
        s.update(loss=f32(R), lse=f32(R, 2))
        if case["kind"] != "loss":
            s["dlogits"] = torch.empty(R, V, device="cuda", dtype=z.dtype)
        if case["kind"] == "grad":
            z32 = z.float()
            s["lse"][:, 0] = torch.logsumexp(z32 / case["tau"], dim=1)
            s["lse"][:, 1] = torch.logsumexp(z32, dim=1)
    return s


# ---------------------------------------------------------------------- one pass
def run(state):
    kind = state["case"]["kind"]
    if kind == "sample":
        return (_own_sample if own else _plain_sample)(state)
    if kind == "top":
        return (_own_top if own else _plain_top)(state)
    return (_own_distill if own else _plain_distill)(state)


def _own_sample(s):
    from paper_2607_08991_gb300 import sats
    sats.sample(s["logits"], s["u"], s["ids"], temperature=s["temperature"], top_k=s["top_k"], top_p=s["top_p"],
                min_p=s["min_p"], logprob=s["logprob"], n_kept=s["n_kept"], dev_status=s["status"])
    return s["ids"], s["logprob"], s["n_kept"]


def _own_top(s):
    from paper_2607_08991_gb300 import sats
    sats.top_logits(s["logits"], s["values"], s["idx"])
    return s["values"], s["idx"]


def _own_distill(s):
    from paper_2607_08991_gb300 import sats
    c = s["case"]
    args = (s["logits"], s["top_idx"], s["top_val"], s["labels"], c["tau"], c["alpha"])
    if c["kind"] == "loss":
        sats.distill_loss(*args, s["loss"], lse=s["lse"], dev_status=s["status"])
        return s["loss"], s["lse"]
    if c["kind"] == "grad":
        sats.distill_grad(*args, s["lse"], s["dlogits"], g=s["g"], dev_status=s["status"])
        return s["dlogits"]
    sats.distill_loss_grad(*args, s["loss"], s["dlogits"], g=s["g"], dev_status=s["status"])
    return s["loss"], s["dlogits"]


def _plain_sample(s):
    """In 64 bits: a drawn number lies next to a border of the cumulated masses once in a while."""
    z = s["logits"].double()
    B, V = z.shape
    T = s["temperature"].double()[:, None]
    greedy = T == 0
    order = torch.sort(s["logits"].float(), dim=1, descending=True, stable=True)[1]
    rank_logit = torch.gather(z, 1, order)
    w = torch.exp((rank_logit - rank_logit[:, :1]) / torch.where(greedy, torch.ones_like(T), T))
    pos = torch.arange(V, device=z.device)[None, :]
    keep = torch.ones(B, V, dtype=torch.bool, device=z.device)
    if s["top_k"] is not None:
        k = s["top_k"].long()[:, None]
        keep &= (k <= 0) | (pos < k)
    keep &= ~greedy | (pos == 0)
    w = w * keep
    if s["top_p"] is not None:
        p = s["top_p"].double()[:, None]
        before = torch.cumsum(w, dim=1) - w
        keep &= (p >= 1) | (before < p * w.sum(dim=1, keepdim=True))
    if s["min_p"] is not None:
        keep &= w >= s["min_p"].double()[:, None]
    w = w * keep
    kept = torch.zeros_like(w).scatter_(1, order, w)       # back in the vocabulary's order
    cum = torch.cumsum(kept, dim=1)
    total = cum[:, -1:]
    hit = cum > s["u"].double()[:, None] * total
    ids = hit.to(torch.uint8).argmax(dim=1)
    logprob = torch.log(torch.gather(kept, 1, ids[:, None]) / total)[:, 0]
    return ids.to(torch.int32), logprob.float(), keep.sum(dim=1).to(torch.int32)


def _plain_top(s):
    K = s["case"]["K"]
    v, i = torch.sort(s["logits"].float(), dim=1, descending=True, stable=True)
    return v[:, :K].contiguous(), i[:, :K].to(torch.int32).contiguous()


def _plain_lse(z):
    m = z.max(dim=1, keepdim=True)[0]
    return m[:, 0] + torch.log(torch.exp(z - m).sum(dim=1))


def _plain_distill(s):
    c = s["case"]
    tau, alpha = c["tau"], c["alpha"]
    z = s["logits"].float()
    live = s["labels"] >= 0
    y = s["labels"].clamp(min=0).long()[:, None]
    if c["kind"] == "grad":
        lse_tau, lse_one = s["lse"][:, 0], s["lse"][:, 1]
    else:
        lse_tau, lse_one = _plain_lse(z / tau), _plain_lse(z)
    q = None
    if c["K"]:
        at = s["top_idx"].long()
        logq = s["top_val"] / tau
        logq = logq - _plain_lse(logq)[:, None]
        q = torch.exp(logq)
    out = []
    if c["kind"] != "grad":
        loss = (1.0 - alpha) * (lse_one - torch.gather(z, 1, y)[:, 0])
        if q is not None:
            logp = torch.gather(z, 1, at) / tau - lse_tau[:, None]
            loss = loss + alpha * tau * tau * (q * (logq - logp)).sum(dim=1)
        out.append(torch.where(live, loss, torch.zeros_like(loss)))
        if c["kind"] == "loss":
            return out[0], torch.where(live[:, None], torch.stack([lse_tau, lse_one], dim=1), 0.0)
    d = (1.0 - alpha) * torch.exp(z - lse_one[:, None])
    d.scatter_add_(1, y, torch.full_like(y, alpha - 1.0, dtype=torch.float32))
    if q is not None:
        d += alpha * tau * torch.exp(z / tau - lse_tau[:, None])
        d.scatter_add_(1, at, -alpha * tau * q)
    d *= torch.where(live, s["g"], torch.zeros_like(s["g"]))[:, None]
    out.append(d.to(s["logits"].dtype))
    return tuple(out) if len(out) > 1 else out[0]


# ---------------------------------------------------------------------- work
def work(case):
    R, V = _rows(case), case["V"]
    es = 2 if case["x"] == "bf16" else 4
    logits = R * V * es
    if case["kind"] == "sample":
        named = {"chat": 3, "mixed": 4, "top_p": 2, "top_k": 2, "min_p": 2, "free": 1, "greedy": 1}[case["mode"]]
        return {"bytes": logits + 4 * R * (named + 1 + 3), "flops": 3 * R * V}
    if case["kind"] == "top":
        return {"bytes": logits + 8 * R * case["K"], "flops": R * V}
    read = logits if R == 1 else 0.95 * logits   # ignored rows need not be read
    exps = (0 < case["alpha"]) + (case["alpha"] < 1 and not (case["alpha"] > 0 and case["tau"] == 1))
    small = R * (8 * case["K"] + 4)
    if case["kind"] == "loss":
        return {"bytes": read + small + 12 * R, "flops": 3 * exps * R * V}
    if case["kind"] == "grad":
        return {"bytes": read + logits + small + 12 * R, "flops": 4 * exps * R * V}
    return {"bytes": read + logits + small + 8 * R, "flops": 6 * exps * R * V}


# ---------------------------------------------------------------------- 64 bits
def exact(case, seed):
    """The definitions row by row in 64 bits: what one row's tokens are worth, sorted, cut and counted."""
    s = prepare(case, seed)
    if case["kind"] == "top":
        return _exact_top(s)
    if case["kind"] == "sample":
        return _exact_sample(s)
    return _exact_distill(s)


def _exact_top(s):
    K = s["case"]["K"]
    values, idx = [], []
    for r0 in range(0, s["logits"].shape[0], 64):
        a = s["logits"][r0:r0 + 64].double()
        o = torch.argsort(-a, dim=1, stable=True)[:, :K]
        idx.append(o.to(torch.int32))
        values.append(torch.gather(a, 1, o))
    return torch.cat(values), torch.cat(idx)


def _exact_sample(s):
    B = s["logits"].shape[0]
    val = lambda name, b, off: off if s[name] is None else float(s[name][b])
    ids, logprobs, counts = [], [], []
    for b in range(B):
        a = s["logits"][b].double()
        T, p, mp = val("temperature", b, 1.0), val("top_p", b, 1.0), val("min_p", b, 0.0)
        k = int(val("top_k", b, 0))
        if T == 0:
            T, k = 1.0, 1
        o = torch.argsort(-a, stable=True)
        n = min(k, a.numel()) if k > 0 else a.numel()
        o = o[:n]
        e = ((a[o] - a[o[0]]) / T).exp()
        if p < 1:
            reach = torch.cumsum(e, 0) >= p * e.sum()
            n = min(n, int(reach.to(torch.uint8).argmax()) + 1)
        if mp > 0:
            n = min(n, int((e >= mp).sum()))
        o, e = o[:n], e[:n]
        inv = torch.argsort(o)
        o, e = o[inv], e[inv]
        c = torch.cumsum(e, 0)
        j = int(torch.searchsorted(c, c[-1:] * float(s["u"][b]), right=True).clamp(max=n - 1))
        ids.append(int(o[j]))
        logprobs.append(float(torch.log(e[j]) - torch.log(c[-1])))
        counts.append(n)
    dev = s["logits"].device
    return (torch.tensor(ids, dtype=torch.int32, device=dev), torch.tensor(logprobs, dtype=torch.float64, device=dev),
            torch.tensor(counts, dtype=torch.int32, device=dev))


def _exact_distill(s):
    c = s["case"]
    tau, alpha, K = c["tau"], c["alpha"], c["K"]
    losses, lses, grads = [], [], []
    for r0 in range(0, s["logits"].shape[0], 256):
        cut = slice(r0, r0 + 256)
        a = s["logits"][cut].double()
        y = s["labels"][cut].long()
        live = (y >= 0).double()
        rows = torch.arange(a.shape[0], device=a.device)
        if c["kind"] == "grad":
            lt, l1 = s["lse"][cut, 0].double(), s["lse"][cut, 1].double()
        else:
            lt, l1 = torch.logsumexp(a / tau, 1), torch.logsumexp(a, 1)
        hard = l1 - a[rows, y.clamp(min=0)]
        soft = torch.zeros_like(hard)
        target = torch.zeros_like(a) if c["kind"] != "loss" else None
        if K:
            i, t = s["top_idx"][cut].long(), s["top_val"][cut].double() / tau
            lq = torch.log_softmax(t, 1)
            soft = tau * tau * (lq.exp() * (lq - (torch.gather(a, 1, i) / tau - lt[:, None]))).sum(1)
        losses.append(live * (alpha * soft + (1 - alpha) * hard))
        lses.append(torch.stack([lt, l1], 1) * live[:, None])
        if target is not None:
            target[rows, y.clamp(min=0)] += 1 - alpha
            d = (1 - alpha) * (a - l1[:, None]).exp()
            if K:
                target.scatter_add_(1, i, alpha * tau * lq.exp())
                d += alpha * tau * (a / tau - lt[:, None]).exp()
            grads.append((d - target) * (live * s["g"][cut].double())[:, None])
    if c["kind"] == "loss":
        return torch.cat(losses), torch.cat(lses)
    if c["kind"] == "grad":
        return torch.cat(grads)
    return torch.cat(losses), torch.cat(grads)
