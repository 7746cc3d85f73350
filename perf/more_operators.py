"""Cases of what keeps a pruned layer small while it is tuned and served, and judges its answers.

* 4-bit weights with group scales: the adapted projection on a frozen weight that is kept in 4 bits,
  from one token to a prompt, in 16 and 32 bits, with and without adapters;
* 8-bit activation checkpoints: packing them (and packing the weights), and the adapters' gradients
  taken from them;
* log probabilities of given tokens, with entropy and top alternatives, and their gradient.

``own`` is set from outside: false computes the plain forms (elementary torch operations in 32
bits, rounded once), true calls the library.
"""

import math

import torch

own = False


# ------------------------------------------------------------------------------------- the cases
def listed():
    return [
        # a decoding step's logits: the chosen token's log probability and eight alternatives
        dict(name="logp decode 1x32000", op="logp", T=1, V=32000, k=8, dtype="bf16"),
        # a scored batch of text: every token's log probability, entropy and sixteen alternatives
        dict(name="logp score 4096x32000", op="logp", T=4096, V=32000, k=16, dtype="bf16"),
        # a short batch in training, odd vocabulary in 32 bits, gradients of the alternatives too
        dict(name="dlogp 61x50021 f32", op="dlogp", T=61, V=50021, k=5, dtype="f32"),
        # a training batch with a large vocabulary
        dict(name="dlogp 2048x128000", op="dlogp", T=2048, V=128000, k=0, dtype="bf16"),
        # a layer's input kept for the backward pass, ragged
        dict(name="pack acts 1000x1752 f32", op="pack8", T=1000, b=1752, dtype="f32"),
        # a layer's weights packed after pruning
        dict(name="pack weights 11008x4096", op="pack4", c=11008, b=4096, g=128, dtype="bf16"),
        # the 32-bit layer set in training, inputs kept in 8 bits
        dict(name="bwd8 f32 1000", op="bwd8", T=1000, c=768, b=768, r=8, n=3, w4=False, g=64,
             dtype="f32"),
        # a training batch on a frozen 4-bit projection, inputs kept in 8 bits
        dict(name="bwd8 8192", op="bwd8", T=8192, c=4096, b=4096, r=64, n=3, w4=True, g=128,
             dtype="bf16"),
        # one token of one request
        dict(name="fwd4 decode 1", op="fwd4", T=1, c=4096, b=4096, r=0, n=0, g=128, dtype="bf16"),
        # a decoding batch, a request and an adapter per token
        dict(name="fwd4 decode 16", op="fwd4", T=16, c=11008, b=4096, r=16, n=16, g=64,
             dtype="bf16"),
        # a handful of tokens in 32 bits, ragged widths, a rank that is no multiple of 8
        dict(name="fwd4 f32 5", op="fwd4", T=5, c=1001, b=1752, r=12, n=2, g=64, dtype="f32"),
        # prompts of several requests in one batch
        dict(name="fwd4 prefill 2048", op="fwd4", T=2048, c=4096, b=4096, r=16, n=4, g=128,
             dtype="bf16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("logp", "logp", "dlogp", "dlogp", "pack8", "pack4", "bwd8", "bwd8", "fwd4",
                     "fwd4", "fwd4"))
    f32 = rng.random() < 0.3
    dt = "f32" if f32 else "bf16"
    if op in ("logp", "dlogp"):
        V = _log(rng, 500, 131072)
        T = min(_log(rng, 1, 4096), max(1, (1 << (27 if f32 else 28)) // (2 * V)))
        return dict(op=op, T=T, V=V, k=rng.choice((0, 1, 5, 8, 16, 20)), dtype=dt)
    b = 8 * _log(rng, 32, 256 if f32 else 1376)
    g = rng.choice((64, 128))
    if op == "pack8":
        return dict(op=op, T=_log(rng, 16, 8192), b=b, dtype=dt)
    c = _log(rng, 256, 2048 if f32 else 11008)
    if c * b > 4096 * 11008:
        c = 4096 * 11008 // b
    if op == "pack4":
        return dict(op=op, c=c, b=b, g=g, dtype=dt)
    r = rng.choice((4, 8, 12, 16, 20, 32, 64))
    n = _log(rng, 1, 32 if r <= 16 else 8)
    if op == "bwd8":
        T = _log(rng, 64, 1024 if f32 else 8192)
        if c * b > 4096 * 4096:
            c = 4096 * 4096 // b
        return dict(op=op, T=T, c=c, b=b, r=r, n=n, w4=rng.random() < 0.5, g=g, dtype=dt)
    T = _log(rng, 1, 512 if f32 else 2048) if rng.random() < 0.5 else _log(rng, 1, 64)
    if T * c * b > 2048 * 4096 * 4096:
        T = max(1, 2048 * 4096 * 4096 // (c * b))
    if rng.random() < 0.4:
        n = r = 0
    return dict(op=op, T=T, c=c, b=b, r=r, n=n, g=g, dtype=dt)


# ------------------------------------------------------------------------------------- the inputs
def _dtype(case):
    return torch.float32 if case["dtype"] == "f32" else torch.bfloat16


def _activations(T, b, gen):
    """Heavy-tailed activations (Student-t, 4 degrees) with a few outlier channels."""
    z = torch.randn((T, b), generator=gen, device="cuda")
    u = torch.rand((2, T, b), generator=gen, device="cuda").clamp_(min=1e-7)
    x = z / torch.sqrt(-0.5 * torch.log(u[0] * u[1]))
    hot = torch.rand((b,), generator=gen, device="cuda") < 0.005
    return x * torch.where(hot, 20.0, 1.0)


def _pruned_weight(c, b, gen):
    """N(0, 0.02^2), two of every four columns removed."""
    W = 0.02 * torch.randn((c, b), generator=gen, device="cuda")
    u = torch.rand((c, b // 4, 4), generator=gen, device="cuda")
    return torch.where((u.argsort(-1).argsort(-1) < 2).view(c, b), 0.0, W)


def _pitch(n, to):
    return -(-n // to) * to


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed) * 6151 + 29)
    dt = _dtype(case)
    rn = lambda *s: torch.randn(s, generator=gen, device="cuda")  # noqa: E731
    op = case["op"]
    s = dict(case=case)
    if op in ("logp", "dlogp"):
        T, V, k = case["T"], case["V"], case["k"]
        # a broad floor whose weight does not go by the vocabulary, a few candidates above it, some
        # of the vocabulary masked out
        Z = 2.5 * rn(T, V) - 4.0 + math.log(32000 / V)
        cand = torch.randint(0, V // 12, (T, 12), generator=gen, device="cuda")
        cand = cand + torch.arange(12, device="cuda") * (V // 12)
        Z.scatter_(1, cand, 6.0 + 3.0 * rn(T, 12))
        barred = torch.rand((V,), generator=gen, device="cuda") < 0.02
        Z = torch.where(barred, -math.inf, Z).to(dt)
        # mostly a likely token, some at random, one in sixteen left out (padding)
        u = torch.rand((T,), generator=gen, device="cuda")
        some = torch.randint(0, V, (T,), generator=gen, device="cuda")
        some = torch.where(barred[some], Z.argmax(1), some)
        target = torch.where(u < 0.7, Z.argmax(1), some)
        target = torch.where(u > 0.94, -1, target)
        s.update(Z=Z, target=target)
        if op == "dlogp":
            f = _logprobs(Z, target, k)
            s.update(stats=f["stats"], entropy=f["entropy"], top=f.get("top_index"),
                     dlogp=-torch.rand((T,), generator=gen, device="cuda") / T,
                     dentropy=1e-2 * rn(T) / T)
            if k:
                s["dtop"] = rn(T, k) / T
        return s
    if op == "pack8":
        s["X"] = _activations(case["T"], case["b"], gen).to(dt)
        return s
    if op == "pack4":
        s["W"] = _pruned_weight(case["c"], case["b"], gen).to(dt)
        return s
    T, c, b, r, n, g = (case[k] for k in ("T", "c", "b", "r", "n", "g"))
    W = _pruned_weight(c, b, gen).to(dt)
    if op == "fwd4" or case["w4"]:
        code, scale = _pack4(W, g)
        s["W4"] = _nibbles(code)
        s["S4"] = scale
    else:
        s["W"] = W
    X = _activations(T, b, gen).to(dt)
    if n:
        s["A"] = (rn(n, r, b) / math.sqrt(b)).to(dt)
        s["B"] = (0.02 * rn(n, c, r)).to(dt)
        s["scale"] = 0.5 + 1.5 * torch.rand((n,), generator=gen, device="cuda")
        if T <= 64:      # decoding: a request per token
            index = torch.randint(0, n, (T,), generator=gen, device="cuda")
        else:            # requests one behind the other
            cut = torch.rand((n,), generator=gen, device="cuda").sort().values * T
            at = torch.arange(T, device="cuda").float()
            index = torch.searchsorted(cut, at, right=True).clamp(max=n - 1)
        if n > 2:        # one in ten tokens without an adapter
            bare = torch.rand((T,), generator=gen, device="cuda") < 0.1
            index = torch.where(bare, -1, index)
        s["index"] = index.to(torch.int32)
    if op == "fwd4":
        s["X"] = X
    else:
        code, exps = _pack8(X)
        s["X8"] = torch.zeros((T, _pitch(b, 16)), dtype=torch.int8, device="cuda")
        s["X8"][:, :b] = code
        s["E8"] = torch.zeros((T, _pitch(exps.shape[1], 4)), dtype=torch.uint8, device="cuda")
        s["E8"][:, :exps.shape[1]] = exps
        s["dY"] = (1e-3 * rn(T, c)).to(dt)
        s["V"] = _shrink(_unpack8(code, exps), s["A"].float(), s["index"])
    return s


# -------------------------------------------------------------------------------- the plain forms
def _logprobs(Z, target, k):
    Zf = Z.float()
    m = Zf.max(1, keepdim=True).values
    d = Zf - m
    e = d.exp()
    S = e.sum(1, keepdim=True)
    logS = S.log()
    p = e / S
    entropy = logS[:, 0] - (p * d.clamp(min=-1e30)).sum(1)
    has = target >= 0
    z = d.gather(1, target.clamp(min=0)[:, None])[:, 0] - logS[:, 0]
    out = dict(logp=torch.where(has, z, 0.0), entropy=entropy,
               stats=torch.cat([m, logS], 1))
    if k:
        order = torch.sort(Zf, dim=1, descending=True, stable=True).indices[:, :k]
        out["top_index"] = order.contiguous()
        out["top_logp"] = d.gather(1, out["top_index"]) - logS
    return out


def _dlogprobs(Z, target, stats, entropy, dlogp, dentropy, top, dtop):
    logq = (Z.float() - stats[:, :1]) - stats[:, 1:]
    g = torch.where(target >= 0, dlogp, 0.0)
    G = g if dtop is None else g + dtop.sum(1)
    inner = G[:, None] + dentropy[:, None] * (logq.clamp(min=-1e30) + entropy[:, None])
    dZ = -(logq.exp() * inner)
    dZ.scatter_add_(1, target.clamp(min=0)[:, None], g[:, None])
    if dtop is not None:
        dZ.scatter_add_(1, top, dtop)
    return dZ.to(Z.dtype)


def _pack8(X):
    """Codes and exponents (biased by 127) of groups of 32 columns: x = code 2^(e - 127)."""
    T, b = X.shape
    n = -(-b // 32)
    Xg = torch.zeros((T, n * 32), dtype=torch.float64, device=X.device)
    Xg[:, :b] = X
    Xg = Xg.view(T, n, 32)
    top = Xg.abs().amax(2)
    e = torch.frexp(top).exponent - 7          # largest value between 64 and 128 steps
    e = e + (torch.round(torch.ldexp(top, -e)) > 127).int()
    e = e.clamp(min=-126, max=121)
    code = torch.round(torch.ldexp(Xg, -e[:, :, None])).clamp(-127, 127)
    exps = torch.where(top > 0, e + 127, 0)
    return code.view(T, n * 32)[:, :b].to(torch.int8), exps.to(torch.uint8)


def _unpack8(code, exps):
    step = torch.ldexp(torch.ones((), device=code.device), exps.int() - 127)
    return code.float() * step.repeat_interleave(32, 1)[:, :code.shape[1]]


def _pack4(W, g):
    """Codes -7 .. 7 and scales of five significant bits, [groups, c]."""
    c, b = W.shape
    n = -(-b // g)
    Wg = torch.zeros((c, n * g), dtype=torch.float32, device=W.device)
    Wg[:, :b] = W
    Wg = Wg.view(c, n, g)
    frac, exp = torch.frexp(Wg.abs().amax(2) / 7.0)
    scale = torch.ldexp(torch.round(frac * 32.0) / 32.0, exp)
    code = torch.where(scale[:, :, None] > 0, torch.round(Wg / scale[:, :, None]), 0.0)
    code = code.clamp(-7, 7).view(c, n * g)[:, :b]
    return code.to(torch.int8), scale.t().contiguous().to(torch.bfloat16)


def _nibbles(code):
    """Two codes a byte, offset by 8, the even column in the low half; rows of whole 32 bytes."""
    c, b = code.shape
    n = torch.full((c, _pitch(b, 64)), 8, dtype=torch.uint8, device=code.device)
    n[:, :b] = (code + 8).to(torch.uint8)
    return n[:, 0::2] | (n[:, 1::2] << 4)


def _unpack4(W4, S4, g, b):
    c = W4.shape[0]
    code = torch.stack([W4 & 15, W4 >> 4], 2).view(c, -1)[:, :b].float() - 8.0
    return code * S4.float().t().repeat_interleave(g, 1)[:, :b]


def _owned(index, n, r):
    cols = torch.arange(n * r, device=index.device) // r
    return index[:, None] == cols[None, :]


def _shrink(Xf, Af, index):
    n, r, b = Af.shape
    all_ = torch.where(_owned(index, n, r), Xf @ Af.reshape(n * r, b).T, 0.0)
    return all_.view(-1, n, r).sum(1)


def _spread(V, index, scale, n):
    r = V.shape[1]
    s = torch.where(index >= 0, scale[index.clamp(min=0).long()], 0.0)
    return torch.where(_owned(index, n, r), (s[:, None] * V).repeat(1, n), 0.0)


def _forward(s, case):
    X, n = s["X"], case["n"]
    Xf = X.float()
    Y = Xf @ _unpack4(s["W4"], s["S4"], case["g"], case["b"]).T
    if not n:
        return Y.to(X.dtype), None
    V = _shrink(Xf, s["A"].float(), s["index"])
    Bs = s["B"].float().permute(0, 2, 1).reshape(n * case["r"], -1)
    return (Y + _spread(V, s["index"], s["scale"], n) @ Bs).to(X.dtype), V


def _backward(s, case):
    n, r, b, c, dY = case["n"], case["r"], case["b"], case["c"], s["dY"]
    W = _unpack4(s["W4"], s["S4"], case["g"], b) if case["w4"] else s["W"].float()
    Xf = _unpack8(s["X8"][:, :b], s["E8"][:, :-(-b // 32)])
    Df, index, scale = dY.float(), s["index"], s["scale"]
    Bs = s["B"].float().permute(0, 2, 1).reshape(n * r, c)
    k = torch.where(index >= 0, scale[index.clamp(min=0).long()], 0.0)
    U = torch.where(_owned(index, n, r), k[:, None] * (Df @ Bs.T), 0.0)
    dX = Df @ W + U @ s["A"].float().reshape(n * r, b)
    dA = (U.T @ Xf).view(n, r, b)
    dB = (_spread(s["V"], index, scale, n).T @ Df).view(n, r, c).permute(0, 2, 1).contiguous()
    return dX.to(dY.dtype), dA, dB


def run(state):
    s, case = state, state["case"]
    op = case["op"]
    if own:
        import paper_2504_05346_b200 as T

        if op == "logp":
            f = T.token_logprobs(s["Z"], s["target"], k=case["k"])
            out = dict(logp=f.logp, entropy=f.entropy, stats=f.stats)
            if case["k"]:
                out.update(top_index=f.top_index, top_logp=f.top_logp)
            return out
        if op == "dlogp":
            return T.token_logprobs_backward(s["Z"], s["stats"], s["target"], s["dlogp"],
                                             entropy=s["entropy"], dentropy=s["dentropy"],
                                             top_index=s["top"], dtop=s.get("dtop"))
        if op == "pack8":
            return T.unpack_activations(T.pack_activations(s["X"]), dtype=s["X"].dtype)
        if op == "pack4":
            return T.unpack_weights(T.pack_weights(s["W"], group=case["g"]), dtype=s["W"].dtype)
        W = T.PackedWeights(s["W4"], s["S4"], case["g"], case["b"]) if "W4" in s else s["W"]
        if op == "fwd4":
            return T.adapter_forward(s["X"], W, s.get("A"), s.get("B"), s.get("index"),
                                     s.get("scale"))
        b = case["b"]
        X = T.PackedActivations(s["X8"][:, :b], s["E8"][:, :(b + 31) // 32])
        return T.adapter_backward(s["dY"], X, s["V"], W, s["A"], s["B"], s["index"], s["scale"])
    if op == "logp":
        return _logprobs(s["Z"], s["target"], case["k"])
    if op == "dlogp":
        return _dlogprobs(s["Z"], s["target"], s["stats"], s["entropy"], s["dlogp"],
                          s["dentropy"], s["top"], s.get("dtop"))
    if op == "pack8":
        return _unpack8(*_pack8(s["X"])).to(s["X"].dtype)
    if op == "pack4":
        code, scale = _pack4(s["W"], case["g"])
        return _unpack4(_nibbles(code), scale, case["g"], case["b"]).to(s["W"].dtype)
    return _forward(s, case) if op == "fwd4" else _backward(s, case)


# ---------------------------------------------------------------------------- what a pass must do
def work(case):
    e = 4 if case["dtype"] == "f32" else 2
    op = case["op"]
    if op == "logp":
        T, V, k = case["T"], case["V"], case["k"]
        return dict(bytes=T * (e * V + 8 + 16 + 12 * k), flops=6.0 * T * V)
    if op == "dlogp":
        T, V, k = case["T"], case["V"], case["k"]
        return dict(bytes=T * (2 * e * V + 8 + 20 + 12 * k), flops=6.0 * T * V)
    if op == "pack8":
        # values in, codes and exponents out, and both back
        n = case["T"] * case["b"]
        return dict(bytes=2 * n * (e + 33 / 32), flops=4.0 * n)
    if op == "pack4":
        n = case["c"] * case["b"]
        return dict(bytes=2 * n * (e + 0.5 + 2.0 / case["g"]), flops=4.0 * n)
    T, c, b, r, n, g = (case[k] for k in ("T", "c", "b", "r", "n", "g"))
    used = min(n, T)
    params = e * used * r * (b + c)
    if op == "fwd4" or case["w4"]:
        params += c * b * (0.5 + 2.0 / g)
    else:
        params += e * c * b
    if op == "fwd4":
        return dict(bytes=params + e * T * (b + c) + (4 * T * (r + 1) if n else 0),
                    flops=2.0 * T * (c * b + r * (b + c)))
    return dict(bytes=params + e * T * (b + c) + T * b * 33 / 32 + 4 * T * (r + 1) +
                4 * n * r * (b + c), flops=2.0 * T * (c * b + 2 * r * (b + c)))


# -------------------------------------------------------------------------------- in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    d = torch.float64
    op = case["op"]
    if op in ("logp", "dlogp"):
        Z, target, k = s["Z"], s["target"].tolist(), case["k"]
        logq = torch.log_softmax(Z.to(d), 1)
        finite = torch.where(logq > -math.inf, logq, 0.0)
        H = -(logq.exp() * finite).sum(1)
        rows = [t for t, i in enumerate(target) if i >= 0]
        at = torch.tensor(rows, dtype=torch.long, device=Z.device)
        ids = s["target"][at]
        if op == "logp":
            logp = torch.zeros_like(H)
            logp[at] = logq[at, ids]
            top = Z.to(d).amax(1)
            # a row's log of the sum is what its largest value's log probability falls short of zero
            best = logq.amax(1)
            out = dict(logp=logp, entropy=H, stats=torch.stack([top, -best], 1))
            if k:
                # the k-th largest, with an order that no two columns share
                rank = torch.argsort(logq.neg(), dim=1, stable=True)[:, :k]
                out["top_index"], out["top_logp"] = None, logq.gather(1, rank)
            return out
        # through the softmax's Jacobian: dz = a - p (1.a), with a the gradient by log probability
        a = torch.zeros_like(logq)
        a[at, ids] += s["dlogp"].to(d)[at]
        if k:
            a.scatter_add_(1, s["top"], s["dtop"].to(d))
        # dH = -sum_j (1 + log p_j) p_j dlogp_j, given the entropy and the row's sums of the call
        logq = (Z.to(d) - s["stats"][:, :1].to(d)) - s["stats"][:, 1:].to(d)
        finite = torch.where(logq > -math.inf, logq, 0.0)
        p = logq.exp()
        bend = s["dentropy"].to(d)[:, None] * p * (finite + s["entropy"].to(d)[:, None])
        return a - p * a.sum(1, keepdim=True) - bend
    if op == "pack8":
        X = s["X"].to(d)
        out = torch.zeros_like(X)
        for j in range(0, X.shape[1], 32):
            x = X[:, j:j + 32]
            top = x.abs().amax(1, keepdim=True)
            step = torch.exp2(torch.floor(torch.log2(torch.where(top > 0, top, 1.0))) - 6.0)
            step = torch.where(torch.round(top / step) > 127, 2.0 * step, step)
            out[:, j:j + 32] = torch.round(x / step) * step
        return out
    if op == "pack4":
        W = s["W"].to(d)
        out = torch.zeros_like(W)
        for j in range(0, W.shape[1], case["g"]):
            w = W[:, j:j + case["g"]]
            top = w.abs().amax(1, keepdim=True) / 7.0
            unit = torch.exp2(torch.floor(torch.log2(torch.where(top > 0, top, 1.0))) - 4.0)
            step = torch.where(top > 0, torch.round(top / unit) * unit, 1.0)
            out[:, j:j + case["g"]] = torch.round(w / step).clamp(-7, 7) * step
        return out
    b, c, g = case["b"], case["c"], case["g"]
    if "W4" in s:
        W = torch.zeros((c, b), dtype=d, device="cuda")
        W[:, 0::2] = (s["W4"] & 15)[:, :b // 2].to(d) - 8
        W[:, 1::2] = (s["W4"] >> 4)[:, :b // 2].to(d) - 8
        for j in range(s["S4"].shape[0]):
            W[:, g * j:g * j + g] *= s["S4"][j].to(d)[:, None]
    else:
        W = s["W"].to(d)
    A, B = (s[k].to(d) if case["n"] else None for k in ("A", "B"))
    rows = {}
    for t, i in enumerate(s["index"].tolist() if case["n"] else ()):
        if i >= 0:
            rows.setdefault(i, []).append(t)
    if op == "fwd4":
        X = s["X"].to(d)
        Y = torch.einsum("tk,ck->tc", X, W)
        if not case["n"]:
            return Y, None
        V = torch.zeros((X.shape[0], case["r"]), dtype=d, device="cuda")
        for i, ts in rows.items():
            V[ts] = torch.einsum("tk,rk->tr", X[ts], A[i])
            Y[ts] += s["scale"][i].to(d) * torch.einsum("tr,cr->tc", V[ts], B[i])
        return Y, V
    X = s["X8"][:, :b].to(d)
    for j in range(0, b, 32):
        X[:, j:j + 32] *= torch.exp2(s["E8"][:, j // 32].to(d) - 127)[:, None]
    dY, V = s["dY"].to(d), s["V"].to(d)
    dX = torch.einsum("tc,ck->tk", dY, W)
    dA, dB = torch.zeros_like(A), torch.zeros_like(B)
    for i, ts in rows.items():
        k = s["scale"][i].to(d)
        U = k * torch.einsum("tc,cr->tr", dY[ts], B[i])
        dX[ts] += torch.einsum("tr,rk->tk", U, A[i])
        dA[i] = torch.einsum("tr,tk->rk", U, X[ts])
        dB[i] = k * torch.einsum("tc,tr->cr", dY[ts], V[ts])
    return dX, dA, dB
