"""Cases of the recovery operators: what a pruned layer needs to be tuned and served again.

Two operators of the library are measured here, each direction and type of them:

* the adapted projection, ``Y = X W^T + s_i (X A_i^T) B_i^T``: a pruned, frozen weight beside the
  low-rank adapters (A_i, B_i) of many requests, every token with an adapter of its own or none;
  forward for serving and training, backward for training;
* the orthogonalised update (Newton-Schulz products, as the Muon optimiser takes it): on its own,
  and as a whole step with momentum, the pruning mask and the new weights.

``own`` is set from outside: false computes the plain forms (elementary torch operations in 32
bits, rounded once), true calls the library.
"""

import math

import torch

own = False

COEF = (3.4445, -4.7750, 2.0315)   # the quintic of the Newton-Schulz iteration
STEPS = 5
EPS = 1e-7
MOMENTUM = 0.95
DECAY = 0.01


# ------------------------------------------------------------------------------------- the cases
def listed():
    return [
        # one token of one request: the smallest call of a served 4096 x 4096 projection
        dict(name="fwd decode 1", op="forward", T=1, c=4096, b=4096, r=16, n=8, order="token",
             dtype="bf16"),
        # a decoding batch, one token per request and nearly as many adapters as requests
        dict(name="fwd decode 64", op="forward", T=64, c=11008, b=4096, r=16, n=64, order="token",
             dtype="bf16"),
        # a mixed batch: ragged token count, ragged widths, a rank that is no multiple of 8
        dict(name="fwd ragged 333", op="forward", T=333, c=1001, b=1752, r=12, n=5, order="request",
             dtype="bf16"),
        # prompts of several requests in one batch
        dict(name="fwd prefill 4096", op="forward", T=4096, c=4096, b=4096, r=32, n=7,
             order="request", dtype="bf16"),
        # the 32-bit layer set (768 wide), a short batch
        dict(name="fwd f32 500", op="forward", T=500, c=768, b=768, r=8, n=3, order="request",
             dtype="f32"),
        # one training batch of a few tasks' adapters
        dict(name="bwd 2048", op="backward", T=2048, c=4096, b=4096, r=16, n=4, order="request",
             dtype="bf16"),
        # the wide down projection in training, one adapter of a high rank
        dict(name="bwd 8192 wide", op="backward", T=8192, c=4096, b=11008, r=64, n=1,
             order="request", dtype="bf16"),
        # the 32-bit layer set in training
        dict(name="bwd f32 1000", op="backward", T=1000, c=768, b=768, r=8, n=3, order="request",
             dtype="f32"),
        # the A matrices of a set of adapters, one update for all
        dict(name="ortho adapters 32x16x4096", op="ortho", k=32, m=16, n=4096, dtype="f32"),
        # a layer of the 32-bit set, kept pruned while its other weights are tuned
        dict(name="step 768x768", op="step", k=1, m=768, n=768, dtype="f32", mask="2:4"),
        # a 4096 x 4096 projection in bf16, pruned to half of its weights in no pattern
        dict(name="step 4096x4096", op="step", k=1, m=4096, n=4096, dtype="bf16", mask="half"),
        # the up projection: tall, the largest of the set
        dict(name="ortho 11008x4096", op="ortho", k=1, m=11008, n=4096, dtype="bf16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("forward", "forward", "backward", "ortho", "step"))
    if kind in ("forward", "backward"):
        f32 = rng.random() < 0.2
        c = _log(rng, 256, 2048 if f32 else 11008)
        b = 8 * _log(rng, 32, 256 if f32 else 1376)
        r = rng.choice((4, 8, 12, 16, 20, 32, 64))
        order = rng.choice(("token", "request"))
        n = _log(rng, 1, 64 if r <= 16 else 16)
        T = _log(rng, 1 if kind == "forward" else 64, 2048 if f32 else 8192)
        if order == "token":
            T = min(T, 512)
        if c * b > 4096 * 11008:
            c = 4096 * 11008 // b
        return dict(op=kind, T=T, c=c, b=b, r=r, n=n, order=order, dtype="f32" if f32 else "bf16")
    if rng.random() < 0.4:   # adapters: a short side, many at once
        short, long_ = _log(rng, 4, 64), _log(rng, 256, 11008)
        m, n = (short, long_) if rng.random() < 0.5 else (long_, short)
        k = _log(rng, 1, 64)
    else:
        m, n, k = _log(rng, 192, 4096), _log(rng, 192, 11008), 1
        if rng.random() < 0.3:
            m, n = n, m
        k = rng.choice((1, 1, 2, 4)) if m * n <= 1 << 21 else 1
    case = dict(op=kind, k=k, m=m, n=n, dtype=rng.choice(("f32", "bf16")))
    if kind == "step":
        case["mask"] = rng.choice(("none", "2:4", "half"))
    return case


# ------------------------------------------------------------------------------------- the inputs
def _dtype(case):
    return torch.float32 if case["dtype"] == "f32" else torch.bfloat16


def _pruned(W, how, gen):
    """The mask of a pruned weight (1 = removed): two of every four columns, or half anywhere."""
    u = torch.rand(W.shape, generator=gen, device=W.device)
    if how == "half" or W.shape[-1] % 4:
        return (u < 0.5).to(torch.uint8)
    g = u.view(*W.shape[:-1], -1, 4)
    return (g.argsort(-1).argsort(-1) < 2).to(torch.uint8).view(W.shape)


def _activations(T, b, gen):
    """Heavy-tailed activations (Student-t, 4 degrees) with a few outlier channels."""
    dev = "cuda"
    z = torch.randn((T, b), generator=gen, device=dev)
    u = torch.rand((2, T, b), generator=gen, device=dev).clamp_(min=1e-7)
    x = z / torch.sqrt(-0.5 * torch.log(u[0] * u[1]))
    hot = torch.rand((b,), generator=gen, device=dev) < 0.005
    return x * torch.where(hot, 20.0, 1.0)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed) * 7919 + 17)
    dt = _dtype(case)
    rn = lambda *s: torch.randn(s, generator=gen, device="cuda")  # noqa: E731
    if case["op"] in ("forward", "backward"):
        T, c, b, r, n = (case[k] for k in ("T", "c", "b", "r", "n"))
        W = 0.02 * rn(c, b)
        W = torch.where(_pruned(W, "2:4", gen) != 0, 0.0, W).to(dt)
        X = _activations(T, b, gen).to(dt)
        A = (rn(n, r, b) / math.sqrt(b)).to(dt)
        B = (0.02 * rn(n, c, r)).to(dt)
        scale = 0.5 + 1.5 * torch.rand((n,), generator=gen, device="cuda")
        if case["order"] == "token":      # decoding: a request per token
            index = torch.randint(0, n, (T,), generator=gen, device="cuda", dtype=torch.int32)
        else:                             # requests of unequal lengths, one behind the other
            reqs = max(n, 2)
            cut = torch.rand((reqs - 1,), generator=gen, device="cuda").sort().values * T
            of = torch.searchsorted(cut, torch.arange(T, device="cuda").float(), right=True)
            who = torch.randperm(reqs, generator=gen, device="cuda") % n
            index = who[of].to(torch.int32)
        if n > 2:                         # one in ten tokens without an adapter
            bare = torch.rand((T,), generator=gen, device="cuda") < 0.1
            index = torch.where(bare, -1, index).to(torch.int32)
        s = dict(case=case, X=X, W=W, A=A, B=B, index=index, scale=scale)
        if case["op"] == "backward":
            s["dY"] = (1e-3 * rn(T, c)).to(dt)
            # what the forward pass of the same batch left: X A_i^T in 32 bits
            s["V"] = _shrink(X.float(), A.float(), index)
        return s
    k, m, n = case["k"], case["m"], case["n"]
    # a gradient as layers have it: a sum over tokens with few strong directions over a noisy floor
    q = max(1, min(m, n) // 16)
    lead = torch.bmm(rn(k, m, q), rn(k, q, n)) / math.sqrt(q)
    G = (1e-3 * (0.5 * lead + rn(k, m, n))).to(dt)
    if k == 1:
        G = G[0]
    s = dict(case=case, G=G)
    if case["op"] == "step":
        W = 0.02 * rn(k, m, n).view(G.shape)
        mask = None if case["mask"] == "none" else _pruned(W, case["mask"], gen)
        if mask is not None:
            W = torch.where(mask != 0, 0.0, W)
        M = 3e-3 * rn(k, m, n).view(G.shape)
        if mask is not None:
            M = torch.where(mask != 0, 0.0, M)
        s.update(W=W.to(dt), M=M, mask=mask, lr=2e-4, gain=0.2 * math.sqrt(max(m, n)))
    return s


# -------------------------------------------------------------------------------- the plain forms
def _owned(index, n, r):
    """[T, n r] truth values: the columns of all adapters' stacked ranks that belong to a token."""
    cols = torch.arange(n * r, device=index.device) // r
    return index[:, None] == cols[None, :]


def _shrink(Xf, Af, index):
    """V[t] = X[t] A_i^T of the token's own adapter (0 without one), [T, r] in 32 bits."""
    n, r, b = Af.shape
    all_ = torch.where(_owned(index, n, r), Xf @ Af.reshape(n * r, b).T, 0.0)
    return all_.view(-1, n, r).sum(1)


def _spread(V, index, scale, n):
    """s_i V[t] in the columns of the token's adapter, zeros elsewhere: [T, n r]."""
    r = V.shape[1]
    s = torch.where(index >= 0, scale[index.clamp(min=0).long()], 0.0)
    return torch.where(_owned(index, n, r), (s[:, None] * V).repeat(1, n), 0.0)


def _forward(X, W, A, B, index, scale):
    n, r, b = A.shape
    Xf, Af, Bf = X.float(), A.float(), B.float()
    V = _shrink(Xf, Af, index)
    Bs = Bf.permute(0, 2, 1).reshape(n * r, -1)
    Y = Xf @ W.float().T + _spread(V, index, scale, n) @ Bs
    return Y.to(X.dtype), V


def _backward(dY, X, V, W, A, B, index, scale):
    n, r, b = A.shape
    c = W.shape[0]
    Df, Af = dY.float(), A.float()
    Bs = B.float().permute(0, 2, 1).reshape(n * r, c)
    s = torch.where(index >= 0, scale[index.clamp(min=0).long()], 0.0)
    U = torch.where(_owned(index, n, r), s[:, None] * (Df @ Bs.T), 0.0)
    dX = Df @ W.float() + U @ Af.reshape(n * r, b)
    dA = (U.T @ X.float()).view(n, r, b)
    dB = (_spread(V, index, scale, n).T @ Df).view(n, r, c).permute(0, 2, 1).contiguous()
    return dX.to(X.dtype), dA, dB


def _newton_schulz(G):
    a, b, c = COEF
    X = G.float()
    tall = X.shape[-2] > X.shape[-1]
    if tall:
        X = X.mT
    X = X / (X.square().sum((-2, -1), keepdim=True).sqrt() + EPS)
    for _ in range(STEPS):
        S = X @ X.mT
        X = a * X + (b * S + c * (S @ S)) @ X
    return X.mT if tall else X


def _ortho(G):
    return _newton_schulz(G).to(torch.bfloat16).contiguous()


def _step(W, M, G, mask, lr, gain):
    Gf = G.float()
    if mask is not None:
        Gf = torch.where(mask != 0, 0.0, Gf)
    Mn = MOMENTUM * M + Gf
    O = _newton_schulz(Gf + MOMENTUM * Mn)
    Wn = (1.0 - lr * DECAY) * W.float() - lr * gain * O
    if mask is not None:
        Wn = torch.where(mask != 0, 0.0, Wn)
    return Wn.to(W.dtype), Mn


def run(state):
    op = state["case"]["op"]
    s = state
    if own:
        import paper_2504_05346_b200 as T

        if op == "forward":
            return T.adapter_forward(s["X"], s["W"], s["A"], s["B"], s["index"], s["scale"])
        if op == "backward":
            return T.adapter_backward(s["dY"], s["X"], s["V"], s["W"], s["A"], s["B"], s["index"],
                                      s["scale"])
        if op == "ortho":
            return T.orthogonalise(s["G"], steps=STEPS, coef=COEF, eps=EPS)
        return T.orthogonal_step(s["W"], s["M"], s["G"], s["mask"], lr=s["lr"], gain=s["gain"],
                                 momentum=MOMENTUM, weight_decay=DECAY, steps=STEPS, coef=COEF,
                                 eps=EPS)
    if op == "forward":
        return _forward(s["X"], s["W"], s["A"], s["B"], s["index"], s["scale"])
    if op == "backward":
        return _backward(s["dY"], s["X"], s["V"], s["W"], s["A"], s["B"], s["index"], s["scale"])
    if op == "ortho":
        return _ortho(s["G"])
    return _step(s["W"], s["M"], s["G"], s["mask"], s["lr"], s["gain"])


# ---------------------------------------------------------------------------- what a pass must do
def work(case):
    e = 4 if case["dtype"] == "f32" else 2
    if case["op"] in ("forward", "backward"):
        T, c, b, r, n = (case[k] for k in ("T", "c", "b", "r", "n"))
        used = min(n, T)
        params = e * (c * b + used * r * (b + c))
        if case["op"] == "forward":
            return dict(bytes=params + e * T * (b + c) + 4 * T * (r + 1),
                        flops=2.0 * T * (c * b + r * (b + c)))
        return dict(bytes=params + e * T * (2 * b + c) + 4 * T * (r + 1) + 4 * n * r * (b + c),
                    flops=2.0 * T * (c * b + 2 * r * (b + c)))
    k, m, n = case["k"], case["m"], case["n"]
    s, l = min(m, n), max(m, n)
    # per step the two products of the short side are symmetric: half of each is enough
    flops = k * STEPS * (1.0 * s * s * l + 1.0 * s ** 3 + 2.0 * s * s * l)
    if s * 3 <= l:
        # a long matrix: all steps on the short side's Gram matrix, then one product
        flops = min(flops, k * (3.0 * s * s * l + STEPS * 4.0 * s ** 3))
    if case["op"] == "ortho":
        return dict(bytes=k * m * n * (e + 2), flops=flops)
    return dict(bytes=k * m * n * (3 * e + 8 + (0 if case["mask"] == "none" else 1)), flops=flops)


# -------------------------------------------------------------------------------- in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    d = torch.float64
    if case["op"] in ("forward", "backward"):
        X, W, A, B = (s[k].to(d) for k in ("X", "W", "A", "B"))
        index, scale = s["index"].tolist(), s["scale"].to(d)
        rows = {}
        for t, i in enumerate(index):
            if i >= 0:
                rows.setdefault(i, []).append(t)
        if case["op"] == "forward":
            Y = torch.einsum("tk,ck->tc", X, W)
            V = torch.zeros((X.shape[0], case["r"]), dtype=d, device=X.device)
            for i, ts in rows.items():
                V[ts] = torch.einsum("tk,rk->tr", X[ts], A[i])
                Y[ts] += scale[i] * torch.einsum("tr,cr->tc", V[ts], B[i])
            return Y, V
        dY, V = s["dY"].to(d), s["V"].to(d)
        dX = torch.einsum("tc,ck->tk", dY, W)
        dA, dB = torch.zeros_like(A), torch.zeros_like(B)
        for i, ts in rows.items():
            U = scale[i] * torch.einsum("tc,cr->tr", dY[ts], B[i])
            dX[ts] += torch.einsum("tr,rk->tk", U, A[i])
            dA[i] = torch.einsum("tr,tk->rk", U, X[ts])
            dB[i] = scale[i] * torch.einsum("tc,tr->cr", dY[ts], V[ts])
        return dX, dA, dB
    a, b, c = COEF
    U = s["G"].to(d)
    if case["op"] == "step":
        keep = None if s["mask"] is None else (s["mask"] == 0).to(d)
        U = U if keep is None else U * keep
        Mn = MOMENTUM * s["M"].to(d) + U
        U = U + MOMENTUM * Mn
    norm = torch.linalg.vector_norm(U, dim=(-2, -1), keepdim=True)
    X = U / (norm + EPS)
    for _ in range(STEPS):               # odd polynomial of X, written from the other side
        if X.shape[-2] <= X.shape[-1]:
            S = torch.matmul(X, X.transpose(-2, -1))
            X = a * X + b * torch.matmul(S, X) + c * torch.matmul(S, torch.matmul(S, X))
        else:
            S = torch.matmul(X.transpose(-2, -1), X)
            X = a * X + b * torch.matmul(X, S) + c * torch.matmul(torch.matmul(X, S), S)
    if case["op"] == "ortho":
        return X
    Wn = (1.0 - s["lr"] * DECAY) * s["W"].to(d) - s["lr"] * s["gain"] * X
    return Wn if keep is None else Wn * keep, Mn
