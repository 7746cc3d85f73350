"""A pruned layer kept small, trained and judged, as its operators are used together: 4-bit weights with
adapters as an output head, activations kept in 8 bits, the loss from the log probabilities of given
tokens with entropy and alternatives, its gradient through all of them, and the update.

The reference is float64 autograd on what the codes stand for.  The logits are rounded once between the
operators, so the reference's loss is taken from the operators' own logits, and its gradient is pulled
back through float64 products.  Tolerances: fp32 sums of a few hundred to a thousand terms (1e-5 of the
result); in bf16 the logits' gradient is rounded once more (2^-9 of each value, at most 2^-8 of the
norm of the result), dX as well, the adapters' gradients keep fp32.
"""

import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

DEV = "cuda"
BF16, F32, F64 = torch.bfloat16, torch.float32, torch.float64


@pytest.fixture(scope="module")
def T():
    import paper_2504_05346_b200 as T_
    from paper_2504_05346_b200 import build as B_

    B_.build()
    T_.load_library()
    return T_


def layer(T, Tn, V, b, n, r, dtype, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    rn = lambda *s: torch.randn(s, generator=g, device=DEV)  # noqa: E731
    W = (2.0 * rn(V, b) / math.sqrt(b)).to(dtype)
    u = torch.rand((V, b // 4, 4), generator=g, device=DEV)
    W[(u.argsort(-1).argsort(-1) < 2).view(V, b)] = 0          # 2:4
    X = rn(Tn, b).to(dtype)
    A, B = (rn(n, r, b) / math.sqrt(b)).to(dtype), (0.3 * rn(n, V, r)).to(dtype)
    index = torch.randint(-1, n, (Tn,), generator=g, device=DEV, dtype=torch.int32)
    scale = 0.5 + torch.rand((n,), generator=g, device=DEV)
    target = torch.randint(0, V, (Tn,), generator=g, device=DEV)
    target[::7] = -1
    return W, X, A, B, index, scale, target


def loss_of(logq, target, top, weights):
    """dlogp, dentropy and dtop weighted sums in float64, for autograd."""
    wl, wh, wt = (w.double() for w in weights)
    q = logq.exp()
    H = -(q * logq).sum(1)
    has = target >= 0
    picked = torch.where(has, logq.gather(1, target.clamp(min=0)[:, None])[:, 0], 0.0)
    return (wl * picked).sum() + (wh * H).sum() + (wt * logq.gather(1, top)).sum()


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("Tn", [1, 9, 40, 300])
def test_the_operators_together(T, Tn, dtype):
    V, b, n, r, k = 1001, 264, 3, 8, 4
    W, X, A, B, index, scale, target = layer(T, Tn, V, b, n, r, dtype, seed=Tn)
    P = T.pack_weights(W, 64)
    Wq = T.unpack_weights(P, F32).double()
    assert bool((Wq[W == 0] == 0).all())            # what is pruned stays pruned
    Z, Vr = T.adapter_forward(X, P, A, B, index, scale, check=True)
    X8 = T.pack_activations(X)                      # X itself may go now
    f = T.token_logprobs(Z, target, k)
    g = torch.Generator(device=DEV).manual_seed(Tn + 1)
    rn = lambda *s: torch.randn(s, generator=g, device=DEV)  # noqa: E731
    weights = (rn(Tn) / Tn, 0.1 * rn(Tn) / Tn, 0.1 * rn(Tn, k) / Tn)
    dZ = T.token_logprobs_backward(Z, f.stats, target, weights[0], f.entropy, weights[1], f.top_index,
                                   weights[2])
    dX, dA, dB = T.adapter_backward(dZ, X8, Vr, P, A, B, index, scale, check=True)

    # the loss and its gradient by the logits
    Zr = Z.double().requires_grad_()
    loss = loss_of(torch.log_softmax(Zr, 1), target, f.top_index, weights)
    loss.backward()
    mine = (weights[0] * f.logp).double().sum() + (weights[1] * f.entropy).double().sum() + \
        (weights[2] * f.top_logp).double().sum()
    size = weights[0].abs().sum() * 12 + weights[1].abs().sum() * 7 + weights[2].abs().sum() * 12
    assert abs(mine - loss.detach()).item() <= 3e-6 * size.item()
    err = (dZ.double() - Zr.grad).norm() / Zr.grad.norm()
    assert err.item() <= (2.0 ** -8 if dtype == BF16 else 2e-5)
    # and on through the layer, from the gradient that was handed on
    up = dZ.double()
    x8 = T.unpack_activations(X8, F32).double()
    rX, rA, rB = up @ Wq, torch.zeros_like(A, dtype=F64), torch.zeros_like(B, dtype=F64)
    for i in range(n):
        at = (index == i).nonzero()[:, 0]
        U = scale[i].double() * (up[at] @ B[i].double())
        rX[at] += U @ A[i].double()
        rA[i] = U.T @ x8[at]
        rB[i] = scale[i].double() * (up[at].T @ Vr[at].double())
    rel = lambda x, y: ((x.double() - y).norm() / y.norm().clamp(min=1e-30)).item()  # noqa: E731
    assert rel(dX, rX) <= (3e-3 if dtype == BF16 else 1e-5)
    assert rel(dA, rA) <= 1e-5 and rel(dB, rB) <= 1e-5
    # the update takes the gradients as they are
    A32, M = A.float(), torch.zeros_like(dA)
    A1, _ = T.orthogonal_step(A32, M, dA, lr=0.01, momentum=0.0)
    assert A1.shape == A.shape and bool(A1.isfinite().all())


def test_gradient_of_the_whole_against_differences(T):
    """d loss along one direction of A and of B, in fp32.  Central differences with h = 2^-7: the third
    derivative's part is h^2 / 6 of a number of order 1 (1e-5), and the operators' own error, 1e-6 of a
    loss of order 5, comes back over h: 6e-4.  The gradient is taken with the activations in 32 bits; in 8
    bits its A part is that of the rounded activations (half a step of 2^-7 of a group's largest, spread
    over 264 columns: below 1 % of the norm)."""
    W, X, A, B, index, scale, target = layer(T, 24, 501, 264, 3, 8, F32, seed=5)
    target = target.clamp(min=0)
    P = T.pack_weights(W, 128)
    g = torch.Generator(device=DEV).manual_seed(6)
    w = torch.full((24,), 1.0 / 24, device=DEV)

    def loss(A, B):
        return (w * T.token_logprobs(T.adapter_forward(X, P, A, B, index, scale)[0], target).logp).double().sum()

    Z, V = T.adapter_forward(X, P, A, B, index, scale)
    f = T.token_logprobs(Z, target)
    dZ = T.token_logprobs_backward(Z, f.stats, target, w)
    _, dA, dB = T.adapter_backward(dZ, X, V, P, A, B, index, scale)
    _, dA8, dB8 = T.adapter_backward(dZ, T.pack_activations(X), V, P, A, B, index, scale)
    assert torch.equal(dB, dB8) and (dA8 - dA).norm() <= 1e-2 * dA.norm()
    h = 2.0 ** -7
    for which, d in (("A", dA), ("B", dB)):
        direction = d / d.norm()
        up = loss(A + h * direction, B) if which == "A" else loss(A, B + h * direction)
        down = loss(A - h * direction, B) if which == "A" else loss(A, B - h * direction)
        slope = ((up - down) / (2 * h)).item()
        assert abs(slope - d.norm().item()) <= 2e-3 * max(1.0, d.norm().item())


def test_a_training_step_in_a_graph(T):
    """Forward, loss, gradient and update captured once and replayed on new batches."""
    W, X, A, B, index, scale, target = layer(T, 40, 777, 136, 3, 8, BF16, seed=7)
    P = T.pack_weights(W, 64)
    w = torch.full((40,), 1.0 / 40, device=DEV)
    bufs = [X.clone(), index.clone(), target.clone()]

    def step(X, index, target):
        Z, V = T.adapter_forward(X, P, A, B, index, scale)
        X8 = T.pack_activations(X)
        f = T.token_logprobs(Z, target)
        dZ = T.token_logprobs_backward(Z, f.stats, target, w, out=Z)
        return (f.logp,) + T.adapter_backward(dZ, X8, V, P, A, B, index, scale, need_dx=False)[1:]

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        step(*bufs)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step(*bufs)
    for seed in (8, 9):
        _, Xn, _, _, inew, _, tn = layer(T, 40, 777, 136, 3, 8, BF16, seed=seed)
        for buf, new in zip(bufs, (Xn, inew, tn)):
            buf.copy_(new)
        graph.replay()
        want = step(Xn, inew, tn)
        assert all(torch.equal(x, y) for x, y in zip(out, want))
