"""The recovery operators against plain float64 implementations: the projection with low-rank
adapters (forward, backward) and the orthogonalised update (alone and as a masked step).

Tolerances, from the arithmetic (relative Frobenius errors unless stated):
  * a bf16 result is one rounding of an fp32 sum: at most 2^-9 = 1.95e-3 elementwise, 1.7e-3 in the
    norm for values spread over a binade; the adapter part's factor is rounded to bf16 first, the
    same size again on that part: 3e-3 in all.
  * fp32 results: fp32 sums of K products in some order, error below K^0.5 2^-24 to K 2^-24
    of the sum of magnitudes: 1e-5 for the sizes here (K up to a few thousand).
  * the orthogonalised update has fp16 operands (2^-12 each) and a bf16 result: 4e-3.
"""

import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

DEV = "cuda"
TOL_BF16 = 3e-3
TOL_F32 = 1e-5
TOL_ORTHO = 4e-3


@pytest.fixture(scope="module")
def T():
    import paper_2504_05346_b200 as T_
    from paper_2504_05346_b200 import build as B_

    B_.build()
    T_.load_library()
    return T_


def rel(x, ref):
    x, ref = x.double(), ref.double()
    n = ref.norm().item()
    return (x - ref).norm().item() / n if n else x.norm().item()


def make(Tn, c, b, n, r, dtype, seed, order="mixed", pad=0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    rn = lambda *s: torch.randn(s, generator=g, device=DEV)  # noqa: E731
    X = rn(Tn, b + pad).to(dtype)[:, :b]
    W = (0.02 * rn(c, b + pad)).to(dtype)[:, :b]
    A = (rn(n, r, b) / math.sqrt(b)).to(dtype)
    B = (0.1 * rn(n, c, r)).to(dtype)
    scale = 0.5 + torch.rand((n,), generator=g, device=DEV)
    if order == "mixed":
        index = torch.randint(-1, n, (Tn,), generator=g, device=DEV, dtype=torch.int32)
    elif order == "none":
        index = torch.full((Tn,), -1, dtype=torch.int32, device=DEV)
    elif order == "one":
        index = torch.full((Tn,), n - 1, dtype=torch.int32, device=DEV)
    else:
        index = (torch.arange(Tn, device=DEV) * n // max(Tn, 1)).to(torch.int32)
    dY = rn(Tn, c).to(dtype)
    return X, W, A, B, index, scale, dY


def ref_forward(X, W, A, B, index, scale):
    X, W, A, B, scale = (t.double() for t in (X, W, A, B, scale))
    Y = X @ W.T
    V = torch.zeros((X.shape[0], A.shape[1]), dtype=torch.float64, device=X.device)
    for i in range(A.shape[0]):
        at = (index == i).nonzero()[:, 0]
        V[at] = X[at] @ A[i].T
        Y[at] += scale[i] * (V[at] @ B[i].T)
    return Y, V


def ref_backward(dY, X, V, W, A, B, index, scale):
    dY, X, V, W, A, B, scale = (t.double() for t in (dY, X, V, W, A, B, scale))
    dX = dY @ W
    dA, dB = torch.zeros_like(A), torch.zeros_like(B)
    for i in range(A.shape[0]):
        at = (index == i).nonzero()[:, 0]
        U = scale[i] * (dY[at] @ B[i])
        dX[at] += U @ A[i]
        dA[i] = U.T @ X[at]
        dB[i] = scale[i] * (dY[at].T @ V[at])
    return dX, dA, dB


SHAPES = [
    # T, c, b, n, r, order
    (1, 64, 64, 1, 4, "one"),
    (1, 4096, 1024, 8, 16, "mixed"),
    (2, 130, 72, 3, 1, "mixed"),
    (15, 1001, 520, 5, 12, "mixed"),
    (16, 256, 512, 16, 16, "blocks"),
    (33, 1, 8, 2, 8, "mixed"),
    (64, 777, 1032, 64, 16, "blocks"),
    (100, 129, 136, 40, 5, "mixed"),
    (127, 512, 768, 3, 64, "mixed"),
    (129, 384, 1096, 2, 128, "mixed"),
    (257, 260, 264, 9, 20, "mixed"),
    (300, 512, 512, 4, 8, "none"),
    (513, 768, 768, 3, 8, "blocks"),
    (700, 1536, 1000, 150, 7, "mixed"),
    (1025, 515, 2056, 6, 32, "mixed"),
    (2048, 2048, 1024, 1, 16, "one"),
    (3000, 640, 1280, 5, 24, "blocks"),
]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_adapter_forward(T, shape, dtype):
    Tn, c, b, n, r, order = shape
    X, W, A, B, index, scale, _ = make(Tn, c, b, n, r, dtype, seed=Tn + c, order=order)
    Y, V = T.adapter_forward(X, W, A, B, index, scale, check=True)
    Yr, Vr = ref_forward(X, W, A, B, index, scale)
    assert rel(V, Vr) <= TOL_F32
    assert rel(Y, Yr) <= (TOL_BF16 if dtype == torch.bfloat16 else TOL_F32)
    # a wrong row would hide in the norm of many: every token on its own
    err = (Y.double() - Yr).norm(dim=1) / Yr.norm(dim=1).clamp(min=1e-30)
    assert err.max().item() <= (2 * TOL_BF16 if dtype == torch.bfloat16 else 3 * TOL_F32) * (
        1 if c > 8 else 4)
    assert bool((V[index < 0] == 0).all())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_adapter_backward(T, shape, dtype):
    Tn, c, b, n, r, order = shape
    X, W, A, B, index, scale, dY = make(Tn, c, b, n, r, dtype, seed=Tn + c + 1, order=order)
    V = ref_forward(X, W, A, B, index, scale)[1].float()
    dX, dA, dB = T.adapter_backward(dY, X, V, W, A, B, index, scale, check=True)
    rX, rA, rB = ref_backward(dY, X, V, W, A, B, index, scale)
    assert rel(dX, rX) <= (TOL_BF16 if dtype == torch.bfloat16 else TOL_F32)
    assert rel(dA, rA) <= TOL_F32 and rel(dB, rB) <= TOL_F32
    for i in range(n):   # every adapter on its own; exact zeros without tokens
        if not bool((index == i).any()):
            assert bool((dA[i] == 0).all()) and bool((dB[i] == 0).all())
        else:
            assert rel(dA[i], rA[i]) <= 2 * TOL_F32 and rel(dB[i], rB[i]) <= 2 * TOL_F32
    # accumulate adds to what is there; the parts can be had on their own
    seedA, seedB = torch.randn_like(dA), torch.randn_like(dB)
    accA, accB = seedA.clone(), seedB.clone()
    nx, gA, gB = T.adapter_backward(dY, X, V, W, A, B, index, scale, need_dx=False, dA=accA, dB=accB,
                                    accumulate=True, check=True)
    assert nx is None and gA is accA
    assert rel(accA - seedA, rA) <= 4 * TOL_F32 + (2e-7 * seedA.norm() / rA.norm().clamp(min=1e-30)).item() \
        or rA.norm() == 0
    assert rel(accB, seedB.double() + rB) <= TOL_F32
    only, gA, gB = T.adapter_backward(dY, None, None, W, A, B, index, scale, need_grads=False)
    assert gA is None and gB is None and torch.equal(only, dX)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
def test_adapter_strides_and_padding_are_left_alone(T, dtype):
    """Rows with a stride: inputs are read in place, the gaps of outputs are not written."""
    Tn, c, b, n, r = 200, 201, 328, 4, 12
    X, W, A, B, index, scale, dY = make(Tn, c, b, n, r, dtype, seed=3, pad=24)
    assert X.stride(0) == b + 24
    big = torch.full((Tn, c + 7), 7.0, dtype=dtype, device=DEV)
    Y, V = T.adapter_forward(X, W, A, B, index, scale, out=big[:, :c], check=True)
    Y2, V2 = T.adapter_forward(X.contiguous(), W.contiguous(), A, B, index, scale)
    assert torch.equal(Y, Y2) and torch.equal(V, V2) and bool((big[:, c:] == 7.0).all())
    dbig = torch.full((Tn, b + 3), 5.0, dtype=dtype, device=DEV)
    wide = torch.zeros((Tn, c + 5), dtype=dtype, device=DEV)
    wide[:, :c] = dY
    g1 = T.adapter_backward(wide[:, :c], X, V, W, A, B, index, scale, dX=dbig[:, :b], check=True)
    g2 = T.adapter_backward(dY, X.contiguous(), V, W.contiguous(), A, B, index, scale)
    for u, v in zip(g1, g2):
        assert torch.equal(u, v)
    assert bool((dbig[:, b:] == 5.0).all())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
def test_adapter_foreign_values_stay_out(T, dtype):
    """An adapter with infinities or NaN reaches its own tokens alone, and a token's NaN only its own
    row and its own adapter's gradients."""
    Tn, c, b, n, r = 96, 200, 264, 6, 12
    X, W, A, B, index, scale, dY = make(Tn, c, b, n, r, dtype, seed=5)
    A[2], B[3, :, 4] = float("nan"), float("inf")
    good = (index != 2) & (index != 3)
    Y, V = T.adapter_forward(X, W, A, B, index, scale, check=True)
    assert bool(torch.isfinite(Y[good]).all()) and bool(torch.isnan(V[index == 2]).all())
    keep = torch.tensor([0, 1, 4, 5], device=DEV)
    Yr, Vr = ref_forward(X[good], W, A, B, index[good], scale)
    assert rel(Y[good], Yr) <= (TOL_BF16 if dtype == torch.bfloat16 else TOL_F32)
    V = torch.where(torch.isfinite(V), V, 0.0)
    dX, dA, dB = T.adapter_backward(dY, X, V, W, A, B, index, scale, check=True)
    assert bool(torch.isfinite(dX[good]).all())
    assert bool(torch.isfinite(dA[keep]).all()) and bool(torch.isfinite(dB).all())
    # a poisoned token
    X2, dY2 = X.clone(), dY.clone()
    t = int((index == 0).nonzero()[0])
    X2[t], dY2[t] = float("nan"), float("inf")
    Y2, V2 = T.adapter_forward(X2, W, A, B, index, scale)
    rest = good.clone()
    rest[t] = False
    assert bool(torch.isnan(Y2[t]).all()) and torch.equal(Y2[rest], Y[rest])
    dX2, dA2, dB2 = T.adapter_backward(dY2, X2, V, W, A, B, index, scale)
    assert torch.equal(dX2[rest], dX[rest])
    for i in (1, 4, 5):
        assert torch.equal(dA2[i], dA[i]) and torch.equal(dB2[i], dB[i])


def test_adapter_empty_calls_and_no_adapters(T):
    X, W, A, B, index, scale, dY = make(40, 96, 128, 3, 8, torch.bfloat16, seed=9)
    Y, V = T.adapter_forward(X, W, check=True)
    assert V is None and rel(Y, X.double() @ W.double().T) <= TOL_BF16
    dX, dA, dB = T.adapter_backward(dY, X, None, W, check=True)
    assert dA is None and rel(dX, dY.double() @ W.double()) <= TOL_BF16
    Y0, V0 = T.adapter_forward(X[:0], W, A, B, index[:0], scale, check=True)
    assert Y0.shape == (0, 96) and V0.shape == (0, 8)
    dX0, dA0, dB0 = T.adapter_backward(dY[:0], X[:0], V0, W, A, B, index[:0], scale, check=True)
    assert dX0.shape == (0, 128) and bool((dA0 == 0).all()) and bool((dB0 == 0).all())


def test_adapter_index_out_of_range_is_reported(T):
    X, W, A, B, index, scale, _ = make(70, 96, 128, 3, 8, torch.bfloat16, seed=10)
    bad = index.clone()
    bad[5], bad[66] = 3, -2
    with pytest.raises(T.ThanosError) as e:
        T.adapter_forward(X, W, A, B, bad, scale, check=True)
    assert e.value.code == 1
    Y, V = T.adapter_forward(X, W, A, B, bad, scale)     # taken as "no adapter"
    index[5], index[66] = -1, -1
    Y2, V2 = T.adapter_forward(X, W, A, B, index, scale, check=True)
    assert torch.equal(Y, Y2) and torch.equal(V, V2)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
def test_adapter_results_repeat_and_streams(T, dtype):
    """The same bits on every run, on another stream, and with a dirty workspace."""
    X, W, A, B, index, scale, dY = make(600, 640, 520, 10, 16, dtype, seed=11)
    Y, V = T.adapter_forward(X, W, A, B, index, scale)
    g = T.adapter_backward(dY, X, V, W, A, B, index, scale)
    torch.cuda.synchronize()
    st = torch.cuda.Stream()
    lib = T.load_library()
    dt = 1 if dtype == torch.bfloat16 else 0
    for k in range(3):
        ws = torch.full((lib.thanos_adapter_workspace_bytes(0, 600, 640, 520, 10, 16, dt),), 255,
                        dtype=torch.uint8, device=DEV)
        ws2 = torch.full((lib.thanos_adapter_workspace_bytes(1, 600, 640, 520, 10, 16, dt),), 255,
                         dtype=torch.uint8, device=DEV)
        torch.cuda.synchronize()
        Y2, V2 = T.adapter_forward(X, W, A, B, index, scale, stream=st, workspace=ws)
        g2 = T.adapter_backward(dY, X, V2, W, A, B, index, scale, stream=st, workspace=ws2)
        st.synchronize()
        assert torch.equal(Y, Y2) and torch.equal(V, V2)
        assert all(torch.equal(u, v) for u, v in zip(g, g2))


def test_adapter_gradients_against_differences(T):
    """d/deps of sum(Y * dY) by central differences in fp32 with a step of 2^-4: the loss is bilinear
    in each of X, A and B alone, so the difference quotient is exact up to rounding."""
    X, W, A, B, index, scale, dY = make(50, 72, 64, 3, 6, torch.float32, seed=12)
    Y, V = T.adapter_forward(X, W, A, B, index, scale)
    dX, dA, dB = T.adapter_backward(dY, X, V, W, A, B, index, scale)

    def loss(X_, A_, B_):
        return (T.adapter_forward(X_, W, A_, B_, index, scale)[0].double() * dY.double()).sum().item()

    g = torch.Generator(device=DEV).manual_seed(1)
    for grad, k in ((dX, 0), (dA, 1), (dB, 2)):
        d = torch.randn(grad.shape, generator=g, device=DEV)
        args = [X, A, B]
        h = 2.0 ** -4
        up = loss(*[a + h * d if j == k else a for j, a in enumerate(args)])
        dn = loss(*[a - h * d if j == k else a for j, a in enumerate(args)])
        num, ana = (up - dn) / (2 * h), (grad.double() * d.double()).sum().item()
        assert abs(num - ana) <= 2e-4 * grad.double().norm().item() * d.double().norm().item() / math.sqrt(
            grad.numel()) + 1e-4 * abs(ana)


# --------------------------------------------------------------------------- orthogonalised update
COEF = (3.4445, -4.7750, 2.0315)


def ref_ns(G, steps=5, coef=COEF, eps=1e-7):
    a, b, c = coef
    X = G.double()
    tall = X.shape[-2] > X.shape[-1]
    if tall:
        X = X.mT
    X = X / (torch.linalg.matrix_norm(X, keepdim=True) + eps)
    for _ in range(steps):
        S = X @ X.mT
        X = a * X + (b * S + c * (S @ S)) @ X
    return X.mT if tall else X


def spectrum(kind, k, m, n, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    rn = lambda *s: torch.randn(s, generator=g, device=DEV)  # noqa: E731
    q = max(1, min(m, n) // 16)
    if kind == "flat":
        return 1e-3 * rn(k, m, n)
    if kind == "lead":     # few strong directions over a floor
        return 1e-3 * (rn(k, m, q) @ rn(k, q, n) + 0.05 * rn(k, m, n))
    if kind == "low rank":
        return rn(k, m, q) @ rn(k, q, n)
    if kind == "tiny":
        return 1e-12 * rn(k, m, n)
    if kind == "huge":
        return 1e15 * rn(k, m, n)
    raise KeyError(kind)


ORTHO = [(1, 1, 1), (1, 1, 50), (3, 7, 3), (1, 16, 4096), (5, 16, 100), (2, 300, 33), (1, 64, 64),
         (2, 65, 130), (4, 128, 768), (1, 129, 127), (1, 256, 256), (2, 300, 500), (1, 511, 1030),
         (1, 768, 768), (1, 1001, 520), (1, 1500, 700), (1, 640, 2600)]


@pytest.mark.parametrize("kind", ["flat", "lead", "low rank"])
@pytest.mark.parametrize("shape", ORTHO, ids=lambda s: "x".join(map(str, s)))
def test_orthogonalise(T, shape, kind):
    G = spectrum(kind, *shape, seed=shape[1] * 31 + shape[2])
    for dtype in (torch.float32, torch.bfloat16):
        Gd = G.to(dtype)
        O = T.orthogonalise(Gd, check=True)
        assert O.dtype == torch.bfloat16 and O.shape == Gd.shape
        ref = ref_ns(Gd)
        for i in range(shape[0]):
            assert rel(O[i], ref[i]) <= TOL_ORTHO
    if shape[0] == 1:
        assert torch.equal(T.orthogonalise(Gd[0]), O[0])


def test_orthogonalise_scales_zero_and_other_polynomials(T):
    for shape in ((1, 48, 300), (1, 300, 260)):
        for kind in ("tiny", "huge"):
            G = spectrum(kind, *shape, seed=2)
            assert rel(T.orthogonalise(G, check=True), ref_ns(G)) <= TOL_ORTHO
        z = torch.zeros(shape, device=DEV)
        assert bool((T.orthogonalise(z, check=True) == 0).all())
        G = spectrum("flat", *shape, seed=3)
        cubic = (1.5, -0.5, 0.0)
        O = T.orthogonalise(G, steps=9, coef=cubic, check=True)
        assert rel(O, ref_ns(G, 9, cubic)) <= TOL_ORTHO
        G2 = torch.cat([G, G, G])
        G2[1, 0, 5] = float("nan")
        O2 = T.orthogonalise(G2, check=True)      # its neighbours in the batch stay as they are
        assert bool(torch.isnan(O2[1]).any())
        one = T.orthogonalise(G)
        assert torch.equal(O2[0], one[0]) and torch.equal(O2[2], one[0])


STEPS = [(1, 16, 1024), (3, 24, 200), (1, 200, 24), (1, 129, 260), (1, 768, 768), (2, 320, 513),
         (1, 1001, 520)]


@pytest.mark.parametrize("mask", ["none", "2:4", "half", "all", "rows"])
@pytest.mark.parametrize("shape", STEPS, ids=lambda s: "x".join(map(str, s)))
def test_orthogonal_step(T, shape, mask):
    k, m, n = shape
    g = torch.Generator(device=DEV).manual_seed(k + m + n)
    u = torch.rand(shape, generator=g, device=DEV)
    if mask == "none":
        mk = None
    elif mask == "2:4":
        mk = ((torch.arange(n, device=DEV) % 4) < 2).to(torch.uint8).expand(shape).contiguous()
    elif mask == "half":
        mk = (u < 0.5).to(torch.uint8)
    elif mask == "all":
        mk = torch.ones(shape, dtype=torch.uint8, device=DEV)
    else:      # whole rows gone, the last one among them
        mk = torch.zeros(shape, dtype=torch.uint8, device=DEV)
        mk[:, ::3], mk[:, -1] = 1, 1
    gone = torch.zeros(shape, dtype=torch.bool, device=DEV) if mk is None else mk != 0
    for wd, gd, nesterov in ((torch.float32, torch.float32, True),
                             (torch.bfloat16, torch.bfloat16, True),
                             (torch.float32, torch.bfloat16, False)):
        W = torch.where(gone, 0.0, 0.02 * torch.randn(shape, generator=g, device=DEV)).to(wd)
        M = torch.where(gone, 0.0, 3e-3 * torch.randn(shape, generator=g, device=DEV))
        G = spectrum("lead", k, m, n, seed=m).to(gd)
        Gp = G.clone()
        if mk is not None:       # what a removed place holds does not matter
            Gp[gone] = float("nan")
        lr, gain, mu, wdec = 1e-2, 0.2 * math.sqrt(max(m, n)), 0.9, 0.1
        W2, M2 = T.orthogonal_step(W, M, Gp, mk, lr=lr, gain=gain, momentum=mu, nesterov=nesterov,
                                   weight_decay=wdec, check=True)
        gf = torch.where(gone, 0.0, G.double())
        Mr = mu * M.double() + gf
        upd = torch.where(gone, 0.0, gf + mu * Mr if nesterov else Mr)
        O = ref_ns(upd)
        Wr = torch.where(gone, 0.0, (1 - lr * wdec) * W.double() - lr * gain * O)
        assert rel(M2, Mr) <= 1e-6
        assert bool((W2[gone] == 0).all()) and bool((M2[gone] == 0).all())
        if mask != "all":
            moved = W2.double() - (1 - lr * wdec) * W.double()
            want = Wr - (1 - lr * wdec) * W.double()
            # fp16 products without the last rounding to bf16, or the weights' own rounding
            lim = 2.5e-3 if wd == torch.float32 else 0
            if lim:
                assert rel(moved, want) <= lim
            assert rel(W2, Wr) <= (2e-3 if wd == torch.bfloat16 else 1e-3)
        # in place, and the same bits again
        Wi, Mi = W.clone(), M.clone()
        T.orthogonal_step(Wi, Mi, Gp, mk, lr=lr, gain=gain, momentum=mu, nesterov=nesterov,
                          weight_decay=wdec, W_out=Wi, M_out=Mi)
        assert torch.equal(Wi, W2) and torch.equal(Mi, M2)


def test_orthogonal_results_on_another_stream_and_dirty_workspace(T):
    lib = T.load_library()
    for shape in ((3, 16, 500), (1, 384, 640)):
        G = spectrum("flat", *shape, seed=4)
        O = T.orthogonalise(G)
        torch.cuda.synchronize()
        ws = torch.full((lib.thanos_orthogonal_workspace_bytes(*shape),), 255, dtype=torch.uint8,
                        device=DEV)
        torch.cuda.synchronize()
        st = torch.cuda.Stream()
        for _ in range(3):
            O2 = T.orthogonalise(G, stream=st, workspace=ws)
            st.synchronize()
            assert torch.equal(O, O2)


# --------------------------------------------------------------------------------------- refusals
def test_recovery_refusals(T):
    X, W, A, B, index, scale, dY = make(8, 64, 64, 2, 4, torch.bfloat16, seed=1)
    before = T.launch_count()
    with pytest.raises(ValueError):
        T.adapter_forward(X, W.float(), A, B, index, scale)
    with pytest.raises(ValueError):
        T.adapter_forward(X, W, A, B[:, :-1].contiguous(), index, scale)
    with pytest.raises(ValueError):
        T.adapter_forward(X, W, A, B, index.long(), scale)
    with pytest.raises(ValueError):
        T.adapter_forward(X.t(), W, A, B, index, scale)
    with pytest.raises(TypeError):
        T.adapter_forward(X.half(), W.half(), A.half(), B.half(), index, scale)
    with pytest.raises(ValueError):
        T.adapter_forward(X, W, A, B, index[:4].contiguous(), scale)
    odd = torch.zeros((8, 64 + 4), dtype=torch.bfloat16, device=DEV)[:, :64]
    with pytest.raises(T.ThanosError) as e:
        T.adapter_forward(odd, W, A, B, index, scale)          # row stride not a multiple of 8
    assert e.value.code == 4
    with pytest.raises(T.ThanosError) as e:
        T.adapter_forward(X, W, A, B, index, scale,
                          workspace=torch.zeros(16, dtype=torch.uint8, device=DEV))
    assert e.value.code == 5
    with pytest.raises(T.ThanosError) as e:
        T.adapter_forward(X[:, :60].contiguous(), W[:, :60].contiguous(),
                          A[:, :, :60].contiguous(), B, index, scale)
    assert e.value.code == 2
    big = torch.zeros((1, 129, 64), dtype=torch.bfloat16, device=DEV)
    with pytest.raises(T.ThanosError) as e:
        T.adapter_forward(X, W, big, torch.zeros((1, 64, 129), dtype=torch.bfloat16, device=DEV),
                          index, scale[:1].contiguous())
    assert e.value.code == 2
    with pytest.raises(ValueError):
        T.adapter_backward(dY, None, None, W, A, B, index, scale)
    with pytest.raises(ValueError):
        T.adapter_backward(dY, X, torch.zeros((8, 4), device=DEV), W, A, B, index, scale,
                           accumulate=True)
    G = torch.zeros((32, 64), device=DEV)
    with pytest.raises(ValueError):
        T.orthogonalise(G.t())
    with pytest.raises(T.ThanosError) as e:
        T.orthogonalise(G, steps=0)
    assert e.value.code == 1
    with pytest.raises(T.ThanosError) as e:
        T.orthogonalise(G, coef=(float("nan"), 0.0, 0.0))
    assert e.value.code == 1
    with pytest.raises(ValueError):
        T.orthogonal_step(G, G.bfloat16(), G)
    with pytest.raises(ValueError):
        T.orthogonal_step(G, G, G, mask=torch.zeros((32, 63), dtype=torch.uint8, device=DEV))
    assert T.launch_count() == before     # nothing was launched by any of them
