"""Values at the ends of the types: infinities, NaN, the largest numbers, against float64, where they
stand and what sign they have; finite rows beside them keep their accuracy.

Tolerances as in test_recovery_gpu.py (sums in fp32: 1e-5, a rounding to bf16: 3e-3)."""

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from tests.test_recovery_gpu import TOL_F32, make, ref_backward, ref_forward  # noqa: E402

DEV = "cuda"
BF16, F32 = torch.bfloat16, torch.float32
INF, NAN, LARGE = float("inf"), float("nan"), 3.4e38   # LARGE is above bf16's largest, 3.39e38


@pytest.fixture(scope="module")
def T():
    import paper_2504_05346_b200 as T_
    from paper_2504_05346_b200 import build as B_

    B_.build()
    T_.load_library()
    return T_


def same_rows(x, ref, tol):
    """Infinities and NaN as in the reference, rounded to the result's type (what no fp32 number is near
    is an infinity there too), the rest close to it, row by row."""
    ref = ref.to(x.dtype).double().reshape(ref.shape[0], -1)
    x = x.double().reshape(ref.shape[0], -1)
    for kind in (torch.isnan, torch.isposinf, torch.isneginf):
        assert torch.equal(kind(x), kind(ref))
    fin = torch.isfinite(ref)
    d = torch.where(fin, x - ref, 0.0).norm(dim=1)
    assert bool((d <= tol * torch.where(fin, ref, 0.0).norm(dim=1)).all())


def strange(X):
    """Rows with an infinity, two of them, a NaN, and a number that no bf16 is near; a plain one last."""
    X[1, 5], X[2, 5], X[2, 9], X[3, 2], X[4, 1] = INF, -INF, INF, NAN, LARGE
    X[5, 1], X[6] = -LARGE, 0.0
    X[6, 3] = -INF
    return X


# ranks and tokens that take the skinny product on the ALUs and, from 2^14 and 2^16 on, on the tensor
# cores; rows of whole vectors and others (c is the length of the backward sums)
@pytest.mark.parametrize("shape", [(40, 136, 72, 3, 4), (300, 131, 200, 2, 20), (2100, 136, 264, 3, 32),
                                   (2100, 133, 72, 3, 33)], ids=lambda s: "x".join(map(str, s)))
def test_f32_values(T, shape):
    Tn, c, b, n, r = shape
    X, W, A, B, index, scale, dY = make(Tn, c, b, n, r, F32, seed=Tn + r)
    W[W == 0] = 0.01
    index[:7] = torch.tensor([0, -1, 0, 1, 0, -1, -1], device=DEV)
    X, dY = strange(X.clone()), strange(dY.clone())
    for w in (W, W.clone()):
        if w is not W:            # and an infinite weight, which meets an infinite value in row 1
            w[7, 11], w[9, 5], w[5, 8] = INF, -INF, INF
        Y, V = T.adapter_forward(X, w, A, B, index, scale, check=True)
        Yr, Vr = ref_forward(X, w, A, B, index, scale)
        same_rows(V, Vr, 3 * TOL_F32)
        same_rows(Y, Yr, 3 * TOL_F32)
        dX, _, _ = T.adapter_backward(dY, X, Vr.float(), w, A, B, index, scale, check=True)
        same_rows(dX, ref_backward(dY, X, Vr, w, A, B, index, scale)[0], 3 * TOL_F32)
    # the narrow factors
    A2, B2 = A.clone(), B.clone()
    A2[0, 1, 4], B2[1, 3, 2], A2[1, 0, 0] = INF, -INF, LARGE
    _, V = T.adapter_forward(X, W, A2, B, index, scale)
    same_rows(V, ref_forward(X, W, A2, B, index, scale)[1], 3 * TOL_F32)
    dX, _, _ = T.adapter_backward(dY, X, Vr.float(), W, A, B2, index, scale)
    same_rows(dX, ref_backward(dY, X, Vr, W, A, B2, index, scale)[0], 3 * TOL_F32)


@pytest.mark.parametrize("shape", [(5, 136, 72, 5, 4), (40, 136, 72, 5, 4), (300, 131, 200, 5, 20),
                                   (2100, 1290, 1544, 5, 12), (700, 264, 136, 5, 100)],
                         ids=lambda s: "x".join(map(str, s)))
def test_bf16_values(T, shape):
    """The gradients' factor is three planes that meet the activations one by one."""
    Tn, c, b, n, r = shape
    X, W, A, B, index, scale, dY = make(max(Tn, 7), c, b, n, r, BF16, seed=Tn + r)
    index[:7] = torch.tensor([0, 1, 2, 3, 4, 0, 1], device=DEV)
    W[W == 0], B[B == 0], A[A == 0] = 0.01, 0.01, 0.01
    lim = 6e-3     # a rounding of the result, one of the adapter's factor, row by row
    for bad_x, bad_y in ((True, False), (False, True), (True, True)):
        X2, dY2 = X.clone(), dY.clone()
        if bad_x:
            strange(X2)
            X2[4, 1], X2[5, 1] = 3.3e38, -3.3e38    # nearest bf16 of LARGE would be an infinity
        if bad_y:
            strange(dY2)
            dY2[4, 1], dY2[5, 1] = 3.3e38, -3.3e38
        Y, V = T.adapter_forward(X2[:Tn], W, A, B, index[:Tn], scale, check=True)
        Yr, Vr = ref_forward(X2[:Tn], W, A, B, index[:Tn], scale)
        same_rows(V, Vr, 3 * TOL_F32)
        same_rows(Y, Yr, lim)
        Vf = Vr.float()
        dX, dA, dB = T.adapter_backward(dY2[:Tn], X2[:Tn], Vf, W, A, B, index[:Tn], scale, check=True)
        rX, rA, _ = ref_backward(dY2[:Tn], X2[:Tn], Vf, W, A, B, index[:Tn], scale)
        # dB = s_i times an fp32 sum, which may be an infinity where the product would not
        rB = ref_backward(dY2[:Tn], X2[:Tn], Vf, W, A, B, index[:Tn], torch.ones_like(scale))[2]
        rB = rB.float().double() * scale.double()[:, None, None]
        same_rows(dX, rX, lim)
        same_rows(dA, rA, 3 * TOL_F32)
        same_rows(dB, rB, 3 * TOL_F32)


def iterate(G, eps, steps=5, coef=(3.4445, -4.7750, 2.0315)):
    a, b, c = coef
    X = G.double()
    tall = X.shape[-2] > X.shape[-1]
    X = X.mT if tall else X
    X = X / (torch.linalg.matrix_norm(X, keepdim=True) + eps)
    for _ in range(steps):
        S = X @ X.mT
        X = a * X + (b * S + c * (S @ S)) @ X
    return X.mT if tall else X


# sides of up to 16, 32 and 64, and beyond, where other kernels take the norm; several chunks
MATRICES = [(3, 16, 4096), (1, 9000, 20), (1, 48, 300), (2, 64, 1000), (1, 7, 3), (1, 300, 260), (2, 65, 130)]


@pytest.mark.parametrize("scale", [1e19, 1e25, 1e37, 1e-18, 1e-25, 1e-35])
@pytest.mark.parametrize("shape", MATRICES, ids=lambda s: "x".join(map(str, s)))
def test_update_of_matrices_whose_squares_leave_fp32(T, shape, scale):
    """fp16 operands and a bf16 result: 4e-3, as for every matrix; fp32 weights 4e-4 (at the ends of
    fp32 the reciprocal of the norm has at least 14 bits)."""
    gen = torch.Generator(device=DEV).manual_seed(23)
    G = torch.randn(shape, generator=gen, device=DEV) * scale
    mixed = G.clone()          # chunks of another size, some of nothing: the first part decides
    half = shape[2] // 2 if shape[2] >= shape[1] else shape[1] // 2
    if shape[2] >= shape[1]:
        mixed[..., half:] *= 1e-8
        mixed[..., 3 * half // 2:] = 0
    else:
        mixed[:, half:] *= 1e-8
        mixed[:, 3 * half // 2:] = 0
    for M in (G, mixed):
        for eps in (0.0, 1e-7 * scale):
            eps = torch.tensor(eps).item()
            ref = iterate(M, eps)
            O = T.orthogonalise(M, eps=eps, check=True)
            W, _ = T.orthogonal_step(torch.zeros_like(M), torch.zeros_like(M), M, lr=1.0, momentum=0.0,
                                     eps=eps, check=True)
            for i in range(shape[0]):
                n = ref[i].norm()
                assert (O[i].double() - ref[i]).norm() <= 4e-3 * n
                assert (W[i].double() + ref[i]).norm() <= 4e-4 * n


@pytest.mark.parametrize("shape", MATRICES, ids=lambda s: "x".join(map(str, s)))
def test_update_of_zeros_and_of_what_is_not_finite(T, shape):
    z = torch.zeros(shape, device=DEV)
    assert not T.orthogonalise(z, check=True).any()
    for bad in (INF, NAN):
        G = torch.randn(shape, device=DEV)
        G[0, -1, -1] = bad
        O = T.orthogonalise(G, check=True)
        assert torch.isnan(O[0].float()).all()
        assert torch.isfinite(O[1:].float()).all()
