"""The recovery operators where the products run on pairs of SMs (37 tiles of 256 x 256 and more, as
layers and prompts have them), with edges that are no whole tiles, warps or 16-byte vectors, against
the float64 formulas.

Tolerances as in test_recovery_gpu.py: one rounding to bf16 and the same again for the adapter part
(3e-3), sums in fp32 (1e-5 and, where infinities are compared, their places and signs), fp16 operands
and a bf16 result (4e-3), weights as there.  Outputs are passed in full of NaN."""

import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from tests.test_recovery_gpu import (TOL_BF16, TOL_F32, TOL_ORTHO, make, ref_backward,  # noqa: E402
                                     ref_forward, ref_ns, rel)
from tests.test_recovery_step_gpu import TOL_FINE  # noqa: E402

DEV = "cuda"
BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def T():
    import paper_2504_05346_b200 as T_
    from paper_2504_05346_b200 import build as B_

    B_.build()
    T_.load_library()
    return T_


def nan(*shape, dtype=F32):
    return torch.full(shape, float("nan"), dtype=dtype, device=DEV)


def forward(T, X, W, A, B, index, scale, check=True):
    return T.adapter_forward(X, W, A, B, index, scale, check=check,
                             out=nan(X.shape[0], W.shape[0], dtype=X.dtype),
                             V=nan(X.shape[0], A.shape[1]))


def backward(T, dY, X, V, W, A, B, index, scale, check=True):
    return T.adapter_backward(dY, X, V, W, A, B, index, scale, check=check,
                              dX=nan(X.shape[0], W.shape[1], dtype=X.dtype), dA=nan(*A.shape),
                              dB=nan(*B.shape))


# tokens, outputs, inputs, adapters, rank, order: 54 tiles and more in each direction
SHAPES = [(2100, 1290, 1544, 6, 12, "mixed"), (2100, 1290, 1544, 6, 24, "blocks"),
          (2100, 1290, 1544, 6, 128, "mixed"), (2500, 2049, 1032, 300, 8, "mixed"),
          (2057, 1281, 1288, 9, 5, "mixed"), (2304, 2304, 1280, 2, 40, "blocks"),
          (2100, 1400, 1544, 4, 16, "none"), (5000, 516, 520, 1, 1, "one")]


@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_projection_on_pairs(T, shape):
    Tn, c, b, n, r, order = shape
    X, W, A, B, index, scale, dY = make(Tn, c, b, n, r, BF16, seed=c + r, order=order, pad=8)
    Y, V = forward(T, X, W, A, B, index, scale)
    Yr, Vr = ref_forward(X, W, A, B, index, scale)
    assert rel(Y, Yr) <= TOL_BF16 and rel(V, Vr) <= TOL_F32
    assert bool((V[index < 0] == 0).all())
    err = (Y.double() - Yr).norm(dim=1) / Yr.norm(dim=1)     # every token on its own
    assert err.max().item() <= 2 * TOL_BF16
    dX, dA, dB = backward(T, dY, X, V, W, A, B, index, scale)
    rX, rA, rB = ref_backward(dY, X, V, W, A, B, index, scale)
    assert rel(dX, rX) <= TOL_BF16 and rel(dA, rA) <= TOL_F32 and rel(dB, rB) <= TOL_F32
    err = (dX.double() - rX).norm(dim=1) / rX.norm(dim=1)
    assert err.max().item() <= 2 * TOL_BF16
    # the same bits again
    assert torch.equal(forward(T, X, W, A, B, index, scale)[0], Y)
    assert torch.equal(backward(T, dY, X, V, W, A, B, index, scale)[0], dX)


def test_index_out_of_range_on_pairs(T):
    X, W, A, B, index, scale, dY = make(2100, 1290, 1544, 6, 12, BF16, seed=7)
    bad = index.clone()
    bad[3], bad[2099] = 6, -7
    index[3], index[2099] = -1, -1
    Y, V = forward(T, X, W, A, B, index, scale)
    for call in (lambda: forward(T, X, W, A, B, bad, scale),
                 lambda: backward(T, dY, X, V, W, A, B, bad, scale)):
        with pytest.raises(T.ThanosError) as e:
            call()
        assert e.value.code == 1
    Y2, V2 = forward(T, X, W, A, B, bad, scale, check=False)
    assert torch.equal(Y, Y2) and torch.equal(V, V2)
    for u, v in zip(backward(T, dY, X, V, W, A, B, index, scale),
                    backward(T, dY, X, V, W, A, B, bad, scale, check=False)):
        assert torch.equal(u, v)


def same_values(x, ref, tol):
    """Infinities and NaN in the reference's places, and the rest close to it."""
    for kind in (torch.isnan, torch.isposinf, torch.isneginf):
        assert torch.equal(kind(x.double()), kind(ref))
    fin = torch.isfinite(ref)
    assert rel(torch.where(fin, x.double(), 0.0), torch.where(fin, ref, 0.0)) <= tol


@pytest.mark.parametrize("r", [12, 16])
def test_values_that_are_not_finite_stay_with_their_tokens_on_pairs(T, r):
    Tn, c, b, n = 2100, 1290, 1544, 6
    X, W, A, B, index, scale, dY = make(Tn, c, b, n, r, BF16, seed=11 + r)
    inf = float("inf")
    # forward: one adapter whose wide factor has infinities and NaN, one whose V is NaN
    B2, A2 = B.clone(), A.clone()
    B2[3, ::7, 4], B2[3, 5::7, 2], A2[2, 1, 9] = -inf, float("nan"), float("nan")
    t = int((index == 0).nonzero()[0])
    X2 = X.clone()
    X2[t] = float("nan")
    Y, V = forward(T, X2, W, A2, B2, index, scale)
    Yr, Vr = ref_forward(X2, W, A2, B2, index, scale)
    same_values(V, Vr, TOL_F32)
    same_values(Y, Yr, TOL_BF16)
    # backward: there A is the wide factor
    A2 = A.clone()
    A2[2, 1, ::9], A2[2, 3, 4::9] = inf, float("nan")
    V = ref_forward(X, W, A, B, index, scale)[1].float()
    dX, dA, dB = backward(T, dY, X, V, W, A2, B, index, scale)
    rX, rA, rB = ref_backward(dY, X, V, W, A2, B, index, scale)
    same_values(dX, rX, TOL_BF16)
    assert rel(dA, rA) <= TOL_F32 and rel(dB, rB) <= TOL_F32
    # and a poisoned token: its own row, its own adapter's gradients
    dY2, X2 = dY.clone(), X.clone()
    dY2[t], X2[t] = float("nan"), inf
    clean = backward(T, dY, X, V, W, A, B, index, scale)
    dX, dA, dB = backward(T, dY2, X2, V, W, A, B, index, scale)
    rest = torch.arange(Tn, device=DEV) != t
    assert bool(torch.isnan(dX[t]).all()) and torch.equal(dX[rest], clean[0][rest])
    assert torch.equal(dA[1:], clean[1][1:]) and torch.equal(dB[1:], clean[2][1:])


MATRICES = [(2100, 2304), (2304, 2100), (2310, 2104), (2097, 2210), (4500, 1290)]


@pytest.mark.parametrize("shape", MATRICES, ids=lambda s: "x".join(map(str, s)))
def test_update_on_pairs(T, shape):
    gen = torch.Generator(device=DEV).manual_seed(shape[0])
    G = 1e-3 * torch.randn(shape, generator=gen, device=DEV)
    for dtype in (F32, BF16):
        Gd = G.to(dtype)
        assert rel(T.orthogonalise(Gd, out=nan(*shape, dtype=BF16), check=True), ref_ns(Gd)) <= TOL_ORTHO


@pytest.mark.parametrize("wd", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("kind", ["none", "2:4", "half", "rows"])
@pytest.mark.parametrize("shape", MATRICES, ids=lambda s: "x".join(map(str, s)))
def test_masked_step_on_pairs(T, shape, kind, wd):
    m, n = shape
    gen = torch.Generator(device=DEV).manual_seed(m + n)
    rn = lambda: torch.randn(shape, generator=gen, device=DEV)  # noqa: E731
    gone = torch.zeros(shape, dtype=torch.bool, device=DEV)
    if kind == "2:4":
        gone[:, torch.arange(n, device=DEV) % 4 < 2] = True
    elif kind == "half":
        gone = rn() < 0
    elif kind == "rows":
        gone[::3], gone[-1] = True, True
    mask = None if kind == "none" else gone.to(torch.uint8)
    W = torch.where(gone, 0.0, 0.02 * rn()).to(wd)
    M = torch.where(gone, 0.0, 3e-3 * rn())
    G = (1e-3 * rn()).to(wd)
    Gp = torch.where(gone, float("nan"), G.float()).to(wd)    # what a removed place holds: anything
    lr, gain, mu, dec = 1e-2, 0.2 * math.sqrt(max(m, n)), 0.9, 0.1
    Wi, Mi = W.clone(), M.clone()
    T.orthogonal_step(Wi, Mi, Gp, mask, lr=lr, gain=gain, momentum=mu, weight_decay=dec, W_out=Wi,
                      M_out=Mi, check=True)
    g = torch.where(gone, 0.0, G.double())
    Mr = mu * M.double() + g
    keep = (1 - lr * dec) * W.double()
    Wr = torch.where(gone, 0.0, keep - lr * gain * ref_ns(torch.where(gone, 0.0, g + mu * Mr)))
    assert rel(Mi, Mr) <= 1e-6 and bool((Wi[gone] == 0).all())
    if wd == F32:
        assert rel(Wi.double() - keep, Wr - keep) <= TOL_FINE + 2e-5   # 2^-24 of W, 1000 times a step
    else:
        assert rel(Wi, Wr) <= 2e-3
    Wo, Mo = T.orthogonal_step(W, M, Gp, mask, lr=lr, gain=gain, momentum=mu, weight_decay=dec,
                               W_out=nan(*shape, dtype=wd), M_out=nan(*shape))
    assert torch.equal(Wo, Wi) and torch.equal(Mo, Mi)


@pytest.mark.parametrize("shape", SHAPES[:6] + [(40, 1290, 1544, 6, 12, "mixed")],
                         ids=lambda s: "x".join(map(str, s)))
def test_adapter_part_is_rounded_once_whatever_the_batch(T, shape):
    """Without the frozen part, every entry of a bf16 result is within half a unit of itself (8 bits: at
    most 2^-8 of it) and 2^-14 of its terms' magnitudes: 2^-16 for two planes of the factor, the rest for fp32 sums."""
    Tn, c, b, n, r, order = shape
    X, W, A, B, index, scale, dY = make(Tn, c, b, n, r, BF16, seed=c + r, order=order)
    W = torch.zeros_like(W)
    D = torch.float64
    i = index.long().clamp(min=0)
    s = torch.where(index >= 0, scale[i], 0.0).to(D)[:, None]

    def terms(v, wide):     # sum over ranks of factor times wide, and of their magnitudes
        out = torch.zeros(Tn, wide.shape[1], dtype=D, device=DEV)
        size = torch.zeros_like(out)
        for k in range(n):
            own = (index == k).nonzero()[:, 0]
            out[own] = v[own] @ wide[k].to(D).T
            size[own] = v[own].abs() @ wide[k].to(D).T.abs()
        return out, size

    Y, V = forward(T, X, W, A, B, index, scale)
    ref, size = terms(s * ref_forward(X, W, A, B, index, scale)[1], B)
    assert bool(((Y.to(D) - ref).abs() <= 2.0 ** -8 * ref.abs() + 2.0 ** -14 * size).all())
    dX, _, _ = backward(T, dY, X, V, W, A, B, index, scale)
    u = torch.zeros(Tn, r, dtype=D, device=DEV)
    for k in range(n):
        own = (index == k).nonzero()[:, 0]
        u[own] = dY[own].to(D) @ B[k].to(D)
    # U is an fp32 sum of c terms: 2^-24 c^0.5 of their magnitudes goes into it, here below 2^-14 of size
    ref, size = terms(s * u, A.transpose(1, 2))
    assert bool(((dX.to(D) - ref).abs() <= 2.0 ** -8 * ref.abs() + 2.0 ** -14 * size).all())
