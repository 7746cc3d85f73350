"""Accuracy of what the recovery operators keep in fp32, tighter than the tests of their paths: it
would show the loss of an operand plane or of the drains of the tensor cores' accumulators.

A product is exact; the tensor cores cut up to 2^-23 of an accumulator each time they add to it, half of
that on average, and between two drains they add 32 times (512 terms; 64 times in fp32 products) to sums
that grow like the square root: 32 2^-24 2/3 = 1.3e-6 of the result, always towards zero, and the fp32
additions behind the drains add some 2^-24.  2e-6 in all.  (Sums over 8192 terms without drains cut 512
times; without the third plane of the fp32 factor each term is off by 2^-17.)"""

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from tests.test_recovery_gpu import make, ref_backward, ref_forward, rel  # noqa: E402

TOL = 2e-6


@pytest.fixture(scope="module")
def T():
    import paper_2504_05346_b200 as T_
    from paper_2504_05346_b200 import build as B_

    B_.build()
    T_.load_library()
    return T_


@pytest.mark.parametrize("shape", [(8192, 520, 8192, 1, 16, "one"), (8192, 4096, 1032, 2, 64, "blocks"),
                                   (4096, 2056, 4096, 3, 128, "mixed"), (60, 256, 8192, 4, 12, "mixed"),
                                   (1, 512, 4096, 2, 16, "one"), (300, 8200, 520, 5, 20, "blocks")],
                         ids=lambda s: "x".join(map(str, s)))
def test_bf16_factors_and_gradients(T, shape):
    Tn, c, b, n, r, order = shape
    X, W, A, B, index, scale, dY = make(Tn, c, b, n, r, torch.bfloat16, seed=51, order=order)
    _, V = T.adapter_forward(X, W, A, B, index, scale, check=True)
    assert rel(V, ref_forward(X, W, A, B, index, scale)[1]) <= TOL
    _, dA, dB = T.adapter_backward(dY, X, V, W, A, B, index, scale, need_dx=False, check=True)
    _, rA, rB = ref_backward(dY, X, V, W, A, B, index, scale)
    assert rel(dA, rA) <= TOL and rel(dB, rB) <= TOL


@pytest.mark.parametrize("shape", [(500, 768, 768, 3, 8, "blocks"), (2100, 768, 4096, 3, 8, "mixed"),
                                   (1024, 4096, 768, 1, 64, "one"), (2100, 1000, 2056, 2, 40, "mixed"),
                                   (33, 1024, 8192, 2, 16, "mixed"), (1, 4096, 1024, 2, 16, "one")],
                         ids=lambda s: "x".join(map(str, s)))
def test_f32(T, shape):
    Tn, c, b, n, r, order = shape
    X, W, A, B, index, scale, dY = make(Tn, c, b, n, r, torch.float32, seed=53, order=order)
    Y, V = T.adapter_forward(X, W, A, B, index, scale, check=True)
    Yr, Vr = ref_forward(X, W, A, B, index, scale)
    assert rel(Y, Yr) <= TOL and rel(V, Vr) <= TOL
    got = T.adapter_backward(dY, X, V, W, A, B, index, scale, check=True)
    for x, ref in zip(got, ref_backward(dY, X, V, W, A, B, index, scale)):
        assert rel(x, ref) <= TOL


@pytest.mark.parametrize("shape", [(100, 256, 16384), (33, 200, 65536), (700, 300, 24584), (5, 129, 8200)],
                         ids=lambda s: "x".join(map(str, s)))
def test_f32_long_sums(T, shape):
    """As many inputs as the projection takes, and as many outputs for the backward sums; on positive
    numbers, where every cut goes the same way, 64 additions of full size cut 64 2^-24 = 3.9e-6."""
    Tn, c, b = shape
    X, W, A, B, index, scale, dY = make(Tn, c, b, 2, 12, torch.float32, seed=57)
    Y, V = T.adapter_forward(X, W, A, B, index, scale, check=True)
    Yr, Vr = ref_forward(X, W, A, B, index, scale)
    assert rel(Y, Yr) <= TOL and rel(V, Vr) <= TOL
    P, Q = X.abs(), W.abs()
    assert rel(T.adapter_forward(P, Q, check=True)[0], P.double() @ Q.double().T) <= 2 * TOL
    # the same matrices the other way round: c is the long side
    Wt, dY2 = W.t().contiguous(), X
    At = torch.randn(2, 12, Wt.shape[1] // 8 * 8, device="cuda") / 16
    Wt = Wt[:, :At.shape[2]].contiguous()
    Bt = 0.1 * torch.randn(2, Wt.shape[0], 12, device="cuda")
    dX, _, _ = T.adapter_backward(dY2, None, None, Wt, At, Bt, index, scale, need_grads=False, check=True)
    zero = torch.zeros(Tn, At.shape[2], device="cuda")
    assert rel(dX, ref_backward(dY2, zero, torch.zeros(Tn, 12, device="cuda"), Wt, At, Bt, index, scale)[0]) <= TOL


def test_f32_longest_backward_sum(T):
    gen = torch.Generator(device="cuda").manual_seed(59)
    dY = torch.randn(40, 1 << 20, generator=gen, device="cuda")
    W = torch.randn(1 << 20, 72, generator=gen, device="cuda")
    dX, _, _ = T.adapter_backward(dY, None, None, W, need_grads=False, check=True)
    assert rel(dX, dY.double() @ W.double()) <= TOL


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("positive", [False, True], ids=["signs", "positive"])
def test_gradients_over_many_tokens(T, dtype, positive):
    """2^22 tokens of one adapter: chains of at most 64 and then 2^22 / 512 additions, which round 2^-24
    each, in random directions: 2^-24 (64^0.5 + 8192^0.5) = 5.9e-6 (in one chain of positive terms
    roundings of one direction add up: 8e-5)."""
    Tn, c, b, r = 1 << 22, 24, 16, 9
    gen = torch.Generator(device="cuda").manual_seed(61)
    rn = lambda *s: torch.randn(s, generator=gen, device="cuda")  # noqa: E731
    data = [rn(Tn, b).to(dtype), rn(Tn, c).to(dtype), rn(Tn, r), rn(1, r, b).to(dtype), rn(1, c, r).to(dtype)]
    X, dY, V, A, B = (d.abs() for d in data) if positive else data
    W = torch.zeros(c, b, dtype=dtype, device="cuda")
    index, scale = torch.zeros(Tn, dtype=torch.int32, device="cuda"), torch.ones(1, device="cuda")
    _, dA, dB = T.adapter_backward(dY, X, V, W, A, B, index, scale, need_dx=False, check=True)
    D = torch.float64
    assert rel(dB[0], dY.to(D).T @ V.to(D)) <= 5.9e-6
    assert rel(dA[0], (dY.to(D) @ B[0].to(D)).T @ X.to(D)) <= 5.9e-6


def spectrum(kind, k, m, n, gen):
    rn = lambda *s: torch.randn(s, generator=gen, device="cuda")  # noqa: E731
    q = max(1, min(m, n) // 16)
    if kind == "flat":
        return rn(k, m, n)
    lead = rn(k, m, q) @ rn(k, q, n)
    return lead if kind == "low rank" else lead + 0.05 * rn(k, m, n)


@pytest.mark.parametrize("kind", ["flat", "lead", "low rank"])
@pytest.mark.parametrize("shape", [(1, 16, 65536), (1, 32, 65536), (32, 16, 4096), (3, 11008, 24), (5, 7, 100),
                                   (1, 17, 4099), (2, 1000, 31), (1, 1, 9)],
                         ids=lambda s: "x".join(map(str, s)))
def test_fp32_step_on_short_sides(T, shape, kind):
    """Where the iteration runs on the Gram matrix and the weights are fp32, that matrix and its powers
    are fp64; what is left is the rounding of X and of the factor that is applied to it, 2^-24 of terms
    up to 3.4445^5 = 485 times the result, 2.9e-5, and as much again for their fp32 sums."""
    gen = torch.Generator(device="cuda").manual_seed(67)
    G = spectrum(kind, *shape, gen)
    Z = torch.zeros_like(G)
    W, _ = T.orthogonal_step(Z, Z, G, lr=1.0, momentum=0.0, check=True)
    X = G.double()
    tall = shape[1] > shape[2]
    X = X.mT if tall else X
    X = X / (torch.linalg.matrix_norm(X, keepdim=True) + 1e-7)
    a, b, c = T.NEWTON_SCHULZ
    for _ in range(5):
        S = X @ X.mT
        X = a * X + (b * S + c * (S @ S)) @ X
    X = X.mT if tall else X
    for i in range(shape[0]):
        assert rel(-W[i], X[i]) <= 5.8e-5


@pytest.mark.parametrize("kind", ["flat", "lead"])
@pytest.mark.parametrize("shape", [(2048, 65536), (65536, 2100), (1300, 32776), (200, 65536)],
                         ids=lambda s: "x".join(map(str, s)))
def test_fp32_step_on_long_sides(T, shape, kind):
    """The diagonal of S is a sum of squares of which an accumulator cuts 2^-24 on average each of its
    three products per 16 terms, 3 16384 / 16 times at most, and half of them, on average, at full size:
    9e-5 of the diagonal; the polynomial's slope makes up to four times that of the last step's factor
    and less of the others', on the strong half of the directions: 2e-4."""
    gen = torch.Generator(device="cuda").manual_seed(71)
    G = spectrum(kind, 1, *shape, gen)[0]
    Z = torch.zeros_like(G)
    W, _ = T.orthogonal_step(Z, Z, G, lr=1.0, momentum=0.0, check=True)
    X = G.double()
    tall = shape[0] > shape[1]
    X = X.mT if tall else X
    X = X / (X.norm() + 1e-7)
    a, b, c = T.NEWTON_SCHULZ
    for _ in range(5):
        S = X @ X.mT
        X = a * X + (b * S + c * (S @ S)) @ X
    assert rel(-(W.mT if tall else W), X) <= 2e-4
