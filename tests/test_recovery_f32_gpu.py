"""The adapted projection in fp32 where there are many tokens or ranks, and rows that are no whole
number of 128-byte lines, against the float64 formulas."""

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from tests.test_recovery_gpu import make, ref_backward, ref_forward, rel  # noqa: E402

# Sums of products that are exact to 2^-24 of their size, over at most 2000 terms whose signs vary,
# drained into fp32 every 512 of them: a few 2^-24 of the result's norm, ten times over.
TOL = 1e-5

# tokens, outputs, inputs, adapters, rank, order: tokens times rank around 2^14 and 2^16, adapters times
# rank above and below twice the tokens, rows of whole lines and others
SHAPES = [
    (1024, 200, 264, 5, 16, "mixed"), (1023, 200, 264, 5, 16, "mixed"), (700, 136, 1000, 3, 32, "mixed"),
    (2000, 1000, 72, 7, 9, "mixed"), (2000, 72, 200, 11, 33, "mixed"), (300, 520, 392, 2, 64, "mixed"), (150, 264, 328, 4, 128, "mixed"),
    (129, 100, 136, 3, 127, "mixed"), (512, 96, 64, 64, 32, "mixed"), (2000, 1000, 1000, 1, 20, "mixed"),
]


@pytest.fixture(scope="module")
def T():
    import paper_2504_05346_b200 as T

    return T


@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_f32_forward_and_backward(T, shape):
    Tn, c, b, n, r, order = shape
    X, W, A, B, index, scale, dY = make(Tn, c, b, n, r, torch.float32, seed=29, order=order)
    Y, V = T.adapter_forward(X, W, A, B, index, scale, check=True)
    Yr, Vr = ref_forward(X, W, A, B, index, scale)
    assert rel(Y, Yr) <= TOL and rel(V, Vr) <= TOL
    got = T.adapter_backward(dY, X, V, W, A, B, index, scale, check=True)
    want = ref_backward(dY, X, V, W, A, B, index, scale)
    for x, ref in zip(got, want):
        assert rel(x, ref) <= TOL
    # the gradients alone, and added to what is there
    dA, dB = got[1].clone(), got[2].clone()
    T.adapter_backward(dY, X, V, W, A, B, index, scale, need_dx=False, dA=dA, dB=dB, accumulate=True)
    assert rel(dA, 2 * want[1]) <= TOL and rel(dB, 2 * want[2]) <= TOL


def test_f32_non_finite_values_stay_with_their_tokens(T):
    X, W, A, B, index, scale, dY = make(2800, 136, 200, 4, 24, torch.float32, seed=31)
    index[7], index[8] = 1, 2
    A[1, 3, 5] = float("inf")
    X[9] = float("nan")
    clean = (index != 1) & (torch.arange(2800, device=index.device) != 9)
    Y, V = T.adapter_forward(X, W, A, B, index, scale)
    assert torch.isfinite(Y[clean]).all() and torch.isfinite(V[clean]).all()
    assert not torch.isfinite(Y[7]).any() and torch.isnan(Y[9]).all()
    A2 = A.clone()
    A2[1] = 0
    keep = clean.nonzero().squeeze(1)
    Yr, Vr = ref_forward(X[keep], W, A2, B, index[keep], scale)
    assert rel(Y[keep], Yr) <= TOL and rel(V[keep], Vr) <= TOL
