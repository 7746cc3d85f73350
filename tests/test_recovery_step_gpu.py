"""Accuracy of the orthogonalised update beyond what 16 bits show: steps on fp32 weights, and long
narrow matrices, against the float64 iteration."""

import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from tests.test_recovery_gpu import ref_ns, rel, spectrum  # noqa: E402

# Operands of 22 bits: a rounding is 2^-23 of the largest entries, directions without signal grow by
# 3.45^5 = 480 in five steps, so 6e-5 of the result; sums over up to 11008 / 16 accumulations that cut
# 2^-24 each add 4e-5.  Four times their sum:
TOL_FINE = 4e-4
# 16-bit operands on nearly orthogonal rows: bf16 rounding of the result 1.7e-3, and beside it 2^-12 of
# each entry of S and P once a step, halved by the fp32 diagonals
TOL_NARROW = 2.6e-3

SHAPES = [(1, 768, 768), (2, 40, 600), (1, 33, 1111), (3, 257, 130), (1, 500, 1301), (1, 513, 520),
          (1, 2100, 2050), (64, 48, 36)]


@pytest.fixture(scope="module")
def T():
    import paper_2504_05346_b200 as T

    return T


@pytest.mark.parametrize("kind", ["flat", "lead", "low rank"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_step_on_fp32_weights(T, shape, kind):
    k, m, n = shape
    G = spectrum(kind, k, m, n, seed=41).float()
    W, M = torch.zeros_like(G), torch.zeros_like(G)
    # from zero weights and momentum the step is the update itself, in fp32
    Wo, Mo = T.orthogonal_step(W, M, G, lr=1.0, momentum=0.0, check=True)
    ref = ref_ns(G)
    for i in range(k):
        assert rel(-Wo[i], ref[i]) <= TOL_FINE
    assert torch.equal(Mo, G)
    # bf16 weights take the shorter way: the same update to 16 bits
    Wh, _ = T.orthogonal_step(W.bfloat16(), M, G, lr=1.0, momentum=0.0)
    assert rel(Wh, Wo) <= 8e-3


@pytest.mark.parametrize("shape", [(3, 7697, 40), (1, 64, 4096), (1, 128, 8000), (2, 1500, 200)],
                         ids=lambda s: "x".join(map(str, s)))
def test_long_narrow_matrices(T, shape):
    gen = torch.Generator(device="cuda").manual_seed(43)
    G = torch.randn(shape, generator=gen, device="cuda")
    O, ref = T.orthogonalise(G), ref_ns(G)
    for i in range(shape[0]):
        assert rel(O[i], ref[i]) <= TOL_NARROW
    s = min(shape[1:])
    assert abs(O.float().norm().item() / math.sqrt(shape[0] * s) - 0.95) < 0.25


@pytest.mark.parametrize("side", [31, 32, 33, 36, 37, 63, 64, 65])
@pytest.mark.parametrize("tall", [False, True], ids=["wide", "tall"])
def test_sides_around_the_short_ones(T, side, tall):
    """Bounds of the layouts: sides of whole vectors and others, a few columns and many."""
    gen = torch.Generator(device="cuda").manual_seed(47)
    for k, l in ((1, side), (3, 100), (2, 1030)):
        l = max(l, side)
        G = torch.randn((k, l, side) if tall else (k, side, l), generator=gen, device="cuda")
        G[0, :, 0] = 0
        O, ref = T.orthogonalise(G), ref_ns(G)
        for i in range(k):
            assert rel(O[i], ref[i]) <= 4e-3   # as for every shape in 16 bits
        W = torch.zeros_like(G, dtype=torch.bfloat16)
        mask = torch.zeros(G.shape, dtype=torch.uint8, device="cuda")
        mask[:, 1:] = torch.randint(0, 2, mask[:, 1:].shape, generator=gen, device="cuda").to(torch.uint8)
        bad = torch.where(mask != 0, torch.full_like(G, float("nan")), G)
        Wo, Mo = T.orthogonal_step(W, torch.zeros_like(G), bad, mask=mask, lr=1.0, momentum=0.0,
                                   check=True)
        want = ref_ns(torch.where(mask != 0, 0.0, G))
        assert not Wo[mask != 0].any() and torch.isfinite(Wo.float()).all()
        want = torch.where(mask != 0, 0.0, want)
        for i in range(k):
            assert rel(-Wo[i], want[i]) <= 4e-3
