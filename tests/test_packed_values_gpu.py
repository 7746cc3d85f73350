"""The adapted projection on 4-bit weights at the ends of the types, against float64: infinite and NaN
adapters, tokens that are not finite beside others of the same adapter, the largest activations and small
ones.

Tolerances as in test_packed_gpu.py (a rounding to bf16 3e-3 in the norm, sums in fp32 1e-5); what is not
finite stands where the definition has it, with its sign.
"""

import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from tests.test_recovery_gpu import make, ref_forward, rel  # noqa: E402

DEV = "cuda"
BF16, F32 = torch.bfloat16, torch.float32
INF, NAN = math.inf, math.nan
TOL = {BF16: 3e-3, F32: 1e-5}
BOTH = pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])


@pytest.fixture(scope="module")
def T():
    import paper_2504_05346_b200 as T_
    from paper_2504_05346_b200 import build as B_

    B_.build()
    T_.load_library()
    return T_


def same_values(x, ref, tol):
    for kind in (torch.isnan, torch.isposinf, torch.isneginf):
        assert torch.equal(kind(x.double()), kind(ref))
    fin = torch.isfinite(ref)
    assert rel(torch.where(fin, x.double(), 0.0), torch.where(fin, ref, 0.0)) <= tol


# One token to a lane's row of B and several on the tensor cores; one slice of k and several; weights
# unpacked first.
SHARED = [(3, 300, 264, 2, 24), (16, 300, 264, 2, 64), (20, 300, 264, 2, 24), (60, 300, 264, 3, 64),
          (64, 300, 264, 2, 16), (128, 12000, 72, 2, 64), (128, 300, 4104, 2, 24), (250, 520, 264, 2, 128),
          (300, 300, 264, 2, 24)]


@BOTH
@pytest.mark.parametrize("shape", SHARED, ids=lambda s: "x".join(map(str, s)))
def test_adapters_that_are_not_finite(T, shape, dtype):
    """V are whole numbers of a few bits here: where a factor is split into parts, some of them are
    zeros, which must not meet an infinity."""
    Tn, c, b, n, r = shape
    X, W, A, B, index, scale, _ = make(Tn, c, b, n, r, dtype, seed=Tn + r, order="blocks")
    g = torch.Generator(device=DEV).manual_seed(Tn)
    X = torch.randint(-3, 4, (Tn, b), generator=g, device=DEV).to(dtype)
    A = (2.0 * torch.randint(0, 2, (n, r, b), generator=g, device=DEV) - 1.0).to(dtype)
    B = B.clone()
    B[0, ::7, 4], B[0, 3::7, 9], B[1, 5::7, 2] = INF, -INF, NAN
    B[1, 1::9, 3], B[1, 1::9, r - 1] = INF, INF
    P = T.pack_weights(W, 64)
    Y, V = T.adapter_forward(X, P, A, B, index, scale, check=True)
    Yr, Vr = ref_forward(X, T.unpack_weights(P, F32), A, B, index, scale)
    same_values(V, Vr, TOL[F32])
    same_values(Y, Yr, TOL[dtype])
    assert bool(Yr.isposinf().any()) and bool(Yr.isneginf().any()) and bool(Yr.isnan().any())


@BOTH
@pytest.mark.parametrize("shape", SHARED, ids=lambda s: "x".join(map(str, s)))
def test_tokens_of_one_adapter_that_are_not_finite(T, shape, dtype):
    Tn, c, b, n, r = shape
    X, W, A, B, index, scale, _ = make(Tn, c, b, n, r, dtype, seed=Tn + r, order="blocks")
    W = torch.where(W == 0, 0.01, W.float()).to(dtype)
    P = T.pack_weights(W, 64)
    Wd = T.unpack_weights(P, F32)
    clean, _ = T.adapter_forward(X, P, A, B, index, scale)
    X = X.clone()
    X[0, 5], X[1, 9] = INF, -INF
    X[2, b - 1] = NAN
    Y, V = T.adapter_forward(X, P, A, B, index, scale, check=True)
    Yr, Vr = ref_forward(X, Wd, A, B, index, scale)
    same_values(V, Vr, TOL[F32])
    for kind in (torch.isnan, torch.isposinf, torch.isneginf):
        assert torch.equal(kind(Y.double()), kind(Yr))
    assert torch.equal(Y[3:], clean[3:])


EVERY = pytest.mark.parametrize("Tn", [1, 3, 9, 16, 20, 50, 64, 200, 300])


@BOTH
@EVERY
def test_the_largest_activations(T, Tn, dtype):
    """Codes of -8 (and of 7 in every other row) with scales of 2^-14: 64 products of a code and an
    activation are 2^9 times the activation, beyond the type's largest number, the result is not."""
    c, b = 96, 328
    codes = torch.zeros((c, 192), dtype=torch.uint8, device=DEV)
    codes[1::2] = 0xFF
    P = T.PackedWeights(codes, torch.full((6, c), 2.0 ** -14, dtype=BF16, device=DEV), 64, b)
    W = T.unpack_weights(P, F32).double()
    X = torch.full((Tn, b), torch.finfo(dtype).max, device=DEV).to(dtype)
    X[1::2] = -X[1::2]
    X[2::3, 1::2] *= 0.5
    want = X.double() @ W.t()
    assert float(want.abs().max()) < 0.2 * torch.finfo(dtype).max
    Y, _ = T.adapter_forward(X, P)
    assert bool(Y.isfinite().all())
    assert rel(Y.double() * 2.0 ** -100, want * 2.0 ** -100) <= TOL[dtype]


@BOTH
@EVERY
def test_small_activations(T, Tn, dtype):
    """bf16 some 2^8 above its smallest normal number, fp32 as far down as three parts of eight bits are
    bf16 numbers: products with codes are exact, and their sums keep more than the tolerances ask for."""
    X, W, *_ = make(Tn, 96, 328, 1, 1, dtype, seed=Tn)
    X = (X.float() * 2.0 ** (-118 if dtype == BF16 else -100)).to(dtype)
    P = T.pack_weights(4 * W, 64)
    want = X.double() @ T.unpack_weights(P, F32).double().t()
    Y, _ = T.adapter_forward(X, P)
    assert rel(Y.double() * 2.0 ** 100, want * 2.0 ** 100) <= TOL[dtype]
