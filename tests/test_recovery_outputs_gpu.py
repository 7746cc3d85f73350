"""Every output of the recovery operators is written by the call: outputs are passed in full of NaN,
and the values that stand for "nothing to compute" (tokens without adapter, adapters without tokens)
are exact zeros, at every size where another kernel is in charge of them.

Tolerances as in test_recovery_gpu.py: one rounding to bf16 and the same again for the adapter part
(3e-3), sums in fp32 (1e-5)."""

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from tests.test_recovery_gpu import TOL_BF16, TOL_F32, make, ref_backward, ref_forward, rel  # noqa: E402

DEV = "cuda"
BF16, F32 = torch.bfloat16, torch.float32
TYPES = pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])


@pytest.fixture(scope="module")
def T():
    import paper_2504_05346_b200 as T_
    from paper_2504_05346_b200 import build as B_

    B_.build()
    T_.load_library()
    return T_


def nan(*shape, dtype=F32):
    return torch.full(shape, float("nan"), dtype=dtype, device=DEV)


# one to eight tokens of few products (V on the way), of more products (a launch for V), up to 64
# tokens, and more (V on the tensor cores; fp32: 8192 tokens of rank 8 and more)
BARE = [(1, 4096, 4096, 16), (1, 64, 64, 4), (2, 130, 72, 1), (3, 1001, 520, 12), (8, 512, 1024, 16),
        (8, 64, 64, 128), (9, 200, 264, 5), (64, 256, 512, 16), (65, 256, 512, 16), (300, 136, 72, 7),
        (8200, 72, 64, 8)]


@TYPES
@pytest.mark.parametrize("bad", [None, 5, -2], ids=["none", "beyond", "below"])
@pytest.mark.parametrize("shape", BARE, ids=lambda s: "x".join(map(str, s)))
def test_no_token_has_an_adapter(T, shape, bad, dtype):
    """All indices -1, and all out of range (which count as -1): Y = X W^T and V = 0."""
    Tn, c, b, r = shape
    X, W, A, B, index, scale, dY = make(Tn, c, b, 5, r, dtype, seed=Tn + r, order="none")
    if bad is not None:
        index.fill_(bad)
    Y, V = T.adapter_forward(X, W, A, B, index, scale, out=nan(Tn, c, dtype=dtype), V=nan(Tn, r),
                             check=bad is None)
    assert bool((V == 0).all())
    assert rel(Y, X.double() @ W.double().T) <= (TOL_BF16 if dtype == BF16 else TOL_F32)
    dX, dA, dB = T.adapter_backward(dY, X, V, W, A, B, index, scale, dX=nan(Tn, b, dtype=dtype),
                                    dA=nan(5, r, b), dB=nan(5, c, r), check=bad is None)
    assert bool((dA == 0).all()) and bool((dB == 0).all())
    assert rel(dX, dY.double() @ W.double()) <= (TOL_BF16 if dtype == BF16 else TOL_F32)


WRITTEN = [(1, 4096, 1024, 8, 16, "one"), (7, 1001, 520, 5, 12, "mixed"), (33, 1, 8, 2, 8, "mixed"),
           (64, 777, 1032, 64, 16, "blocks"), (129, 384, 1096, 2, 128, "mixed"),
           (700, 1536, 1000, 150, 7, "mixed"), (2048, 2048, 1024, 1, 16, "one"),
           (2048, 2048, 1024, 6, 20, "mixed"), (3000, 640, 1280, 5, 24, "blocks")]


@TYPES
@pytest.mark.parametrize("shape", WRITTEN, ids=lambda s: "x".join(map(str, s)))
def test_every_output_is_written(T, shape, dtype):
    Tn, c, b, n, r, order = shape
    X, W, A, B, index, scale, dY = make(Tn, c, b, n, r, dtype, seed=Tn + c + 2, order=order)
    tol = TOL_BF16 if dtype == BF16 else TOL_F32
    Y, V = T.adapter_forward(X, W, A, B, index, scale, out=nan(Tn, c, dtype=dtype), V=nan(Tn, r),
                             check=True)
    Yr, Vr = ref_forward(X, W, A, B, index, scale)
    assert rel(Y, Yr) <= tol and rel(V, Vr) <= TOL_F32
    assert bool((V[index < 0] == 0).all())
    got = T.adapter_backward(dY, X, V, W, A, B, index, scale, dX=nan(Tn, b, dtype=dtype),
                             dA=nan(n, r, b), dB=nan(n, c, r), check=True)
    for x, ref, t in zip(got, ref_backward(dY, X, V, W, A, B, index, scale), (tol, TOL_F32, TOL_F32)):
        assert rel(x, ref) <= t


@pytest.mark.parametrize("shape", [(1, 1, 1), (5, 16, 100), (2, 300, 33), (1, 65, 130), (2, 129, 260),
                                   (1, 640, 2600)], ids=lambda s: "x".join(map(str, s)))
def test_every_output_of_the_update_is_written(T, shape):
    gen = torch.Generator(device=DEV).manual_seed(5)
    G = torch.randn(shape, generator=gen, device=DEV)
    O = T.orthogonalise(G, out=nan(*shape, dtype=BF16), check=True)
    assert torch.equal(O, T.orthogonalise(G)) and bool(torch.isfinite(O.float()).all())
    mask = (torch.rand(shape, generator=gen, device=DEV) < 0.5).to(torch.uint8)
    for dtype in (BF16, F32):
        W = torch.where(mask != 0, 0.0, torch.randn(shape, generator=gen, device=DEV)).to(dtype)
        Wo, Mo = T.orthogonal_step(W, torch.zeros(shape, device=DEV), G, mask,
                                   W_out=nan(*shape, dtype=dtype), M_out=nan(*shape), check=True)
        assert torch.equal(Mo, torch.where(mask != 0, 0.0, G))
        assert bool(torch.isfinite(Wo.float()).all()) and bool((Wo[mask != 0] == 0).all())


@TYPES
@pytest.mark.parametrize("bad", [float("inf"), float("nan")])
def test_scale_of_an_adapter_without_tokens_does_not_matter(T, bad, dtype):
    X, W, A, B, index, scale, dY = make(90, 136, 72, 4, 12, dtype, seed=3)
    index[index == 1] = 2
    odd = scale.clone()
    odd[1] = bad
    for u, v in zip(T.adapter_forward(X, W, A, B, index, odd), T.adapter_forward(X, W, A, B, index, scale)):
        assert torch.equal(u, v)
    V = T.adapter_forward(X, W, A, B, index, scale)[1]
    for accumulate in (False, True):
        out = []
        for s in (odd, scale):
            dA, dB = torch.ones(4, 12, 72, device=DEV), torch.ones(4, 136, 12, device=DEV)
            out.append(T.adapter_backward(dY, X, V, W, A, B, index, s, dA=dA, dB=dB,
                                          accumulate=accumulate))
        for u, v in zip(*out):
            assert torch.equal(u, v)
        assert bool((out[0][1][1] == accumulate).all()) and bool((out[0][2][1] == accumulate).all())
