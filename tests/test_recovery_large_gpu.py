"""The adapted projection at the largest number of tokens that it takes (2^24), where the work in
front of a product, the sort of all tokens among it, takes tens of milliseconds: no bounded wait of the
products runs out meanwhile, and no offset wraps.

Tolerances: rows of Y and dX as in test_recovery_gpu.py.  Gradients are sums of 2^22 terms a lane and
adapter: the bf16 kernel adds 512 of them at a time (2^-23 of the sum is cut up to 32 times) and then some
10^3 to 10^4 such sums, each rounding 2^-24, in random directions: 1e-5, four times over; the fp32 kernel
adds 2^19 and more one after another, 2^-24 sqrt(2^21) = 9e-5, four times over."""

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from tests.test_recovery_gpu import TOL_BF16, TOL_F32, rel  # noqa: E402

DEV = "cuda"


@pytest.mark.parametrize("dtype,c,b,tol", [(torch.bfloat16, 136, 136, 4e-5), (torch.float32, 9, 8, 4e-4),
                                           (torch.bfloat16, 9, 8, 4e-5)],
                         ids=["bf16-pairs", "f32", "bf16-tiles"])
def test_largest_number_of_tokens(dtype, c, b, tol):
    import paper_2504_05346_b200 as T

    Tn, n, r = 1 << 24, 3, 4
    gen = torch.Generator(device=DEV).manual_seed(17)
    rn = lambda *s: torch.randn(s, generator=gen, device=DEV, dtype=dtype)  # noqa: E731
    X, dY, W = rn(Tn, b), rn(Tn, c), rn(c, b) / 8
    A, B = rn(n, r, b) / 8, rn(n, c, r) / 2
    index = (torch.arange(Tn, device=DEV) * 7919 % (n + 1) - 1).to(torch.int32)
    scale = torch.tensor([0.5, 1.0, 2.0], device=DEV)
    Y, V = T.adapter_forward(X, W, A, B, index, scale, check=True)
    dX, dA, dB = T.adapter_backward(dY, X, V, W, A, B, index, scale, check=True)
    at = torch.cat([torch.arange(0, Tn, 65521, device=DEV), torch.arange(Tn - 600, Tn, device=DEV)])
    D = torch.float64
    i = index[at].long().clamp(min=0)
    s = torch.where(index[at] >= 0, scale[i], 0.0).to(D)
    x, dy = X[at].to(D), dY[at].to(D)
    own = (index[at] >= 0).to(D)[:, None]
    v = own * torch.einsum("tk,trk->tr", x, A.to(D)[i])
    lim = TOL_BF16 if dtype == torch.bfloat16 else TOL_F32
    assert rel(V[at], v) <= TOL_F32
    assert rel(Y[at], x @ W.to(D).T + s[:, None] * torch.einsum("tr,tcr->tc", v, B.to(D)[i])) <= lim
    u = s[:, None] * torch.einsum("tc,tcr->tr", dy, B.to(D)[i])
    assert rel(dX[at], dy @ W.to(D) + torch.einsum("tr,trk->tk", u, A.to(D)[i])) <= lim
    rA, rB = torch.zeros((n, r, b), dtype=D, device=DEV), torch.zeros((n, c, r), dtype=D, device=DEV)
    for t0 in range(0, Tn, 1 << 21):
        part = slice(t0, t0 + (1 << 21))
        xs, ys, vs, ix = X[part].to(D), dY[part].to(D), V[part].to(D), index[part]
        for k in range(n):
            own = (ix == k).to(D)[:, None] * scale[k].item()
            rA[k] += (own * (ys @ B[k].to(D))).T @ xs
            rB[k] += (own * ys).T @ vs
    assert rel(dA, rA) <= tol and rel(dB, rB) <= tol
