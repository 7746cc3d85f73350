"""The operators together, as examples/recover_layer.py uses them: a small layer is pruned, its
remaining weights are tuned, adapters are trained and served."""

import os
import sys

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.parametrize("shape", [(320, 256, 3, 8), (136, 520, 1, 5)], ids=["320x256", "136x520"])
def test_recover_layer_example(shape):
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    try:
        import recover_layer
    finally:
        sys.path.pop(0)
    rows, cols, tasks, rank = (str(v) for v in shape)
    out = recover_layer.main(["--rows", rows, "--cols", cols, "--tasks", tasks, "--rank", rank,
                              "--tokens", "1024"])
    assert out["tuned"] < out["pruned"] < 1.0
    assert out["tasks after"] < 0.7 * out["tasks before"]
    # one token alone and the same token in a batch differ by their sums' order: a rounding of bf16
    assert out["served together against alone"] < 2.0 ** -8


def test_slices_of_a_batch_are_taken_as_they_are():
    """index[t:] and scale[i:] start between 16-byte lines; every token gets what it gets in the
    whole batch, to a rounding of bf16."""
    import paper_2504_05346_b200 as T

    gen = torch.Generator(device="cuda").manual_seed(3)
    rn = lambda *s: torch.randn(s, generator=gen, device="cuda")  # noqa: E731
    X, W = rn(12, 64).bfloat16(), (rn(64, 64) / 8).bfloat16()
    A, B = (rn(5, 4, 64) / 8).bfloat16(), (rn(5, 64, 4) / 2).bfloat16()
    index = torch.randint(-1, 4, (12,), generator=gen, device="cuda", dtype=torch.int32)
    scale = torch.rand(5, generator=gen, device="cuda") + 0.5
    A, B, scale = A[1:].clone(), B[1:].clone(), scale[1:]
    assert scale.data_ptr() % 16
    Y, V = T.adapter_forward(X, W, A, B, index, scale)
    dX, dA, dB = T.adapter_backward(Y, X, V, W, A, B, index, scale)
    whole = torch.zeros_like(dA)
    for t in range(1, 12):
        assert index[t:].data_ptr() % 16 or t % 4 == 0
        Yt, Vt = T.adapter_forward(X[t:], W, A, B, index[t:], scale)
        assert (Yt.float() - Y[t:].float()).norm() <= 2.0 ** -8 * Y[t:].float().norm()
        torch.testing.assert_close(Vt, V[t:], rtol=1e-5, atol=1e-5)
    for t in range(12):
        part = T.adapter_backward(Y[t:t + 1], X[t:t + 1], V[t:t + 1].clone(), W, A, B,
                                  index[t:t + 1], scale)
        whole += part[1]
    # sums of 12 terms in another order, of products that are exact to 2^-16 or better
    assert (whole - dA).norm() <= 1e-4 * dA.norm()
