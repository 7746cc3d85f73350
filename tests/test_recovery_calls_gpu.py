"""How the recovery operators are called: on another stream than the current one, with nothing to do,
with buffers that are not needed."""

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from tests.test_recovery_gpu import make  # noqa: E402

DEV = "cuda"
BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def T():
    import paper_2504_05346_b200 as T_
    from paper_2504_05346_b200 import build as B_

    B_.build()
    T_.load_library()
    return T_


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("Tn", [3, 40, 200])
def test_check_reads_the_status_behind_a_call_on_another_stream(T, Tn, dtype):
    """The other stream is busy for a while, so the status word is still the last call's when the
    current stream looks."""
    X, W, A, B, index, scale, dY = make(Tn, 96, 128, 3, 8, dtype, seed=10)
    Y, V = T.adapter_forward(X, W, A, B, index, scale)
    ws = torch.zeros(1 << 22, dtype=torch.uint8, device=DEV)
    good, bad = index.clone(), index.clone()
    bad[1] = 3
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    for call in (lambda i: T.adapter_forward(X, W, A, B, i, scale, stream=stream, workspace=ws,
                                             check=True),
                 lambda i: T.adapter_backward(dY, X, V, W, A, B, i, scale, stream=stream, workspace=ws,
                                              check=True)):
        for k in range(2):
            with torch.cuda.stream(stream):
                torch.cuda._sleep(20_000_000)
            with pytest.raises(T.ThanosError) as e:
                call(bad)
            assert e.value.code == 1
            with torch.cuda.stream(stream):
                torch.cuda._sleep(20_000_000)
            call(good)       # and not the status of the call before


def test_empty_batches(T):
    """No matrices: nothing runs, nothing is refused, and a workspace's old status word is not read."""
    ws = torch.full((4096,), 255, dtype=torch.uint8, device=DEV)
    before = T.launch_count()
    for shape in ((0, 16, 300), (0, 200, 130)):
        G = torch.empty(shape, device=DEV)
        O = T.orthogonalise(G, workspace=ws, check=True)
        assert O.shape == shape and O.dtype == BF16
        for dtype in (BF16, F32):
            mask = torch.empty(shape, dtype=torch.uint8, device=DEV)
            W, M = T.orthogonal_step(G.to(dtype), G, G, mask, workspace=ws, check=True)
            assert W.shape == shape and W.dtype == dtype and M.shape == shape
        assert T.orthogonalise(G).shape == shape
    assert T.launch_count() == before
    with pytest.raises(T.ThanosError):
        T.orthogonalise(torch.empty((3, 0, 8), device=DEV))


def test_no_adapters_no_v(T):
    """Without adapters there is no V, also where a buffer for one or an empty set of adapters is given."""
    X, W, A, B, index, scale, _ = make(40, 96, 128, 3, 8, BF16, seed=9)
    buf = torch.full((40, 8), 7.0, device=DEV)
    Y, V = T.adapter_forward(X, W, V=buf, check=True)
    Y2, V2 = T.adapter_forward(X, W, A[:0], B[:0], torch.full_like(index, -1), scale[:0], V=buf,
                               check=True)
    assert V is None and V2 is None and torch.equal(Y, Y2) and bool((buf == 7.0).all())
