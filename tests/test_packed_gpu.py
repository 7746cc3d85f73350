"""Weights in 4 bits and activations in 8, and the adapted projection on them, against float64.

Packing is exact arithmetic: codes, scales and what they stand for are compared for equality.  The
projection's tolerances are those of the projection on plain operands, because a packed weight is a bf16
number: a bf16 result is one rounding of an fp32 sum (2^-9 elementwise, 1.7e-3 in the norm; 3e-3 with the
adapter's part), fp32 results are fp32 sums (1e-5 for the lengths here).
"""

import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from tests.test_recovery_gpu import make, ref_backward, ref_forward, rel  # noqa: E402

DEV = "cuda"
BF16, F32, F64 = torch.bfloat16, torch.float32, torch.float64
TOL = {BF16: 3e-3, F32: 1e-5}
BOTH = pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])


@pytest.fixture(scope="module")
def T():
    import paper_2504_05346_b200 as T_
    from paper_2504_05346_b200 import build as B_

    B_.build()
    T_.load_library()
    return T_


def ref_weights(W, group):
    """Codes, scales [groups, c] and values in float64."""
    c, b = W.shape
    out = torch.zeros((c, b), dtype=F64, device=DEV)
    codes = torch.zeros_like(out)
    scales = []
    for j in range(0, b, group):
        w = W[:, j:j + group].double()
        top = w.abs().amax(1) / 7
        frac, exp = torch.frexp(top)
        s = torch.ldexp(torch.round(frac * 32) / 32, exp)
        s = torch.where(s < 2.0 ** -126, 0.0, s)
        q = torch.where(s[:, None] > 0, torch.round(w / s.clamp(min=1e-300)[:, None]), 0.0)
        q = q.clamp(-7, 7)
        codes[:, j:j + group] = q
        out[:, j:j + group] = q * s[:, None]
        scales.append(s)
    return codes, torch.stack(scales), out


def nibbles(P):
    n = torch.stack([P.codes & 15, P.codes >> 4], 2).flatten(1)
    return n.to(F64) - 8


@BOTH
@pytest.mark.parametrize("group", [64, 128])
@pytest.mark.parametrize("c, b, pad", [(1, 8, 0), (3, 64, 0), (17, 72, 8), (64, 128, 0), (5, 1000, 24),
                                       (300, 520, 0), (1001, 1752, 0), (33, 4096, 8), (2, 65536, 0)])
def test_pack_weights(T, c, b, pad, group, dtype):
    g = torch.Generator(device=DEV).manual_seed(c * b)
    W = (0.02 * torch.randn((c, b + pad), generator=g, device=DEV)).to(dtype)[:, :b]
    W[torch.rand((c, b), generator=g, device=DEV) < 0.5] = 0
    P = T.pack_weights(W, group)
    codes, scales, values = ref_weights(W, group)
    n = nibbles(P)
    assert torch.equal(n[:, :b], codes) and not bool(n[:, b:].any())
    assert torch.equal(P.scales.double(), scales)
    for out in (BF16, F32):
        U = T.unpack_weights(P, out)
        assert U.dtype == out and torch.equal(U.double(), values)
    assert bool((values[W == 0] == 0).all())
    step = scales.t().repeat_interleave(group, 1)[:, :b]
    assert bool(((values - W.double()).abs() <= 0.5 * step).all())


@BOTH
def test_pack_weights_at_the_ends_of_the_type(T, dtype):
    W = torch.zeros((10, 128), device=DEV)
    W[1] = torch.finfo(dtype).max
    W[2] = 2.0 ** -126
    W[3, 5] = 2.0 ** -120
    W[4, 3], W[4, 70] = math.inf, 1.0
    W[5, 3], W[5, 70] = math.nan, 1.0
    W[6] = torch.arange(128, device=DEV) - 64.0
    W[7] = -7.0
    W[8, ::2] = 7 * 17 / 16
    W[9] = 2.0 ** -130
    W = W.to(dtype)
    P = T.pack_weights(W, 64)
    U = T.unpack_weights(P, F32)
    _, _, values = ref_weights(W, 64)
    fine = [0, 1, 2, 3, 6, 7, 8, 9]
    assert torch.equal(U[fine].double(), values[fine])
    for row in (4, 5):       # the group that holds it, and no other
        assert bool(U[row, :64].isnan().all())
        assert bool(U[row, 64:].isfinite().all())


@BOTH
def test_codes_and_scales_of_ones_own(T, dtype):
    """Code -8, scales whose low bits are set (they take no part), padding that holds anything."""
    g = torch.Generator(device=DEV).manual_seed(2)
    codes = torch.randint(0, 256, (70, 96), generator=g, device=DEV, dtype=torch.uint8)
    bits = torch.randint(0x3C00, 0x3D00, (3, 70), generator=g, device=DEV)
    scales = bits.to(torch.int16).view(BF16)
    kept = (bits & 0xFFF8).to(torch.int16).view(BF16).double()
    P = T.PackedWeights(codes, scales, 64, 136)
    W = nibbles(P)[:, :136] * kept.t().repeat_interleave(64, 1)[:, :136]
    assert torch.equal(T.unpack_weights(P, dtype).double(), W)
    for Tn in (1, 9, 40, 130):
        X = torch.randn((Tn, 136), generator=g, device=DEV).to(dtype)
        Y, _ = T.adapter_forward(X, P)
        assert rel(Y, X.double() @ W.T) <= TOL[dtype]


def ref_activations(X):
    T_, b = X.shape
    out = torch.zeros((T_, b), dtype=F64, device=DEV)
    exps = []
    for j in range(0, b, 32):
        x = X[:, j:j + 32].double()
        top = x.abs().amax(1)
        e = torch.frexp(top).exponent - 7
        e = torch.where(torch.round(torch.ldexp(top, -e)) > 127, e + 1, e).clamp(-126, 121)
        q = torch.round(torch.ldexp(x, -e[:, None])).clamp(-127, 127)
        out[:, j:j + 32] = torch.ldexp(q, e[:, None])
        exps.append(torch.where(top > 0, e + 127, 0))
    return out, torch.stack(exps, 1)


@BOTH
@pytest.mark.parametrize("Tn, b, pad", [(1, 8, 0), (3, 32, 8), (7, 40, 0), (33, 520, 0), (100, 1752, 40),
                                        (5, 65536, 0), (1025, 264, 0), (9000, 64, 0)])
def test_pack_activations(T, Tn, b, pad, dtype):
    g = torch.Generator(device=DEV).manual_seed(Tn + b)
    X = torch.randn((Tn, b + pad), generator=g, device=DEV) * torch.exp(
        4 * torch.randn((Tn, 1), generator=g, device=DEV))
    X = X.to(dtype)[:, :b]
    if Tn > 2:
        X[1] = 0
        X[2] = -127.6
    P = T.pack_activations(X)
    values, exps = ref_activations(X)
    assert torch.equal(P.exps.long(), exps.long())
    assert P.codes.shape == (Tn, b) and int(P.codes.min()) >= -127
    for out in (BF16, F32):
        assert torch.equal(T.unpack_activations(P, out).double(), values)
    step = torch.exp2((exps - 127).double()).repeat_interleave(32, 1)[:, :b]
    assert bool(((values - X.double()).abs() <= 0.5 * step).all())
    again = T.pack_activations(T.unpack_activations(P, dtype))   # what is packed packs to itself
    assert torch.equal(T.unpack_activations(again, F32).double(), values)


@BOTH
def test_pack_activations_at_the_ends_of_the_type(T, dtype):
    big = torch.finfo(dtype).max
    X = torch.zeros((9, 64), device=DEV)
    X[0] = big
    X[1] = -big
    X[2] = 2.0 ** -126
    X[3] = 2.0 ** -133                     # below half a step of the smallest power
    X[4, 3], X[4, 4], X[4, 40] = math.inf, 5.0, 2.0
    X[5, 3] = -math.inf
    X[6, 3], X[6, 7] = math.nan, math.inf
    X[7] = 127.0
    X[8] = 128.0
    X = X.to(dtype)
    P = T.pack_activations(X)
    U = T.unpack_activations(P, F32)
    fine = [2, 3, 7, 8]
    assert torch.equal(U[fine].double(), ref_activations(X[fine])[0])
    # the largest numbers keep code 127: at most a step of 2^121 short
    assert bool(U.isfinite()[:2].all()) and bool(((U[0].double() - big).abs() <= 2.0 ** 121).all())
    assert torch.equal(U[0], -U[1])
    assert U[4, 3].item() == math.inf and U[4, 4].isnan() and U[4, 40].item() == 2.0
    assert U[5, 3].item() == -math.inf and U[5, 0].isnan() and U[6, 3].isnan()
    assert U[6, 7].item() == math.inf and bool((U[4:7, 32:].isfinite()).all())


SHAPES = [
    # T, c, b, n, r, order
    (1, 1, 8, 0, 0, "one"),
    (1, 64, 64, 1, 4, "one"),
    (1, 4096, 4096, 0, 0, "one"),
    (2, 130, 72, 3, 1, "mixed"),
    (5, 1001, 1752, 2, 12, "mixed"),
    (7, 17, 136, 4, 128, "mixed"),
    (8, 2000, 512, 8, 16, "mixed"),
    (9, 333, 11008, 2, 8, "mixed"),
    (16, 256, 520, 16, 16, "blocks"),
    (17, 1, 1032, 2, 8, "mixed"),
    (31, 777, 1000, 5, 20, "mixed"),
    (33, 515, 264, 40, 5, "mixed"),
    (64, 640, 2056, 64, 16, "blocks"),
    (65, 640, 2056, 3, 16, "none"),
    (129, 384, 1096, 2, 128, "mixed"),
    (300, 512, 520, 0, 0, "one"),
    (700, 1536, 1000, 50, 7, "mixed"),
]


def operands(T, shape, dtype, group, seed, pad=8):
    Tn, c, b, n, r, order = shape
    X, W, A, B, index, scale, dY = make(Tn, c, b, max(n, 1), max(r, 1), dtype, seed=seed, order=order,
                                        pad=pad)
    P = T.pack_weights(W, group)
    if n == 0:
        A = B = index = scale = None
    return X, P, T.unpack_weights(P, F32), A, B, index, scale, dY


@BOTH
@pytest.mark.parametrize("group", [64, 128])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_forward(T, shape, group, dtype):
    Tn, c, b, n, r, order = shape
    X, P, W, A, B, index, scale, _ = operands(T, shape, dtype, group, seed=Tn + c)
    out = torch.full((Tn + 1, c + 3), math.nan, dtype=dtype, device=DEV)
    Y, V = T.adapter_forward(X, P, A, B, index, scale, out=out[:Tn, :c], check=True)
    if n:
        Yr, Vr = ref_forward(X, W, A, B, index, scale)
        assert rel(V, Vr) <= TOL[F32] and bool((V[index < 0] == 0).all())
    else:
        Yr = X.double() @ W.double().T
        assert V is None
    assert rel(Y, Yr) <= TOL[dtype]
    err = (Y.double() - Yr).norm(dim=1) / Yr.norm(dim=1).clamp(min=1e-30)
    assert err.max().item() <= (2 if dtype == BF16 else 3) * TOL[dtype] * (1 if c > 8 else 4)
    assert bool(out[Tn:].isnan().all()) and bool(out[:, c:].isnan().all())
    again, _ = T.adapter_forward(X, P, A, B, index, scale)
    assert torch.equal(again, Y)


@BOTH
@pytest.mark.parametrize("packed", ["w", "x", "wx"])
@pytest.mark.parametrize("shape", [s for s in SHAPES if s[3]], ids=lambda s: "x".join(map(str, s)))
def test_backward(T, shape, packed, dtype):
    Tn, c, b, n, r, order = shape
    X, P, W, A, B, index, scale, dY = operands(T, shape, dtype, 64, seed=Tn + c + 1)
    Wd = W if "w" in packed else W.to(dtype)
    X8 = T.pack_activations(X)
    Xd = T.unpack_activations(X8, F32) if "x" in packed else X
    V = ref_forward(X, W, A, B, index, scale)[1].float()
    args = (X8 if "x" in packed else X, V, P if "w" in packed else Wd, A, B, index, scale)
    dX, dA, dB = T.adapter_backward(dY, *args, check=True)
    rX, rA, rB = ref_backward(dY, Xd, V, Wd, A, B, index, scale)
    assert rel(dX, rX) <= TOL[dtype]
    assert rel(dA, rA) <= TOL[F32] and rel(dB, rB) <= TOL[F32]
    for i in range(n):
        if bool((index == i).any()):
            assert rel(dA[i], rA[i]) <= 2 * TOL[F32] and rel(dB[i], rB[i]) <= 2 * TOL[F32]
        else:
            assert not bool(dA[i].any()) and not bool(dB[i].any())
    sA, sB = torch.full_like(dA, 0.5), torch.full_like(dB, -0.25)
    none, tA, tB = T.adapter_backward(dY, *args, need_dx=False, dA=sA, dB=sB, accumulate=True)
    assert none is None
    for total, was, part in ((tA, 0.5, rA), (tB, -0.25, rB)):   # one more rounding, of the new sum
        err = (total.double() - was - part).norm()
        assert err <= TOL[F32] * part.norm() + 2.0 ** -24 * (part.abs() + abs(was)).norm()
    only, nA, nB = T.adapter_backward(dY, *args, need_grads=False)
    assert torch.equal(only, dX) and nA is None and nB is None


@BOTH
@pytest.mark.parametrize("Tn", [3, 20, 50, 200])
def test_a_token_that_is_not_finite_stays_alone(T, Tn, dtype):
    shape = (Tn, 96, 328, 2, 8, "mixed")
    X, P, W, A, B, index, scale, _ = operands(T, shape, dtype, 64, seed=3)
    want, _ = T.adapter_forward(X, P, A, B, index, scale)
    X = X.clone()
    X[1, 5], X[2, 300] = math.inf, math.nan
    Y, V = T.adapter_forward(X, P, A, B, index, scale)
    keep = [t for t in range(Tn) if t not in (1, 2)]
    assert torch.equal(Y[keep], want[keep])
    assert bool(Y[2].isnan().all())
    # infinity times a weight: its sign, or NaN where the weight is zero
    w = W[:, 5]
    if int(index[1]) < 0:
        assert bool((Y[1][w > 0] == math.inf).all()) and bool((Y[1][w < 0] == -math.inf).all())
    assert bool(Y[1][w == 0].isnan().all())


@BOTH
@pytest.mark.parametrize("Tn", [3, 20, 50, 200])
def test_activations_up_to_the_stated_limit(T, Tn, dtype):
    """Few tokens: 64 products of a code (8 at most) and an activation are summed before the scale is
    applied, 2^9 times the largest activation: below 2^119 no sum overflows that is finite in the end."""
    X, P, W, *_ = operands(T, (Tn, 96, 328, 2, 8, "mixed"), dtype, 64, seed=5)
    X = (X.double() / X.double().abs().max() * 2.0 ** 119 * (1 - 2.0 ** -8)).to(dtype)
    want = X.double() @ W.double().t()
    assert float(want.abs().max()) < 2.0 ** 126
    Y, _ = T.adapter_forward(X, P)
    assert rel(Y.double() * 2.0 ** -119, want * 2.0 ** -119) < TOL[dtype]


@BOTH
def test_gradients_of_packed_activations_that_are_not_finite(T, dtype):
    """An infinity in a token of adapter 0 reaches dA of adapter 0 in that column's group, nothing else."""
    shape = (90, 64, 136, 3, 8, "blocks")
    X, P, W, A, B, index, scale, dY = operands(T, shape, dtype, 64, seed=4)
    V = ref_forward(X, W, A, B, index, scale)[1].float()
    _, want, wantB = T.adapter_backward(dY, T.pack_activations(X), V, P, A, B, index, scale)
    X = X.clone()
    X[0, 70] = math.inf
    _, dA, dB = T.adapter_backward(dY, T.pack_activations(X), V, P, A, B, index, scale)
    assert int(index[0]) == 0
    assert not bool(dA[0, :, 64:96].isfinite().any())
    cols = [j for j in range(136) if not 64 <= j < 96]
    assert torch.equal(dA[0][:, cols], want[0][:, cols])
    assert torch.equal(dA[1:], want[1:]) and torch.equal(dB, wantB)


@BOTH
@pytest.mark.parametrize("Tn", [4, 40, 100])
def test_an_index_that_names_no_adapter(T, Tn, dtype):
    shape = (Tn, 96, 128, 3, 8, "mixed")
    X, P, W, A, B, index, scale, dY = operands(T, shape, dtype, 128, seed=5)
    bad = index.clone()
    bad[2] = 3
    none = index.clone()
    none[2] = -1
    with pytest.raises(T.ThanosError) as e:
        T.adapter_forward(X, P, A, B, bad, scale, check=True)
    assert e.value.code == 1
    Y, V = T.adapter_forward(X, P, A, B, bad, scale)
    Yn, Vn = T.adapter_forward(X, P, A, B, none, scale, check=True)
    assert torch.equal(Y, Yn) and torch.equal(V, Vn)
    T.adapter_forward(X, P, check=True)


def test_calls(T):
    """Another stream, two calls at once, a captured graph, single rows, nothing to do."""
    shape = (12, 640, 1032, 3, 16, "mixed")
    X, P, W, A, B, index, scale, dY = operands(T, shape, BF16, 64, seed=6)
    Y, V = T.adapter_forward(X, P, A, B, index, scale)
    X8 = T.pack_activations(X)
    want = T.adapter_backward(dY, X8, V, P, A, B, index, scale)
    streams = [torch.cuda.Stream() for _ in range(3)]
    torch.cuda.synchronize()
    got = [T.adapter_forward(X, P, A, B, index, scale, stream=s, check=True) for s in streams]
    back = [T.adapter_backward(dY, X8, V, P, A, B, index, scale, stream=s) for s in streams]
    torch.cuda.synchronize()
    for (y, v), g in zip(got, back):
        assert torch.equal(y, Y) and torch.equal(v, V)
        assert all(torch.equal(p, q) for p, q in zip(g, want))
    graph = torch.cuda.CUDAGraph()
    buf = X.clone()
    with torch.cuda.graph(graph):
        yg, vg = T.adapter_forward(buf, P, A, B, index, scale)
        x8 = T.pack_activations(buf)
        gg = T.adapter_backward(dY, x8, vg, P, A, B, index, scale)
    for k in (1.0, -0.5):
        buf.copy_(X * k)
        graph.replay()
        y, v = T.adapter_forward(X * k, P, A, B, index, scale)
        g = T.adapter_backward(dY, T.pack_activations(X * k), v, P, A, B, index, scale)
        assert torch.equal(yg, y) and torch.equal(vg, v)
        assert all(torch.equal(p, q) for p, q in zip(gg, g))
    # rows one at a time, from a batch whose rows lie apart
    one, _ = T.adapter_forward(X[3:4], P, A, B, index[3:4], scale)
    assert rel(one, Y[3:4]) <= 2.0 ** -8
    x1 = T.pack_activations(X[3:4])
    assert torch.equal(T.unpack_activations(x1), T.unpack_activations(X8)[3:4])
    sliced = T.PackedActivations(X8.codes[3:4], X8.exps[3:4].clone())
    assert torch.equal(T.unpack_activations(sliced), T.unpack_activations(X8)[3:4])
    before = T.launch_count()
    Y0, V0 = T.adapter_forward(X[:0], P, A, B, index[:0], scale)
    assert Y0.shape == (0, 640) and V0.shape == (0, 16)
    x0 = T.pack_activations(X[:0])
    assert T.unpack_activations(x0).shape == (0, 1032)
    _, dA, dB = T.adapter_backward(dY[:0], x0, V0, P, A, B, index[:0], scale)
    assert not bool(dA.any()) and not bool(dB.any()) and T.launch_count() == before


def test_refusals(T):
    shape = (12, 64, 128, 3, 16, "mixed")
    X, P, W, A, B, index, scale, dY = operands(T, shape, BF16, 64, seed=7, pad=0)
    V = torch.zeros((12, 16), device=DEV)
    with pytest.raises(ValueError):
        T.pack_weights(W, 32)
    with pytest.raises(T.ThanosError):
        T.pack_weights(W[:, :100].contiguous())
    with pytest.raises(TypeError):
        T.pack_weights(W.half())
    for bad in (P._replace(group=32), P._replace(cols=512), P._replace(codes=P.codes.to(torch.int8)),
                P._replace(scales=P.scales.float()), P._replace(scales=P.scales[:1]),
                P._replace(codes=P.codes.cpu()), P._replace(codes=P.codes.t())):
        with pytest.raises(ValueError):
            T.adapter_forward(X, bad, A, B, index, scale)
    X8 = T.pack_activations(X)
    for bad in (X8._replace(codes=X8.codes[:5]), X8._replace(exps=X8.exps[:, :2]),
                X8._replace(codes=X8.codes.to(torch.uint8)), X8._replace(exps=X8.exps.cpu())):
        with pytest.raises(ValueError):
            T.adapter_backward(dY, bad, V, P, A, B, index, scale)
    with pytest.raises(ValueError):
        T.adapter_backward(dY, T.pack_activations(X[:5]), V, P, A, B, index, scale)
    with pytest.raises(T.ThanosError):      # a leading dimension that is no multiple of 16
        T.unpack_activations(T.PackedActivations(
            torch.zeros((4, 40), dtype=torch.int8, device=DEV),
            torch.zeros((4, 4), dtype=torch.uint8, device=DEV)[:, :2]))


def test_offsets_beyond_32_bits(T):
    """Codes past 2^32 bytes and outputs past 2^31 elements: the last rows and tokens are right."""
    c, b = 1 << 20, 8256
    g = torch.Generator(device=DEV).manual_seed(8)
    codes = torch.randint(0, 256, (c, b // 2), generator=g, device=DEV, dtype=torch.uint8)
    scales = torch.full((b // 64, c), 0.0625, dtype=BF16, device=DEV)
    P = T.PackedWeights(codes, scales, 64, b)
    X = torch.randn((3, b), generator=g, device=DEV).to(BF16)
    Y, _ = T.adapter_forward(X, P)
    for rows in (slice(0, 100), slice(c - 100, c)):
        part = T.PackedWeights(codes[rows], scales[:, rows].contiguous(), 64, b)
        assert torch.equal(T.adapter_forward(X, part)[0], Y[:, rows])
    out = torch.empty((2050, 1 << 20), dtype=BF16, device=DEV)[:, :64]
    part = T.PackedWeights(codes[:64], scales[:, :64].contiguous(), 64, b)
    Xl = X.repeat(2, 1)
    T.adapter_forward(Xl, part, out=out[2044:])
    assert torch.equal(out[2044:], T.adapter_forward(Xl, part)[0])


MORE = [
    # T, c, b, n, r, order: every kernel, slice of k and width of token tiles
    (1, 5000, 136, 2, 4, "one"),
    (8, 4737, 4200, 3, 8, "mixed"),
    (12, 4800, 264, 0, 0, "one"),
    (16, 6000, 2056, 4, 12, "mixed"),
    (20, 100, 16400, 2, 8, "mixed"),
    (48, 12000, 520, 3, 16, "mixed"),
    (80, 300, 4104, 5, 16, "mixed"),
    (100, 2000, 1096, 0, 0, "one"),
    (128, 1000, 1032, 3, 20, "mixed"),
    (200, 260, 2056, 0, 0, "one"),
    (256, 129, 72, 0, 0, "one"),
    (256, 700, 264, 2, 8, "mixed"),
    (3, 200, 65536, 1, 4, "one"),
    (40, 200, 65536, 1, 4, "one"),
]


@BOTH
@pytest.mark.parametrize("group", [64, 128])
@pytest.mark.parametrize("shape", MORE, ids=lambda s: "x".join(map(str, s)))
def test_forward_by_every_kernel(T, shape, group, dtype):
    """As test_forward; sums of 65536 terms in fp32 may be off by a few more roundings: 2e-5."""
    Tn, c, b, n, r, order = shape
    X, P, W, A, B, index, scale, _ = operands(T, shape, dtype, group, seed=Tn + c, pad=0)
    out = torch.full((Tn + 1, c + 5), math.nan, dtype=dtype, device=DEV)
    Y, V = T.adapter_forward(X, P, A, B, index, scale, out=out[:Tn, :c], check=True)
    if n:
        Yr, Vr = ref_forward(X, W, A, B, index, scale)
        assert rel(V, Vr) <= TOL[F32]
    else:
        Yr = X.double() @ W.double().T
    tol = 2e-5 if dtype == F32 and b > 10000 else TOL[dtype]
    assert rel(Y, Yr) <= tol
    err = (Y.double() - Yr).norm(dim=1) / Yr.norm(dim=1)
    assert err.max().item() <= 2 * tol
    worst = (Y.double() - Yr).abs().max(0).values          # and no row of weights by itself
    assert bool((worst <= 0.05 * Yr.abs().max()).all())
    assert bool(out[Tn:].isnan().all()) and bool(out[:, c:].isnan().all())
    again, _ = T.adapter_forward(X, P, A, B, index, scale)
    assert torch.equal(again, Y)


def test_more_rows_than_a_grid_is_high(T):
    """65535 rounds of four rows and more: the last rows are packed and unpacked as they are alone."""
    n, b = 4 * 65535 + 700, 2056
    g = torch.Generator(device=DEV).manual_seed(9)
    X = torch.empty((n, b), dtype=BF16, device=DEV).normal_(generator=g)
    P, X8 = T.pack_weights(X, 64), T.pack_activations(X)
    W, U = T.unpack_weights(P), T.unpack_activations(X8)
    for rows in (slice(0, 50), slice(n - 900, n)):
        part = X[rows].contiguous()
        Pp, Xp = T.pack_weights(part, 64), T.pack_activations(part)
        assert torch.equal(P.codes[rows], Pp.codes) and torch.equal(P.scales[:, rows], Pp.scales)
        assert torch.equal(X8.codes[rows], Xp.codes) and torch.equal(X8.exps[rows], Xp.exps)
        assert torch.equal(W[rows], T.unpack_weights(Pp))
        assert torch.equal(U[rows], T.unpack_activations(Xp))


def test_every_scale_and_every_code(T):
    """All largest values of eight bits, and beside each all smaller ones down to a 32nd of a step: the
    ties that a quotient of eight bits over five can be, both signs, against float64."""
    tops = (torch.arange(128, device=DEV).float() / 128 + 1).to(BF16)          # [1, 2)
    fine = torch.cat([(torch.arange(128, device=DEV).float() / 128 + 1) * 2.0 ** -e for e in range(10)])
    cols = -(-fine.numel() // 63)
    grid = torch.zeros(cols * 63, device=DEV)
    grid[:fine.numel()] = fine
    W = torch.zeros((128, cols, 64), device=DEV)
    W[:, :, 0] = tops[:, None].float()
    W[:, :, 1:] = torch.minimum(grid.view(1, cols, 63), tops.float()[:, None, None])
    W = torch.cat([W.view(128, -1), -W.view(128, -1)]).to(BF16).contiguous()
    for k in (1.0, 2.0 ** 100, 2.0 ** -100):
        for dtype in (BF16, F32):
            Wk = (W.float() * k).to(dtype)
            P = T.pack_weights(Wk, 64)
            codes, scales, values = ref_weights(Wk, 64)
            assert torch.equal(P.scales.double(), scales)
            assert torch.equal(nibbles(P)[:, :Wk.shape[1]], codes)
            assert torch.equal(T.unpack_weights(P, F32).double(), values)


# Rows of adapters held for several tokens, in one slice of k and in several, two CTAs to an SM and one;
# tokens one by one beside them, of more and of fewer ranks; sixteen tokens of many rows.
TOGETHER = [
    (128, 12000, 264, 1, 64, "mixed"),
    (97, 12000, 264, 2, 40, "mixed"),
    (125, 8200, 136, 2, 56, "mixed"),
    (64, 19200, 264, 1, 64, "mixed"),
    (50, 19300, 72, 2, 24, "blocks"),
    (128, 300, 4104, 1, 64, "mixed"),
    (100, 1000, 2056, 2, 32, "blocks"),
    (128, 12000, 264, 100, 64, "mixed"),
    (128, 2100, 520, 2, 128, "mixed"),
    (64, 2100, 520, 2, 20, "mixed"),
    (128, 12000, 264, 40, 16, "mixed"),
    (16, 5001, 264, 3, 16, "mixed"),
    (11, 9001, 136, 2, 12, "mixed"),
    (200, 300, 1032, 3, 40, "mixed"),
    (256, 12000, 136, 4, 64, "mixed"),
    (177, 2000, 2056, 9, 16, "blocks"),
    (257, 700, 264, 3, 24, "mixed"),
]


@BOTH
@pytest.mark.parametrize("shape", TOGETHER, ids=lambda s: "x".join(map(str, s)))
def test_forward_of_tokens_that_share_adapters(T, shape, dtype):
    """As test_forward; one index names no adapter, as if it were none."""
    Tn, c, b, n, r, order = shape
    X, P, W, A, B, index, scale, _ = operands(T, shape, dtype, 128, seed=Tn + r)
    out = torch.full((Tn + 1, c + 5), math.nan, dtype=dtype, device=DEV)
    Y, V = T.adapter_forward(X, P, A, B, index, scale, out=out[:Tn, :c], check=True)
    Yr, Vr = ref_forward(X, W, A, B, index, scale)
    assert rel(V, Vr) <= TOL[F32]
    err = (Y.double() - Yr).norm(dim=1) / Yr.norm(dim=1)
    assert err.max().item() <= 2 * TOL[dtype]
    worst = (Y.double() - Yr).abs().max(0).values
    assert bool((worst <= 0.05 * Yr.abs().max()).all())
    assert bool(out[Tn:].isnan().all()) and bool(out[:, c:].isnan().all())
    bad, none = index.clone(), index.clone()
    bad[Tn // 2], none[Tn // 2] = n, -1
    with pytest.raises(T.ThanosError):
        T.adapter_forward(X, P, A, B, bad, scale, check=True)
    Yb, _ = T.adapter_forward(X, P, A, B, bad, scale)
    Yn, _ = T.adapter_forward(X, P, A, B, none, scale, check=True)
    assert torch.equal(Yb, Yn)
    keep = [t for t in range(Tn) if t != Tn // 2]
    assert torch.equal(Yn[keep], Y[keep])


@BOTH
@pytest.mark.parametrize("shape", [(100, 640, 1032, 3, 16, "mixed"), (300, 515, 520, 0, 0, "one"),
                                   (1100, 264, 9000, 2, 8, "mixed"), (900, 9001, 136, 2, 12, "mixed")],
                         ids=lambda s: "x".join(map(str, s)))
def test_no_more_scratch_than_is_asked_for(T, shape, dtype):
    """A workspace of the stated size, memory behind it that stays as it is; gradients alone need no room
    for unpacked weights."""
    Tn, c, b, n, r, order = shape
    X, P, W, A, B, index, scale, dY = operands(T, shape, dtype, 64, seed=c)
    size, dt = T.load_library().thanos_adapter_packed_workspace_bytes, int(dtype == BF16)
    args = (A, B, index, scale)

    def room(nbytes):
        buf = torch.full((nbytes + 4096,), 0xAB, dtype=torch.uint8, device=DEV)
        return buf[:nbytes], buf[nbytes:]

    want, V = T.adapter_forward(X, P, *args)
    ws, behind = room(size(0, 1, 0, Tn, c, b, n, r, dt))
    Y, _ = T.adapter_forward(X, P, *args, workspace=ws, check=True)
    assert torch.equal(Y, want) and bool((behind == 0xAB).all())
    with pytest.raises(T.ThanosError):
        T.adapter_forward(X, P, *args, workspace=ws[:-1])
    X8 = T.pack_activations(X)
    full = T.adapter_backward(dY, X8, V, P, *args)
    ws, behind = room(size(1, 1, 1, Tn, c, b, n, r, dt))
    got = T.adapter_backward(dY, X8, V, P, *args, workspace=ws, check=True)
    assert bool((behind == 0xAB).all())
    for x, y in zip(got, full):
        assert x is y is None or torch.equal(x, y)
    with pytest.raises(T.ThanosError):
        T.adapter_backward(dY, X8, V, P, *args, workspace=ws[:-1])
    if n:
        ws, behind = room(min(size(1, p, 1, Tn, c, b, n, r, dt) for p in (0, 1)))
        none, dA, dB = T.adapter_backward(dY, X8, V, P, *args, need_dx=False, workspace=ws, check=True)
        assert none is None and bool((behind == 0xAB).all())
        assert torch.equal(dA, full[1]) and torch.equal(dB, full[2])
        # and that is what a call without a workspace takes
        del ws, behind
        torch.cuda.synchronize()
        torch.cuda.reset_peak_memory_stats()
        before = torch.cuda.memory_allocated()
        out = T.adapter_backward(dY, X8, V, P, *args, need_dx=False)
        held = torch.cuda.memory_allocated() - before
        assert len(out) == 3
        assert torch.cuda.max_memory_allocated() - before - held <= min(
            size(1, p, 1, Tn, c, b, n, r, dt) for p in (0, 1)) + 4096
