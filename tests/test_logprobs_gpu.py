"""Token log probabilities, entropy, top alternatives and their gradient against float64.

Tolerances, from the arithmetic (u = 2^-24, a rounding of fp32):
  * log p = (z - m) - log S: z - m and the difference are rounded (u of each), log S has the error of S.
    S is a sum of positive terms, each with an exponential of at most 2 units of 2^-23 and an exponent
    d log2(e) that is off by 2 u |d| (terms count by their size, e^d, and |d| e^d <= 1): 8 u of S at
    most; sums of up to 130 terms in a thread and 20 levels of sums above it: 150 u at most, in
    practice their square root.  log S is off by the same absolutely: 160 u < 1e-5, and one unit of
    log S itself, which is below 20: 2e-6 more.  Absolute: 1.2e-5 + 2 u |log p|.
  * H = log S - (sum e^d d) / S: both sums as above, the second below log V <= 20: 2e-4 at most if all
    roundings went one way; as they do not, 2e-5.
  * the gradient is a product with p (relative 1.2e-5 plus |log p| 2 u <= 2e-5), rounded to its type once:
    2e-5 of the sum of the terms' magnitudes, plus 2^-9 of the result for bf16.
"""

import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

DEV = "cuda"
BF16, F32 = torch.bfloat16, torch.float32
INF = math.inf


@pytest.fixture(scope="module")
def T():
    import paper_2504_05346_b200 as T_
    from paper_2504_05346_b200 import build as B_

    B_.build()
    T_.load_library()
    return T_


def ref_forward(Z, target, k):
    """In float64 on the CPU's terms: the definition, row by row where a row is special."""
    Zd = Z.double()
    m = Zd.amax(1)
    none = m == -INF
    base = torch.where(none, 0.0, m)
    d = Zd - base[:, None]
    S = d.exp().sum(1)
    logS = torch.where(none, 0.0, S.log())
    logq = torch.where(none[:, None], -INF, d - logS[:, None])
    q = logq.exp()
    H = -torch.where(q > 0, q * logq, torch.where(q == 0, 0.0, q)).sum(1)
    logp = None
    if target is not None:
        at = target.clamp(min=0)
        logp = torch.where(target < 0, 0.0, logq.gather(1, at[:, None])[:, 0])
    # order: NaN first, then by value, then by column
    key = torch.where(Zd.isnan(), INF, Zd)
    order = torch.sort(Zd.isnan().double(), dim=1, descending=True, stable=True).indices
    order = order.gather(1, torch.sort(key.gather(1, order), dim=1, descending=True,
                                       stable=True).indices)
    # +infinity and NaN share a key: put NaN in front again
    nan = Zd.isnan().gather(1, order).double()
    order = order.gather(1, torch.sort(nan, dim=1, descending=True, stable=True).indices)[:, :k]
    return logp, H, torch.stack([m, logS], 1), order, logq.gather(1, order), logq


def close(x, ref, tol, rel=2.0 ** -22):
    x, ref = x.double(), ref.double()
    assert torch.equal(x.isnan(), ref.isnan())
    fine = ref.isfinite()
    assert torch.equal(x[~fine & ~ref.isnan()], ref[~fine & ~ref.isnan()])
    err = (x - ref).abs()[fine] - rel * ref.abs()[fine]
    assert err.numel() == 0 or err.max().item() <= tol, err.max().item()


def check_forward(T, Z, target, k):
    f = T.token_logprobs(Z, target, k)
    logp, H, stats, order, top, _ = ref_forward(Z, target, k)
    if target is not None:
        close(f.logp, logp, 1.2e-5)
    else:
        assert f.logp is None
    close(f.entropy, H, 2e-5)
    special = Z.double().amax(1).isfinite() | (Z.double().amax(1) == -INF)
    close(f.stats[special], stats[special], 1.2e-5)
    if k:
        assert torch.equal(f.top_index, order)
        close(f.top_logp, top, 1.2e-5)
    else:
        assert f.top_index is None and f.top_logp is None
    return f


def logits(Tn, V, dtype, seed, spread=3.0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    Z = (spread * torch.randn((Tn, V), generator=g, device=DEV)).to(dtype)
    target = torch.randint(-1, V, (Tn,), generator=g, device=DEV)
    return Z, target


SHAPES = [(1, 1, 1), (1, 2, 2), (3, 7, 5), (2, 8, 8), (5, 9, 3), (4, 63, 63), (7, 64, 64), (2, 65, 64),
          (9, 255, 20), (3, 1000, 16), (1, 2047, 1), (2, 8191, 64), (1, 16384, 10), (3, 32000, 8),
          (1, 50021, 20), (2, 131072, 33), (1, 300001, 64), (600, 511, 7), (333, 10007, 5),
          (1184, 500, 20), (1300, 64, 64), (1200, 8190, 5), (1500, 3, 2)]


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_forward(T, shape, dtype):
    Tn, V, k = shape
    Z, target = logits(Tn, V, dtype, seed=V + Tn)
    f = check_forward(T, Z, target, k)
    again = T.token_logprobs(Z, target, k)
    for x, y in zip(f, again):
        assert torch.equal(x, y)
    check_forward(T, Z, None, 0)


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("offset", [0, 1, 3, 5])
@pytest.mark.parametrize("V, ld", [(100, 117), (4099, 4200), (20001, 20001)])
def test_strided_rows_that_start_anywhere(T, dtype, offset, V, ld):
    g = torch.Generator(device=DEV).manual_seed(V + offset)
    buf = torch.full((5 * ld + 16,), INF, dtype=dtype, device=DEV)   # what is beside a row is not read
    Z = buf[offset:offset + 5 * ld].view(5, ld)[:, :V]
    Z.copy_(2 * torch.randn((5, V), generator=g, device=DEV))
    target = torch.randint(0, V, (5,), generator=g, device=DEV)
    f = check_forward(T, Z, target, 9)
    dlogp = torch.ones(5, device=DEV)
    check_backward(T, Z, f, target, dlogp, None, None)
    # into another buffer of another alignment, whose gaps stay as they are
    out_buf = torch.full((5 * ld + 16,), 7.0, dtype=dtype, device=DEV)
    out = out_buf[2:2 + 5 * ld].view(5, ld)[:, :V]
    dZ = T.token_logprobs_backward(Z, f.stats, target, dlogp, out=out)
    assert dZ is out
    assert torch.equal(out, T.token_logprobs_backward(Z, f.stats, target, dlogp))
    inside = torch.zeros(5 * ld + 16, dtype=torch.bool, device=DEV)
    inside[2:2 + 5 * ld].view(5, ld)[:, :V] = True
    assert bool((out_buf[~inside] == 7.0).all())


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("V, times", [(37, 1), (5000, 1), (40000, 1), (37, 70), (5000, 70)])
def test_special_rows(T, V, times, dtype):
    """Masked, constant and extreme rows, ties, infinities and NaN; a few of them, and among many."""
    big = torch.finfo(dtype).max
    g = torch.Generator(device=DEV).manual_seed(V)
    Z = torch.randn((18, V), generator=g, device=DEV)
    Z[0] = -INF                              # nothing left
    Z[1] = -INF
    Z[1, V - 1] = 3.0                        # one left
    Z[2] = -big                              # the lowest value everywhere: all alike
    Z[3] = -big
    Z[3, 5] = -INF
    Z[4] = big
    Z[5] = 0.0                               # ties all over
    Z[6] = torch.arange(V, device=DEV) % 3   # ties in every place
    Z[7, V // 2:] = -INF                     # fewer than the alternatives, in the smallest case
    Z[7, 3:V // 2] = -INF
    Z[8, 7] = INF
    Z[9, 11] = math.nan
    Z[10] = math.nan
    Z[11, 3], Z[11, 4], Z[11, 5] = math.nan, INF, -INF
    Z[12] = torch.where(torch.arange(V, device=DEV) % 2 == 0, -0.0, 0.0)
    Z[13] = -1e30
    Z[13, 1] = 1e30                          # far apart
    Z[14] = torch.arange(V, device=DEV).float() * 1e-3
    Z[15] = -torch.arange(V, device=DEV).float()
    Z[16] = -big
    Z[16, 2:6] = 50.0
    Z[17] = torch.randint(0, 2, (V,), generator=g, device=DEV) * -big
    Z = Z.to(dtype)
    target = torch.randint(0, V, (18,), generator=g, device=DEV)
    target[5] = -7
    target[9] = -1
    Z, target = Z.repeat(times, 1), target.repeat(times)
    for k in (0, 1, 20, 33):
        check_forward(T, Z, target, k)
    f = check_forward(T, Z, target, 5)
    assert f.entropy[0].item() == 0.0 and f.logp[0].item() == -INF and f.logp[5].item() == 0.0
    fine = [t for t in range(18) if t not in (8, 9, 10, 11)]
    Zf, tf = Z[fine].contiguous(), target[fine].contiguous()
    f = T.token_logprobs(Zf, tf, 5)
    check_backward(T, Zf, f, tf, torch.randn(len(fine), generator=g, device=DEV),
                   torch.randn(len(fine), generator=g, device=DEV),
                   torch.randn((len(fine), 5), generator=g, device=DEV))


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("V, threads, times", [(60000, 256, 1), (7999, 128, 300)])
def test_more_candidates_than_the_list_holds(T, V, threads, times, dtype):
    """Large values that all fall to one thread, in rising order, and many that tie with the k-th."""
    vec = 8 if dtype == BF16 else 4
    Z = torch.zeros((4, V), device=DEV)
    own = (torch.arange(V, device=DEV) // vec) % threads == 17       # columns of one thread
    Z[0, own] = 1.0 + torch.arange(int(own.sum()), device=DEV).float() / 64
    own2 = (torch.arange(V, device=DEV) // vec) % threads < 20
    Z[1, own2] = 2.0
    Z[1, V - 1] = 3.0
    Z[2, ::2] = 1.0
    Z[3] = -INF
    Z[3, 100:130] = 1.0
    Z = Z.to(dtype).repeat(times, 1)
    target = torch.tensor([1, 2, 3, 4], device=DEV).repeat(times)
    for k in (1, 19, 40, 64):
        check_forward(T, Z, target, k)


def test_target_outside_the_vocabulary(T):
    Z, _ = logits(3, 500, F32, seed=1)
    target = torch.tensor([500, 4, 1 << 40], device=DEV)
    f = T.token_logprobs(Z, target, 3)
    assert f.logp[0].isnan() and f.logp[2].isnan() and f.logp[1].isfinite()
    assert f.entropy.isfinite().all() and f.top_logp.isfinite().all()
    dZ = T.token_logprobs_backward(Z, f.stats, target, torch.ones(3, device=DEV))
    assert dZ[0].isnan().all() and dZ[2].isnan().all() and dZ[1].isfinite().all()


def check_backward(T, Z, f, target, dlogp, dentropy, dtop, top=None):
    top = f.top_index if top is None else top
    dZ = T.token_logprobs_backward(Z, f.stats, target, dlogp, entropy=f.entropy, dentropy=dentropy,
                                   top_index=top if dtop is not None else None, dtop=dtop)
    Tn, V = Z.shape
    _, H, _, _, _, logq = ref_forward(Z, target, 0)
    q = logq.exp()
    low = logq.clamp(min=-1e4)
    G = torch.zeros(Tn, dtype=torch.float64, device=DEV)
    add = torch.zeros((Tn, V), dtype=torch.float64, device=DEV)
    size = torch.zeros_like(add)

    def point(at, g):
        ok = (at >= 0) & (at < V)
        g = torch.where(ok, g.double(), 0.0)
        G.add_(g.sum(1))
        for i in range(at.shape[1]):          # one column at a time: the same index twice adds up
            r = torch.arange(Tn, device=DEV)
            add[r, at[:, i].clamp(0, V - 1)] += g[:, i]
            size[r, at[:, i].clamp(0, V - 1)] += g[:, i].abs()

    if target is not None:
        point(target[:, None], dlogp[:, None])
    if dtop is not None:
        point(top, dtop)
    gh = torch.zeros(Tn, dtype=torch.float64, device=DEV) if dentropy is None else dentropy.double()
    dead = Z.double().amax(1) == -INF
    want = add - q * (G[:, None] + gh[:, None] * (low + H[:, None]))
    want[dead] = 0.0
    factor = G.abs()[:, None] + gh.abs()[:, None] * (low.abs() + H[:, None])
    sums = size + q * factor
    if dtop is not None:
        sums += q * dtop.double().abs().sum(1, keepdim=True)
    err = (dZ.double() - want).abs() - 2e-5 * sums
    if Z.dtype == BF16:
        err -= 2.0 ** -8 * want.abs()
    # A p below the smallest normal number, 2^-126, may be cut to zero before it meets its factor:
    # |p factor - 0| <= 2^-126 factor; and so may the product itself, by 2^-126.
    err -= 2.0 ** -126 * (1.0 + factor)
    assert err.max().item() <= 0.0, err.max().item()
    return dZ


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_backward(T, shape, dtype):
    Tn, V, k = shape
    Z, target = logits(Tn, V, dtype, seed=2 * V + Tn)
    g = torch.Generator(device=DEV).manual_seed(V)
    rn = lambda *s: torch.randn(s, generator=g, device=DEV)  # noqa: E731
    f = T.token_logprobs(Z, target, k)
    check_backward(T, Z, f, target, rn(Tn), rn(Tn), rn(Tn, k))
    check_backward(T, Z, f, target, rn(Tn), None, None)
    check_backward(T, Z, f, None, None, rn(Tn), None)
    check_backward(T, Z, f, None, None, None, rn(Tn, k))
    # tokens of any kind, some twice, some that name none
    top = torch.randint(-2, V + 2, (Tn, k), generator=g, device=DEV)
    top[:, k // 2:] = top[:, :k - k // 2].clone()
    dtop = rn(Tn, k)
    dZ = check_backward(T, Z, f, target, rn(Tn).mul_(0).add_(0.5), None, dtop, top)
    # in place: the gradient takes the logits' place
    Zc = Z.clone()
    out = T.token_logprobs_backward(Zc, f.stats, target, torch.full((Tn,), 0.5, device=DEV),
                                    top_index=top, dtop=dtop, out=Zc)
    assert out is Zc and torch.equal(out, dZ)


def test_gradient_against_differences(T):
    """Central differences of the operator's own fp32 forward pass: (f(z + h) - f(z - h)) / 2h with h =
    2^-6 is off by h^2 / 6 times the third derivative (below 1 here: 5e-5) and by the forward pass's own
    error over h: 2e-5 / 2^-6 = 1.3e-3 at most."""
    Z, target = logits(6, 40, F32, seed=5, spread=1.0)
    target = target.clamp(min=0)
    f = T.token_logprobs(Z, target, 3)
    a, b, c = torch.ones(6, device=DEV), torch.full((6,), 0.7, device=DEV), torch.full((6, 3), 0.3, device=DEV)
    dZ = T.token_logprobs_backward(Z, f.stats, target, a, f.entropy, b, f.top_index, c)
    h = 2.0 ** -6

    def value(Z):
        logq = T.token_logprobs(Z, target)
        top = sum(T.token_logprobs(Z, f.top_index[:, i].contiguous()).logp for i in range(3))
        return logq.logp + 0.7 * logq.entropy + 0.3 * top

    for j in range(0, 40, 3):
        up, down = Z.clone(), Z.clone()
        up[:, j] += h
        down[:, j] -= h
        diff = (value(up) - value(down)) / (2 * h)
        assert (diff - dZ[:, j]).abs().max().item() <= 4e-3


def test_left_out_rows_are_zero_whatever_they_hold(T):
    Z, target = logits(4, 1000, BF16, seed=3)
    target = target.clamp(min=0)
    target[1] = -1
    f = T.token_logprobs(Z, target)
    dlogp = torch.ones(4, device=DEV)
    dlogp[1] = math.nan      # not read
    dlogp[2] = 0.0
    Z2 = Z.clone()
    Z2[1], Z2[2] = math.nan, INF
    dZ = T.token_logprobs_backward(Z2, f.stats, target, dlogp)
    assert bool((dZ[1] == 0).all()) and bool((dZ[2] == 0).all())
    assert torch.equal(dZ[0], T.token_logprobs_backward(Z, f.stats, target, dlogp)[0])


def test_calls(T):
    """Another stream, a captured graph that is replayed on new logits, and nothing to do."""
    Z, target = logits(64, 9000, BF16, seed=4)
    f = T.token_logprobs(Z, target, 6)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    fs = T.token_logprobs(Z, target, 6, stream=side)
    side.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(f, fs))
    buf, tgt = Z.clone(), target.clone()
    dl = torch.ones(64, device=DEV)
    with torch.cuda.stream(side):
        T.token_logprobs(buf, tgt, 6)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        fg = T.token_logprobs(buf, tgt, 6)
        dg = T.token_logprobs_backward(buf, fg.stats, tgt, dl, fg.entropy, dl)
    for seed in (4, 5):
        Zn, tn = logits(64, 9000, BF16, seed=seed)
        buf.copy_(Zn)
        tgt.copy_(tn)
        graph.replay()
        want = T.token_logprobs(Zn, tn, 6)
        assert all(torch.equal(x, y) for x, y in zip(fg, want))
        assert torch.equal(dg, T.token_logprobs_backward(Zn, want.stats, tn, dl, want.entropy, dl))
    before = T.launch_count()
    f = T.token_logprobs(Z[:0], target[:0], 6)
    assert f.top_index.shape == (0, 6) and f.logp.shape == (0,)
    assert T.token_logprobs_backward(Z[:0], f.stats, target[:0], f.logp).shape == (0, 9000)
    assert T.launch_count() == before


def test_refusals(T):
    Z, target = logits(4, 100, BF16, seed=6)
    f = T.token_logprobs(Z, target)
    one = torch.ones(4, device=DEV)
    with pytest.raises(T.ThanosError):
        T.token_logprobs(Z, target, 65)
    with pytest.raises(T.ThanosError):
        T.token_logprobs(Z[:, :10], target, 11)
    with pytest.raises(ValueError):
        T.token_logprobs(Z, target.int())
    with pytest.raises(ValueError):
        T.token_logprobs(Z, target[:3])
    with pytest.raises(ValueError):
        T.token_logprobs(Z.t(), None)
    with pytest.raises(TypeError):
        T.token_logprobs(Z.half(), target)
    with pytest.raises(ValueError):
        T.token_logprobs_backward(Z, f.stats, target)
    with pytest.raises(ValueError):
        T.token_logprobs_backward(Z, f.stats, target, one, dentropy=one)
    with pytest.raises(ValueError):
        T.token_logprobs_backward(Z, f.stats, target, one, out=Z.float())
    with pytest.raises(ValueError):
        T.token_logprobs_backward(Z, f.stats, target, one, dtop=one[:, None])


def test_offsets_beyond_32_bits(T):
    """Row offsets past 2^31 elements; rows at both ends of the buffer."""
    V, ld = 1000, 1 << 20
    buf = torch.empty((2100, ld), dtype=BF16, device=DEV)     # 2.2e9 elements
    Z = buf[:, :V]
    Zs, target = logits(2100, V, BF16, seed=7)
    Z.copy_(Zs)
    f, fs = T.token_logprobs(Z, target, 4), T.token_logprobs(Zs, target, 4)
    assert all(torch.equal(x, y) for x, y in zip(f, fs))
    dl = torch.ones(2100, device=DEV)
    T.token_logprobs_backward(Z, f.stats, target, dl, out=Z)
    assert torch.equal(Z, T.token_logprobs_backward(Zs, f.stats, target, dl))


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("Tn, V", [(1, 16384), (2, 40000), (37, 65536), (100, 300001), (147, 32768)])
def test_rows_of_a_cluster_without_alternatives(T, Tn, V, dtype):
    """With and without alternatives a row's sums are the same, added in the same order; where a cluster
    shares a row there are barriers between them in one case only."""
    Z, target = logits(Tn, V, dtype, seed=V)
    want = T.token_logprobs(Z, target, 2)
    check_forward(T, Z, target, 0)
    for _ in range(50):
        f = T.token_logprobs(Z, target, 0)
        for x, y in zip(f[:3], want[:3]):
            assert torch.equal(x, y)
