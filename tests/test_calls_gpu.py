"""The short way of a call (csrc/calls.cpp) and the long way in Python are the same call: equal results,
the same refusals."""

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

DEV = "cuda"
BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def T():
    import paper_2504_05346_b200 as T_
    from paper_2504_05346_b200 import build as B_

    B_.build()
    T_.load_library()
    return T_


def flat(r):
    if isinstance(r, torch.Tensor) or r is None:
        return [r]
    return [y for x in r for y in (flat(x) if not isinstance(x, int) else [])]


def calls(T):
    g = torch.Generator(device=DEV).manual_seed(1)
    rn = lambda *s: torch.randn(s, generator=g, device=DEV)  # noqa: E731
    out = {}
    Z = rn(5, 300)
    target = torch.tensor([3, -1, 7, 299, 0], device=DEV)
    f = T.token_logprobs(Z, target, 4)
    one, four = rn(5), rn(5, 4)
    for name, z in (("f32", Z), ("bf16", Z.to(BF16)), ("slice", Z[:, 7:207]), ("row", Z[2:3]),
                    ("empty", Z[:0]), ("half", Z.half()), ("turned", Z.t()), ("flat", Z[0]),
                    ("host", Z.cpu())):
        t = target[:z.shape[0]].clamp(max=150) if z.dim() == 2 and z.shape[0] <= 5 else target
        for k in (0, 4, 64, 65, 301, -1):
            out["logp %s %d" % (name, k)] = lambda z=z, t=t, k=k: T.token_logprobs(z, t, k)
        out["logp %s none" % name] = lambda z=z: T.token_logprobs(z)
        n = t.shape[0]
        out["dlogp %s" % name] = lambda z=z, t=t, n=n: T.token_logprobs_backward(
            z, f.stats[:n], t, one[:n], f.entropy[:n], one[:n], f.top_index[:n], four[:n])
    for name, kw in (("no dlogp", dict(target=target)), ("entropy", dict(entropy=f.entropy, dentropy=one)),
                     ("no entropy", dict(dentropy=one)), ("top", dict(top_index=f.top_index, dtop=four)),
                     ("no top", dict(dtop=four)), ("nothing", {}),
                     ("k 0", dict(top_index=f.top_index[:, :0], dtop=four[:, :0])),
                     ("wrong type", dict(target=target.int(), dlogp=one)),
                     ("wrong shape", dict(target=target, dlogp=one[:3]))):
        out["dlogp " + name] = lambda kw=kw: T.token_logprobs_backward(Z, f.stats, **kw)
    W, X = 0.02 * rn(40, 136), rn(6, 136)
    for name, w in (("f32", W), ("bf16", W.to(BF16)), ("slice", W[:, 8:80]), ("row", W[:1]),
                    ("odd", W[:, :100]), ("turned", W.t()), ("half", W.half()), ("host", W.cpu()),
                    ("offset", W[:, 1:129])):
        out["pack w " + name] = lambda w=w: T.pack_weights(w, 64)
        out["pack x " + name] = lambda w=w: T.pack_activations(w)
    out["pack w 32"] = lambda: T.pack_weights(W, 32)
    out["pack x empty"] = lambda: T.pack_activations(X[:0])
    P, X8 = T.pack_weights(W, 64), T.pack_activations(X)
    for dt in (F32, BF16, torch.float16):
        out["unpack w %s" % dt] = lambda dt=dt: T.unpack_weights(P, dt)
        out["unpack x %s" % dt] = lambda dt=dt: T.unpack_activations(X8, dt)
    out["unpack w bad"] = lambda: T.unpack_weights(P._replace(scales=P.scales[:1]))
    out["unpack x bad"] = lambda: T.unpack_activations(X8._replace(exps=X8.exps[:3]))
    A, B, scale = rn(3, 4, 136) / 12, rn(3, 40, 4), rn(3)
    index = torch.tensor([0, 1, -1, 2, 2, 0], device=DEV, dtype=torch.int32)
    dY, V = rn(6, 40), T.adapter_forward(X, W, A, B, index, scale)[1]
    for name, w in (("plain", W), ("packed", P), ("bad", P._replace(cols=999)), ("other", W.to(BF16))):
        out["fwd %s" % name] = lambda w=w: T.adapter_forward(X, w, A, B, index, scale)
        out["fwd %s alone" % name] = lambda w=w: T.adapter_forward(X, w)
        out["fwd %s half" % name] = lambda w=w: T.adapter_forward(X, w, A)
        out["fwd %s rows" % name] = lambda w=w: T.adapter_forward(X[1:2], w, A, B, index[1:2], scale)
        out["fwd %s index" % name] = lambda w=w: T.adapter_forward(X, w, A, B, index.long(), scale)
        for xn, x in (("X", X), ("X8", X8), ("short", X8._replace(codes=X8.codes[:4], exps=X8.exps[:4])),
                      ("none", None)):
            for dx, gr in ((True, True), (True, False), (False, True)):
                out["bwd %s %s %d%d" % (name, xn, dx, gr)] = lambda w=w, x=x, dx=dx, gr=gr: \
                    T.adapter_backward(dY, x, V, w, A, B, index, scale, need_dx=dx, need_grads=gr)
    return out


def result(f):
    try:
        return flat(f())
    except Exception as e:   # what a call refuses, and how
        return type(e), getattr(e, "code", None), str(e)


def test_both_ways_agree(T):
    from paper_2504_05346_b200 import binding

    short = binding._calls
    assert short is not None
    for name, call in calls(T).items():
        a = result(call)
        binding._calls = None
        try:
            b = result(call)
        finally:
            binding._calls = short
        if isinstance(a, tuple) or isinstance(b, tuple):
            assert a == b, name
            continue
        assert len(a) == len(b), name
        for x, y in zip(a, b):
            if x is None or y is None:
                assert x is y, name
                continue
            assert x.dtype == y.dtype and x.shape == y.shape and x.stride() == y.stride(), name
            assert x.device == y.device and not x.requires_grad, name
            assert torch.equal(x.nan_to_num(7.0) if x.is_floating_point() else x,
                               y.nan_to_num(7.0) if y.is_floating_point() else y), name


def test_the_short_way_takes_the_current_stream(T):
    """Inputs are made on another stream behind a wait: a call on the wrong one would read zeros."""
    side = torch.cuda.Stream()
    W = torch.randn((64, 64), device=DEV)
    P = T.pack_weights(W, 64)
    X = torch.zeros((4, 64), device=DEV)
    Xn = torch.randn((4, 64), device=DEV)
    want = T.adapter_forward(Xn, P)[0]
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(20_000_000)
        X.copy_(Xn)
        got = T.adapter_forward(X, P)[0]
    side.synchronize()
    assert torch.equal(got, want)


def test_other_threads_run_while_a_launch_waits(T):
    """A launch waits when the stream's queue is full.  Whoever has to run before it empties (a callback
    of another library, say) must not have to wait for the interpreter's lock meanwhile."""
    import threading
    import time

    Z = torch.zeros((1, 8), device=DEV)
    T.token_logprobs(Z)
    torch.cuda.synchronize()
    ticks, stop = [], threading.Event()

    def tick():
        while not stop.is_set():
            ticks.append(time.perf_counter())
            time.sleep(0.001)

    other = threading.Thread(target=tick)
    other.start()
    try:
        torch.cuda._sleep(1_000_000_000)          # about half a second
        longest = 0.0
        for _ in range(6000):
            a = time.perf_counter()
            T.token_logprobs(Z)
            longest = max(longest, time.perf_counter() - a)
        torch.cuda.synchronize()
    finally:
        stop.set()
        other.join()
    if longest < 0.1:
        pytest.skip("the queue held every launch")
    assert max(b - a for a, b in zip(ticks, ticks[1:])) < longest / 2


@pytest.mark.parametrize("k", [65, 1 << 20, (1 << 31) + 3, (1 << 32) + 3, 1 << 50])
def test_far_too_many_alternatives_are_refused(T, k):
    """By the library, as a shape: no room is made for them first."""
    Z = torch.zeros((4096, 100), device=DEV)
    free = torch.cuda.memory_reserved()
    with pytest.raises(T.ThanosError) as e:
        T.token_logprobs(Z, None, k)
    assert "shape" in str(e.value).lower()
    assert torch.cuda.memory_reserved() - free < 1 << 26
