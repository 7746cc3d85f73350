"""What the packed operands' calls refuse, through the C ABI and without a GPU: every refusal comes back
before a kernel is launched."""

import ctypes

import pytest

OK, INVALID, SHAPE, DTYPE, ALIGNMENT, WORKSPACE = 0, 1, 2, 3, 4, 5
F32, BF16 = 0, 1


@pytest.fixture(scope="module")
def lib():
    from paper_2504_05346_b200 import build as B
    import paper_2504_05346_b200 as T

    B.build()
    return T.load_library()


@pytest.fixture(scope="module")
def at():
    """A 16-byte aligned host address: none of these calls gets as far as reading it."""
    buf = (ctypes.c_char * 4096)()
    yield (ctypes.addressof(buf) + 255) // 256 * 256
    del buf


CALLS = {
    "thanos_pack_weights": dict(codes="p", ldq=64, scales="p", W="p", ldw=128, dtype=BF16, c=8, b=104,
                                group=64),
    "thanos_unpack_weights": dict(W="p", ldw=128, dtype=BF16, codes="p", ldq=64, scales="p", c=8, b=104,
                                  group=64),
    "thanos_pack_activations": dict(codes="p", ldc=112, exps="p", lde=4, X="p", ldx=104, dtype=BF16,
                                    T=5, b=104),
    "thanos_unpack_activations": dict(X="p", ldx=104, dtype=BF16, codes="p", ldc=112, exps="p", lde=4,
                                      T=5, b=104),
    "thanos_adapter_forward_packed": dict(
        Y="p", ldy=64, V="p", X="p", ldx=104, codes="p", ldq=64, scales="p", group=64, A="p", B="p",
        index="p", scale="p", dtype=BF16, T=8, c=64, b=104, n=2, r=4, ws="p", ws_bytes=1 << 30),
    "thanos_adapter_backward_packed": dict(
        dX="p", lddx=104, dA="p", dB="p", accumulate=0, dY="p", lddy=64, X="p", ldx=112, exps="p",
        lde=4, V="p", W="p", ldw=64, scales="p", group=64, A="p", B="p", index="p", scale="p",
        dtype=BF16, T=8, c=64, b=104, n=2, r=4, ws="p", ws_bytes=1 << 30),
}


def call(lib, at, name, **change):
    args = []
    for key, value in {**CALLS[name], **change}.items():
        if value == "p":
            value = at
        elif isinstance(value, str) and value.startswith("p+"):
            value = at + int(value[2:])
        args.append(value)
    return getattr(lib, name)(*args, None)


PW, UW, PA, UA = list(CALLS)[:4]
FWD, BWD = list(CALLS)[4:]
REFUSED = [
    (PW, dict(codes=None), INVALID), (PW, dict(scales=None), INVALID), (PW, dict(W=None), INVALID),
    (PW, dict(group=32), SHAPE), (PW, dict(group=0), SHAPE), (PW, dict(b=100), SHAPE),
    (PW, dict(c=0), SHAPE), (PW, dict(ldq=48), SHAPE), (PW, dict(ldw=96), SHAPE),
    (PW, dict(ldq=72), ALIGNMENT), (PW, dict(ldw=108), ALIGNMENT), (PW, dict(codes="p+8"), ALIGNMENT),
    (PW, dict(W="p+2"), ALIGNMENT), (PW, dict(scales="p+1"), ALIGNMENT), (PW, dict(dtype=2), DTYPE),
    (UW, dict(codes=None), INVALID), (UW, dict(group=256), SHAPE), (UW, dict(ldq=48), SHAPE),
    (UW, dict(ldw=96), SHAPE), (UW, dict(W="p+8"), ALIGNMENT), (UW, dict(dtype=-1), DTYPE),
    (PA, dict(codes=None), INVALID), (PA, dict(exps=None), INVALID), (PA, dict(X=None), INVALID),
    (PA, dict(ldc=96), SHAPE), (PA, dict(lde=0), SHAPE), (PA, dict(b=60), SHAPE), (PA, dict(T=-1), SHAPE),
    (PA, dict(ldx=96), SHAPE), (PA, dict(ldc=120), ALIGNMENT), (PA, dict(lde=5), ALIGNMENT),
    (PA, dict(exps="p+2"), ALIGNMENT), (PA, dict(X="p+8"), ALIGNMENT), (PA, dict(dtype=3), DTYPE),
    (PA, dict(T=0, X=None, codes=None, exps=None), OK),
    (UA, dict(X=None), INVALID), (UA, dict(ldx=100), SHAPE), (UA, dict(ldx=108), ALIGNMENT),
    (UA, dict(T=0), OK),
    (FWD, dict(codes=None), INVALID), (FWD, dict(scales=None), INVALID), (FWD, dict(X=None), INVALID),
    (FWD, dict(index=None), INVALID), (FWD, dict(group=96), SHAPE), (FWD, dict(ldq=48), SHAPE),
    (FWD, dict(ldq=72), ALIGNMENT), (FWD, dict(codes="p+4"), ALIGNMENT), (FWD, dict(b=100), SHAPE),
    (FWD, dict(r=129), SHAPE), (FWD, dict(ldy=63), SHAPE), (FWD, dict(ldx=96), SHAPE),
    (FWD, dict(X="p+2"), ALIGNMENT), (FWD, dict(dtype=4), DTYPE), (FWD, dict(ws=None), WORKSPACE),
    (FWD, dict(ws_bytes=128), WORKSPACE), (FWD, dict(ws="p+8"), ALIGNMENT),
    (BWD, dict(W=None), INVALID), (BWD, dict(X=None), INVALID), (BWD, dict(V=None), INVALID),
    (BWD, dict(dA=None), INVALID), (BWD, dict(group=1), SHAPE), (BWD, dict(ldw=48), SHAPE),
    (BWD, dict(ldx=96), SHAPE), (BWD, dict(lde=3), SHAPE), (BWD, dict(ldx=104), ALIGNMENT),
    (BWD, dict(exps="p+1"), ALIGNMENT), (BWD, dict(lde=6), ALIGNMENT), (BWD, dict(dtype=7), DTYPE),
    (BWD, dict(ws_bytes=1000), WORKSPACE),
    # without scales or exponents W or X is what it is in thanos_adapter_backward
    (BWD, dict(scales=None, group=1, ldw=96), SHAPE), (BWD, dict(exps=None, ldx=100), SHAPE),
    (BWD, dict(scales=None, group=1, ldw=104, ws_bytes=0), WORKSPACE),
]


@pytest.mark.parametrize("name, change, code", REFUSED,
                         ids=lambda v: v[7:] if isinstance(v, str) else
                         ",".join(v) if isinstance(v, dict) else str(v))
def test_refused_before_any_launch(lib, at, name, change, code):
    before = lib.thanos_launch_count()
    assert call(lib, at, name, **change) == code
    assert lib.thanos_launch_count() == before


def test_workspace_query(lib):
    size = lib.thanos_adapter_packed_workspace_bytes
    plain = lib.thanos_adapter_workspace_bytes
    assert 0 < size(0, 1, 0, 1, 4096, 4096, 0, 0, BF16) < 4096       # one token: straight from the codes
    assert size(0, 1, 0, 2048, 4096, 4096, 0, 0, BF16) >= 4096 * 4096 * 2
    assert size(1, 0, 1, 100, 64, 104, 2, 4, F32) >= plain(1, 100, 64, 104, 2, 4, F32)
    assert size(0, 1, 0, 8, 64, 100, 0, 0, BF16) == 0 and size(1, 1, 1, 8, 64, 64, 2, 129, F32) == 0


def test_python_layer_refuses():
    import torch
    import paper_2504_05346_b200 as T

    X = torch.zeros(4, 64)
    P = T.PackedWeights(torch.zeros(8, 32, dtype=torch.uint8), torch.zeros(1, 8, dtype=torch.bfloat16),
                        64, 64)
    for f in (T.pack_weights, T.pack_activations):
        with pytest.raises(ValueError):
            f(X)
    with pytest.raises(ValueError):
        T.unpack_weights(P)
    with pytest.raises(ValueError):
        T.unpack_activations(T.PackedActivations(X.to(torch.int8), torch.zeros(4, 2, dtype=torch.uint8)))
    with pytest.raises(ValueError):
        T.adapter_forward(X, P)


def test_the_short_way_is_built(lib):
    """csrc/calls.cpp is there, is bound to the library, and leaves host tensors to the long way."""
    import torch
    from paper_2504_05346_b200 import binding

    assert binding._calls is not None
    X = torch.zeros(4, 64)
    assert binding._calls.adapter_forward(X, X, None, None, None, None) is None
    assert binding._calls.pack_activations(X) is None and binding._calls.token_logprobs(X, None, 1) is None
    assert binding._calls.pack_weights(None, 64) is None and binding._calls.pack_weights(X) is None


@pytest.mark.parametrize("backward", [0, 1])
def test_scratch_holds_the_weights_once(lib, backward):
    """2 bytes a weight where they are unpacked, in either type, beside what plain operands need without
    theirs; nothing where they are not."""
    size, plain = lib.thanos_adapter_packed_workspace_bytes, lib.thanos_adapter_workspace_bytes
    T, c, b, n, r = 2048, 11008, 4096, 4, 16
    weights = c * b
    # fp32: plain weights are three planes of 2 bytes, packed ones are one
    assert plain(backward, T, c, b, n, r, F32) - size(backward, 1, 0, T, c, b, n, r, F32) >= 4 * weights - 512
    assert size(backward, 1, 0, T, c, b, n, r, BF16) <= plain(backward, T, c, b, n, r, BF16) + 2 * weights + 512
    assert size(backward, 0, 1, T, c, b, n, r, BF16) <= plain(backward, T, c, b, n, r, BF16) + 512
