"""What the token log probabilities refuse, through the C ABI and without a GPU: every refusal comes
back before a kernel is launched."""

import ctypes

import pytest

OK, INVALID, SHAPE, DTYPE, ALIGNMENT = 0, 1, 2, 3, 4
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


FORWARD = dict(logp="p", entropy="p", stats="p", top_index="p", top_logp="p", Z="p", ldz=100,
               dtype=BF16, target="p", T=4, V=100, k=5)
BACKWARD = dict(dZ="p", lddz=100, Z="p", ldz=100, dtype=BF16, stats="p", target="p", dlogp="p",
                entropy="p", dentropy="p", top_index="p", dtop="p", T=4, V=100, k=5)
FWD, BWD = "thanos_token_logprobs", "thanos_token_logprobs_backward"
CALLS = {FWD: FORWARD, BWD: BACKWARD}


def call(lib, at, name, **change):
    args = []
    for key, value in {**CALLS[name], **change}.items():
        if value == "p":
            value = at
        elif isinstance(value, str) and value.startswith("p+"):
            value = at + int(value[2:])
        args.append(value)
    return getattr(lib, name)(*args, None)


REFUSED = [
    (FWD, dict(Z=None), INVALID), (FWD, dict(entropy=None), INVALID),
    (FWD, dict(stats=None), INVALID), (FWD, dict(logp=None), INVALID),
    (FWD, dict(top_index=None), INVALID), (FWD, dict(top_logp=None), INVALID),
    (FWD, dict(dtype=2), DTYPE), (FWD, dict(dtype=-1), DTYPE),
    (FWD, dict(T=-1), SHAPE), (FWD, dict(T=(1 << 24) + 1), SHAPE), (FWD, dict(V=0), SHAPE),
    (FWD, dict(V=(1 << 24) + 1, ldz=1 << 25), SHAPE), (FWD, dict(k=-1), SHAPE),
    (FWD, dict(k=65), SHAPE), (FWD, dict(V=4, k=5), SHAPE), (FWD, dict(ldz=99), SHAPE),
    (FWD, dict(T=1 << 24, V=1 << 20, ldz=1 << 20), SHAPE),       # more than a grid holds
    (FWD, dict(Z="p+1"), ALIGNMENT), (FWD, dict(dtype=F32, Z="p+2"), ALIGNMENT),
    (FWD, dict(target="p+4"), ALIGNMENT), (FWD, dict(stats="p+2"), ALIGNMENT),
    (FWD, dict(top_index="p+4"), ALIGNMENT), (FWD, dict(T=0), OK), (FWD, dict(T=0, Z=None), OK),
    (BWD, dict(dZ=None), INVALID), (BWD, dict(Z=None), INVALID), (BWD, dict(stats=None), INVALID),
    (BWD, dict(target=None), INVALID), (BWD, dict(dlogp=None), INVALID),
    (BWD, dict(entropy=None), INVALID), (BWD, dict(top_index=None), INVALID),
    (BWD, dict(k=0), INVALID), (BWD, dict(dtype=9), DTYPE), (BWD, dict(lddz=99), SHAPE),
    (BWD, dict(ldz=99), SHAPE), (BWD, dict(k=65), SHAPE), (BWD, dict(T=-5), SHAPE),
    (BWD, dict(dZ="p+1"), ALIGNMENT), (BWD, dict(dtop="p+2"), ALIGNMENT),
    (BWD, dict(dentropy="p+1"), ALIGNMENT), (BWD, dict(T=0), OK),
]


@pytest.mark.parametrize("name, change, code", REFUSED,
                         ids=lambda v: v[7:] if isinstance(v, str) else
                         ",".join(v) if isinstance(v, dict) else str(v))
def test_refused_before_any_launch(lib, at, name, change, code):
    before = lib.thanos_launch_count()
    assert call(lib, at, name, **change) == code
    assert lib.thanos_launch_count() == before


def test_python_layer_refuses_host_tensors():
    import torch
    import paper_2504_05346_b200 as T

    Z = torch.zeros(4, 64)
    with pytest.raises(ValueError):
        T.token_logprobs(Z)
    with pytest.raises(ValueError):
        T.token_logprobs_backward(Z, torch.zeros(4, 2))
