"""What the recovery operators refuse, through the C ABI and without a GPU: every refusal comes back
before a kernel is launched."""

import ctypes
import os

import pytest

INVALID, SHAPE, DTYPE, ALIGNMENT, WORKSPACE = 1, 2, 3, 4, 5
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


FORWARD = dict(Y="p", ldy=64, V="p", X="p", ldx=64, W="p", ldw=64, A="p", B="p", index="p",
               scale="p", dtype=BF16, T=8, c=64, b=64, n=2, r=4, ws="p", ws_bytes=1 << 30)
BACKWARD = dict(dX="p", lddx=64, dA="p", dB="p", accumulate=0, dY="p", lddy=64, X="p", ldx=64,
                V="p", W="p", ldw=64, A="p", B="p", index="p", scale="p", dtype=BF16, T=8, c=64,
                b=64, n=2, r=4, ws="p", ws_bytes=1 << 30)
ORTHO = dict(O="p", G="p", dtype=F32, batch=1, m=64, n=32, coef=(3.4445, -4.775, 2.0315), steps=5,
             eps=1e-7, ws="p", ws_bytes=1 << 30)
STEP = dict(W_out="p", W_in="p", wdtype=BF16, M_out="p", M_in="p", G="p", gdtype=F32, mask="p",
            batch=1, m=64, n=32, lr=1e-3, gain=1.0, momentum=0.9, nesterov=1, weight_decay=0.1,
            coef=(3.4445, -4.775, 2.0315), steps=5, eps=1e-7, ws="p", ws_bytes=1 << 30)
CALLS = {"thanos_adapter_forward": FORWARD, "thanos_adapter_backward": BACKWARD,
         "thanos_orthogonalise": ORTHO, "thanos_orthogonal_step": STEP}


def call(lib, at, name, **change):
    args = []
    for key, value in {**CALLS[name], **change}.items():
        if value == "p":
            value = at
        elif isinstance(value, str) and value.startswith("p+"):
            value = at + int(value[2:])
        if key == "coef" and value is not None:
            value = (ctypes.c_float * 3)(*value)
        args.append(value)
    return getattr(lib, name)(*args, None)


FWD, BWD = "thanos_adapter_forward", "thanos_adapter_backward"
ORT, STP = "thanos_orthogonalise", "thanos_orthogonal_step"
REFUSED = [
    (FWD, dict(W=None), INVALID), (FWD, dict(X=None), INVALID), (FWD, dict(Y=None), INVALID),
    (FWD, dict(A=None), INVALID), (FWD, dict(B=None), INVALID), (FWD, dict(index=None), INVALID),
    (FWD, dict(scale=None), INVALID),
    (FWD, dict(dtype=2), DTYPE), (FWD, dict(dtype=-1), DTYPE),
    (FWD, dict(b=60), SHAPE), (FWD, dict(b=0), SHAPE), (FWD, dict(b=65544, ldx=65544, ldw=65544), SHAPE),
    (FWD, dict(c=0), SHAPE), (FWD, dict(c=(1 << 20) + 1, ldy=1 << 21), SHAPE),
    (FWD, dict(T=-1), SHAPE), (FWD, dict(T=(1 << 24) + 1), SHAPE),
    (FWD, dict(n=-1), SHAPE), (FWD, dict(n=(1 << 20) + 1), SHAPE),
    (FWD, dict(r=0), SHAPE), (FWD, dict(r=129), SHAPE),
    (FWD, dict(T=1 << 24, n=1 << 15), SHAPE),          # 2^29 tiles of 128 ranks x 32 tokens
    (FWD, dict(ldy=63), SHAPE), (FWD, dict(ldx=56), SHAPE), (FWD, dict(ldw=56), SHAPE),
    (FWD, dict(ldx=68), ALIGNMENT), (FWD, dict(ldw=68), ALIGNMENT),
    (FWD, dict(X="p+8"), ALIGNMENT), (FWD, dict(Y="p+2"), ALIGNMENT), (FWD, dict(V="p+4"), ALIGNMENT),
    (FWD, dict(index="p+2"), ALIGNMENT), (FWD, dict(scale="p+1"), ALIGNMENT),
    (FWD, dict(ws="p+8"), ALIGNMENT), (FWD, dict(ws_bytes=64), WORKSPACE),
    (FWD, dict(ws=None), WORKSPACE),
    # an index or scale that starts between 16-byte lines is no reason to refuse
    (FWD, dict(index="p+4", scale="p+12", ws_bytes=64), WORKSPACE),
    (BWD, dict(W=None), INVALID), (BWD, dict(dY=None), INVALID), (BWD, dict(dA=None), INVALID),
    (BWD, dict(dB=None), INVALID), (BWD, dict(X=None), INVALID), (BWD, dict(V=None), INVALID),
    (BWD, dict(n=0), INVALID),                          # gradients of no adapters
    (BWD, dict(dtype=7), DTYPE), (BWD, dict(r=129), SHAPE), (BWD, dict(b=12), SHAPE),
    (BWD, dict(lddy=60), SHAPE), (BWD, dict(lddx=60), SHAPE), (BWD, dict(ldx=56), SHAPE),
    (BWD, dict(ldx=65), ALIGNMENT), (BWD, dict(dA="p+4"), ALIGNMENT),
    (BWD, dict(index="p+4", ws_bytes=0), WORKSPACE),
    (ORT, dict(O=None), INVALID), (ORT, dict(G=None), INVALID), (ORT, dict(coef=None), INVALID),
    (ORT, dict(steps=0), INVALID), (ORT, dict(steps=33), INVALID),
    (ORT, dict(eps=-1.0), INVALID), (ORT, dict(eps=float("inf")), INVALID),
    (ORT, dict(coef=(float("nan"), 0.0, 0.0)), INVALID),
    (ORT, dict(dtype=3), DTYPE), (ORT, dict(m=0), SHAPE), (ORT, dict(n=65537), SHAPE),
    (ORT, dict(batch=65536), SHAPE), (ORT, dict(batch=-1), SHAPE),
    (ORT, dict(G="p+8"), ALIGNMENT), (ORT, dict(O="p+2"), ALIGNMENT),
    (ORT, dict(ws_bytes=16), WORKSPACE),
    (STP, dict(W_in=None), INVALID), (STP, dict(M_out=None), INVALID), (STP, dict(G=None), INVALID),
    (STP, dict(wdtype=5), DTYPE), (STP, dict(gdtype=5), DTYPE),
    (STP, dict(lr=float("nan")), INVALID), (STP, dict(momentum=float("inf")), INVALID),
    (STP, dict(weight_decay=float("nan")), INVALID), (STP, dict(gain=float("inf")), INVALID),
    (STP, dict(mask="p+1"), ALIGNMENT), (STP, dict(M_in="p+4"), ALIGNMENT),
    (STP, dict(ws=None), WORKSPACE),
    (STP, dict(batch=0), 0),                            # nothing to do
    (ORT, dict(batch=0), 0),
]


@pytest.mark.parametrize("name, change, code", REFUSED,
                         ids=lambda v: v[7:] if isinstance(v, str) else
                         ",".join(v) if isinstance(v, dict) else str(v))
def test_refused_before_any_launch(lib, at, name, change, code):
    before = lib.thanos_launch_count()
    assert call(lib, at, name, **change) == code
    assert lib.thanos_launch_count() == before


def test_workspace_queries(lib):
    size = lib.thanos_adapter_workspace_bytes
    assert size(0, 8, 64, 64, 2, 4, BF16) > 0 and size(1, 8, 64, 64, 2, 4, F32) > 0
    assert size(0, 0, 64, 64, 0, 0, BF16) > 0          # no tokens, no adapters: still a status word
    assert size(1, 4096, 4096, 4096, 8, 16, F32) > size(1, 4096, 4096, 4096, 8, 16, BF16)
    assert size(0, 8, 64, 60, 2, 4, BF16) == 0 and size(0, 8, 64, 64, 2, 129, BF16) == 0
    assert size(0, 8, 64, 64, 2, 4, 9) == 0
    size = lib.thanos_orthogonal_workspace_bytes
    assert size(1, 64, 32) > 0 and size(0, 1, 1) > 0
    assert size(1, 0, 32) == 0 and size(65536, 4, 4) == 0


def test_python_layer_refuses_host_tensors():
    import torch
    import paper_2504_05346_b200 as T

    X, W = torch.zeros(4, 64), torch.zeros(64, 64)
    with pytest.raises(ValueError):
        T.adapter_forward(X, W)
    with pytest.raises(ValueError):
        T.adapter_backward(X, None, None, W, need_grads=False)
    with pytest.raises(ValueError):
        T.orthogonalise(W)
    with pytest.raises(ValueError):
        T.orthogonal_step(W, W, W)


def test_example_names_only_public_entry_points():
    import re
    import paper_2504_05346_b200 as T

    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    src = open(os.path.join(root, "examples", "recover_layer.py")).read()
    used = set(re.findall(r"thanos\.([A-Za-z_]+)\(", src))
    assert {"adapter_forward", "adapter_backward", "orthogonal_step"} <= used
    assert all(hasattr(T, name) for name in used)
