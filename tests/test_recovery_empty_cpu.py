"""An empty batch of matrices is nothing to do, also where an empty tensor has no address; what is
refused with matrices is refused without."""

import pytest

from tests.test_recovery_cpu import (ALIGNMENT, DTYPE, INVALID, ORT, SHAPE, STP, WORKSPACE, at,  # noqa: F401
                                     call, lib)

NONE_O, NONE_S = dict(O=None, G=None), dict(W_out=None, W_in=None, M_out=None, M_in=None, G=None,
                                            mask=None)


@pytest.mark.parametrize("name, change, code", [
    (ORT, dict(batch=0, **NONE_O), 0), (STP, dict(batch=0, **NONE_S), 0),
    (ORT, dict(batch=0, O=None), 0), (STP, dict(batch=0, M_in=None), 0),
    (ORT, dict(batch=1, **NONE_O), INVALID), (STP, dict(batch=1, **NONE_S), INVALID),
    (ORT, dict(batch=-1, **NONE_O), INVALID),
    (ORT, dict(batch=0, coef=None, **NONE_O), INVALID), (ORT, dict(batch=0, steps=0, **NONE_O), INVALID),
    (ORT, dict(batch=0, n=0, **NONE_O), SHAPE), (STP, dict(batch=0, wdtype=7, **NONE_S), DTYPE),
    (ORT, dict(batch=0, ws="p+8", **NONE_O), ALIGNMENT), (STP, dict(batch=0, ws=None, **NONE_S), WORKSPACE),
], ids=lambda v: v[7:] if isinstance(v, str) else ",".join(v) if isinstance(v, dict) else str(v))
def test_empty_batch(lib, at, name, change, code):  # noqa: F811
    before = lib.thanos_launch_count()
    assert call(lib, at, name, **change) == code
    assert lib.thanos_launch_count() == before
