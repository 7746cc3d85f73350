"""Binding of the packing calls: weights in 4 bits with group scales, activations in 8 bits."""

from __future__ import annotations

from typing import Optional

import torch

from . import binding
from .binding import (PackedActivations, PackedWeights, _alloc_scope, _check, _device_of,
                      _dtype_code, _on, _packed_activations, _packed_weights, _rows, _stream_ptr,
                      load_library)


def _matrix(t: torch.Tensor, name: str):
    """Rows, columns, device and leading dimension of a matrix."""
    dev = _device_of(t, name)
    if t.dim() != 2:
        raise ValueError("%s must be a matrix" % name)
    rows, cols = t.shape
    return rows, cols, dev, _rows(t, cols, dev, name)


def _target(out: Optional[torch.Tensor], like: torch.Tensor, rows: int, cols: int, dtype):
    if out is None:
        return like.new_empty((rows, cols), dtype=dtype)
    if out.dtype not in (torch.float32, torch.bfloat16) or out.shape[0] != rows:
        raise ValueError("out must be a float32 or bfloat16 matrix of the packed shape")
    return out


def pack_weights(W: torch.Tensor, group: int = 128, stream=None) -> PackedWeights:
    """thanos_pack_weights: W [c, b] (float32 or bfloat16) in 4 bits, groups of 64 or 128 columns of
    a row with a scale of their own.  Zeros stay zeros."""
    lib = load_library()
    if binding._calls is not None and stream is None:
        done = binding._calls.pack_weights(W, group)
        if done is not None:
            return PackedWeights(*done, group, W.shape[1])
    c, b, dev, ldw = _matrix(W, "W")
    dt = _dtype_code(W)
    if group not in (64, 128):
        raise ValueError("group must be 64 or 128")
    with _on(W):
        with _alloc_scope(stream):
            codes = W.new_empty((c, -(-b // 64) * 32), dtype=torch.uint8)
            scales = W.new_empty((-(-b // group), c), dtype=torch.bfloat16)
        _check(lib.thanos_pack_weights(codes.data_ptr(), codes.shape[1], scales.data_ptr(),
                                       W.data_ptr(), ldw, dt, c, b, group, _stream_ptr(stream)),
               "thanos_pack_weights")
    return PackedWeights(codes, scales, group, b)


def unpack_weights(W: PackedWeights, dtype=torch.bfloat16, stream=None,
                   out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """thanos_unpack_weights: the weights that the codes stand for, [c, b] (exact in either dtype)."""
    lib = load_library()
    if binding._calls is not None and stream is out is None:
        done = binding._calls.unpack_weights(W, dtype)
        if done is not None:
            return done
    dev = _device_of(W.codes, "the weights' codes")
    c, b, ldq = _packed_weights(W, dev)
    with _on(W.codes):
        with _alloc_scope(stream):
            out = _target(out, W.codes, c, b, dtype)
        _check(lib.thanos_unpack_weights(out.data_ptr(), _rows(out, b, dev, "out"), _dtype_code(out),
                                         W.codes.data_ptr(), ldq, W.scales.data_ptr(), c, b, W.group,
                                         _stream_ptr(stream)), "thanos_unpack_weights")
    return out


def pack_activations(X: torch.Tensor, stream=None) -> PackedActivations:
    """thanos_pack_activations: X [n_tok, b] (float32 or bfloat16) in 8 bits, groups of 32 columns
    of a row with a power of two of their own."""
    lib = load_library()
    if binding._calls is not None and stream is None:
        done = binding._calls.pack_activations(X)
        if done is not None:
            return PackedActivations(*done)
    T, b, dev, ldx = _matrix(X, "X")
    dt = _dtype_code(X)
    groups = -(-b // 32)
    ldc, lde = -(-b // 16) * 16, -(-groups // 4) * 4
    with _on(X):
        with _alloc_scope(stream):
            codes = X.new_empty((T, ldc), dtype=torch.int8)
            exps = X.new_empty((T, lde), dtype=torch.uint8)
        _check(lib.thanos_pack_activations(codes.data_ptr(), ldc, exps.data_ptr(), lde, X.data_ptr(),
                                           ldx, dt, T, b, _stream_ptr(stream)),
               "thanos_pack_activations")
    return PackedActivations(codes if ldc == b else codes[:, :b],
                             exps if lde == groups else exps[:, :groups])


def unpack_activations(X: PackedActivations, dtype=torch.bfloat16, stream=None,
                       out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """thanos_unpack_activations: the values that the codes stand for, [n_tok, b] (exact in either
    dtype)."""
    lib = load_library()
    if binding._calls is not None and stream is out is None:
        done = binding._calls.unpack_activations(X, dtype)
        if done is not None:
            return done
    dev = _device_of(X.codes, "the activations' codes")
    if X.codes.dim() != 2:
        raise ValueError("the activations' codes must be a matrix")
    b = X.codes.shape[1]
    T, ldc, lde = _packed_activations(X, b, dev)
    with _on(X.codes):
        with _alloc_scope(stream):
            out = _target(out, X.codes, T, b, dtype)
        _check(lib.thanos_unpack_activations(out.data_ptr(), _rows(out, b, dev, "out"),
                                             _dtype_code(out), X.codes.data_ptr(), ldc,
                                             X.exps.data_ptr(), lde, T, b, _stream_ptr(stream)),
               "thanos_unpack_activations")
    return out
