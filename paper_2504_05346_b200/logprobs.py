"""Binding of the token log probabilities: thanos_token_logprobs and its gradient."""

from __future__ import annotations

from typing import NamedTuple, Optional

import torch

from . import binding
from .binding import (_alloc_scope, _check, _dense, _device_of, _dtype_code, _on, _ptr,
                      _stream_ptr, load_library)


class TokenLogprobs(NamedTuple):
    """What token_logprobs returns: float32 logp [n_tok] (None without targets), entropy [n_tok],
    stats [n_tok, 2] (a row's largest logit and the log of its sum of exp(z - largest): add them for
    log sum exp(z)), and with k > 0 int64 top_index and float32 top_logp [n_tok, k]."""

    logp: Optional[torch.Tensor]
    entropy: torch.Tensor
    stats: torch.Tensor
    top_index: Optional[torch.Tensor]
    top_logp: Optional[torch.Tensor]


def _logits(Z: torch.Tensor, name: str):
    """Rows, columns and leading dimension of a matrix of logits with unit inner stride."""
    if Z.dim() != 2:
        raise ValueError("%s must be a matrix [n_tok, vocab]" % name)
    (T, V), (ld, inner) = Z.shape, Z.stride()
    if inner != 1 and V > 1:
        raise ValueError("%s must have unit inner stride" % name)
    return T, V, ld if T > 1 else max(V, 1)


def token_logprobs(Z: torch.Tensor, target: Optional[torch.Tensor] = None, k: int = 0,
                   stream=None) -> TokenLogprobs:
    """thanos_token_logprobs: log probability of target[t] (int64, negative: left out) under the
    logits Z [n_tok, vocab] (float32 or bfloat16), every row's entropy, and its k <= 64 most likely
    tokens with their log probabilities, equal logits by index."""
    lib = load_library()
    if binding._calls is not None and stream is None:
        done = binding._calls.token_logprobs(Z, target, k)
        if done is not None:
            return TokenLogprobs(*done)
    dev = _device_of(Z, "Z")
    T, V, ldz = _logits(Z, "Z")
    dt = _dtype_code(Z)
    if target is not None:
        _dense(target, (T,), torch.int64, dev, "target")
    k = max(-1, min(k, 65))       # the library refuses both ends, before any room is made for more
    with _on(Z):
        with _alloc_scope(stream):
            f32 = torch.float32
            stats = Z.new_empty((T, 2), dtype=f32)
            entropy = Z.new_empty((T,), dtype=f32)
            logp = None if target is None else Z.new_empty((T,), dtype=f32)
            top_index = top_logp = None
            if k > 0:
                top_index = Z.new_empty((T, k), dtype=torch.int64)
                top_logp = Z.new_empty((T, k), dtype=f32)
        _check(lib.thanos_token_logprobs(_ptr(logp), entropy.data_ptr(), stats.data_ptr(),
                                         _ptr(top_index), _ptr(top_logp), Z.data_ptr(), ldz, dt,
                                         _ptr(target), T, V, k, _stream_ptr(stream)),
               "thanos_token_logprobs")
    return TokenLogprobs(logp, entropy, stats, top_index, top_logp)


def token_logprobs_backward(Z: torch.Tensor, stats: torch.Tensor,
                            target: Optional[torch.Tensor] = None,
                            dlogp: Optional[torch.Tensor] = None,
                            entropy: Optional[torch.Tensor] = None,
                            dentropy: Optional[torch.Tensor] = None,
                            top_index: Optional[torch.Tensor] = None,
                            dtop: Optional[torch.Tensor] = None, stream=None,
                            out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """thanos_token_logprobs_backward: gradient by the logits of sum(dlogp logp) + sum(dentropy
    entropy) + sum(dtop top_logp); stats and entropy are what token_logprobs returned.  Any of the
    three may be left out.  out may be Z itself: the gradient then takes the logits' place."""
    lib = load_library()
    if binding._calls is not None and stream is out is None:
        done = binding._calls.token_logprobs_backward(Z, stats, target, dlogp, entropy, dentropy,
                                                      top_index, dtop)
        if done is not None:
            return done
    dev = _device_of(Z, "Z")
    T, V, ldz = _logits(Z, "Z")
    dt = _dtype_code(Z)
    f32 = torch.float32
    _dense(stats, (T, 2), f32, dev, "stats")
    if (target is None) != (dlogp is None):
        raise ValueError("target and dlogp go together")
    if target is not None:
        _dense(target, (T,), torch.int64, dev, "target")
        _dense(dlogp, (T,), f32, dev, "dlogp")
    if dentropy is not None:
        if entropy is None:
            raise ValueError("dentropy needs the entropy")
        _dense(entropy, (T,), f32, dev, "entropy")
        _dense(dentropy, (T,), f32, dev, "dentropy")
    k = 0
    if dtop is not None:
        if dtop.dim() != 2 or top_index is None:
            raise ValueError("dtop must have the shape [n_tok, k], beside top_index")
        k = dtop.shape[1]
        _dense(dtop, (T, k), f32, dev, "dtop")
        _dense(top_index, (T, k), torch.int64, dev, "top_index")
        if k == 0:
            dtop = None
    with _on(Z):
        if out is None:
            with _alloc_scope(stream):
                out = Z.new_empty((T, V))
        elif out.dtype != Z.dtype or out.shape != Z.shape or out.get_device() != dev:
            raise ValueError("out must be a [n_tok, vocab] tensor of Z's dtype and device")
        lddz = _logits(out, "out")[2]
        if out.data_ptr() == Z.data_ptr() and lddz != ldz and T > 1:
            raise ValueError("out may be Z itself, not another view of it")
        _check(lib.thanos_token_logprobs_backward(
            out.data_ptr(), lddz, Z.data_ptr(), ldz, dt, stats.data_ptr(), _ptr(target),
            _ptr(dlogp), _ptr(entropy), _ptr(dentropy), _ptr(top_index) if k else None, _ptr(dtop),
            T, V, k, _stream_ptr(stream)), "thanos_token_logprobs_backward")
    return out
