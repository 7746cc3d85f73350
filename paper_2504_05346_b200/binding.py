"""ctypes binding of libthanos.so: same names as the C ABI, argument marshalling only."""

from __future__ import annotations

import contextlib
import ctypes
import functools
import os
import sys
from dataclasses import dataclass
from typing import NamedTuple, Optional, Tuple, Union

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))

F32, BF16 = 0, 1
UNSTRUCTURED, NM = 0, 1
WS_HESSIAN, WS_PREPARE, WS_PRUNE, WS_HOST_LAYER, WS_PRUNE_OUTLIERS = 0, 1, 2, 3, 4


class ThanosError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        super().__init__("%s failed: %s (status %d)" % (where, status_string(code), code))


class _Stats(ctypes.Structure):
    _fields_ = [
        ("status", ctypes.c_int32),
        ("err_index", ctypes.c_int32),
        ("n_pruned", ctypes.c_int64),
        ("r_left", ctypes.c_int64),
        ("max_s", ctypes.c_int32),
        ("n_blocks", ctypes.c_int32),
        ("n_tied", ctypes.c_int64),
        ("last_threshold_bits", ctypes.c_uint32),
        ("select_misses", ctypes.c_int32),
        ("select_rescans", ctypes.c_int32),
        ("reserved", ctypes.c_int32 * 3),
    ]


assert ctypes.sizeof(_Stats) == 64


@dataclass
class PruneStats:
    status: int
    err_index: int
    n_pruned: int
    r_left: int
    max_s: int
    n_blocks: int
    n_tied: int
    last_threshold_bits: int
    select_misses: int = 0
    select_rescans: int = 0

    @staticmethod
    def from_bytes(raw: bytes) -> "PruneStats":
        s = _Stats.from_buffer_copy(raw)
        return PruneStats(s.status, s.err_index, s.n_pruned, s.r_left, s.max_s, s.n_blocks,
                          s.n_tied, s.last_threshold_bits, s.select_misses, s.select_rescans)


_lib = None
_calls = None     # the short way to the calls below (csrc/calls.cpp), once the library is loaded
_NO_SCOPE = contextlib.nullcontext()


def lib_path() -> str:
    return os.path.join(_HERE, "libthanos.so")


def load_library():
    """Load libthanos.so.  There is no fallback: a missing library is an error."""
    global _lib
    if _lib is not None:
        return _lib
    path = lib_path()
    if not os.path.exists(path):
        raise FileNotFoundError(
            "%s is missing: build it with `python -m paper_2504_05346_b200.build` "
            "(there is no CPU or PyTorch fallback)" % path)
    lib = ctypes.CDLL(path)
    vp, i64, i32, sz = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int32, ctypes.c_size_t
    lib.thanos_hessian_accumulate.argtypes = [vp, i64, vp, i32, i64, i64, vp, sz, vp]
    lib.thanos_hessian_accumulate.restype = i32
    lib.thanos_hessian_accumulate_ordered.argtypes = [vp, i64, vp, i32, i64, i64, vp, sz, vp]
    lib.thanos_hessian_accumulate_ordered.restype = i32
    lib.thanos_prepare_inverse.argtypes = [vp, i64, ctypes.c_float, vp, vp, vp, sz, vp, vp]
    lib.thanos_prepare_inverse.restype = i32
    lib.thanos_prune_layer.argtypes = [vp, vp, vp, i32, i64, i64, vp, vp, i32, ctypes.c_double,
                                       i32, i32, i32, vp, sz, vp, vp]
    lib.thanos_prune_layer.restype = i32
    lib.thanos_prune_layer_outliers.argtypes = [vp, vp, vp, i32, i64, i64, vp, vp, vp, i32, i32, i32,
                                                ctypes.c_double, vp, vp, sz, vp, vp]
    lib.thanos_prune_layer_outliers.restype = i32
    lib.thanos_prune_layer_structured.argtypes = [vp, vp, vp, vp, i32, i64, i64, vp, vp, vp,
                                                  ctypes.c_double, ctypes.c_double, vp, sz, vp, vp]
    lib.thanos_prune_layer_structured.restype = i32
    lib.thanos_structured_workspace_bytes.argtypes = [i64, i64, ctypes.c_double, ctypes.c_double,
                                                      i32]
    lib.thanos_structured_workspace_bytes.restype = sz
    lib.thanos_prune_block.argtypes = [vp, vp, i64, i64, vp, vp, i32, i32, i32, i32, i64, vp, vp,
                                       sz, vp, vp]
    lib.thanos_prune_block.restype = i32
    lib.thanos_prune_layer_host.argtypes = [vp, vp, vp, vp, i32, i64, i64, i64, ctypes.c_float,
                                            i32, ctypes.c_double, i32, i32, i32, i32, vp, sz,
                                            ctypes.POINTER(_Stats), vp]
    lib.thanos_prune_layer_host.restype = i32
    lib.thanos_prune_layer_noalloc.argtypes = [vp, vp, vp, i32, i64, i64, vp, vp, i32,
                                               ctypes.c_double, i32, i32, i32, vp, vp]
    lib.thanos_prune_layer_noalloc.restype = i32
    lib.thanos_dense_product.argtypes = [vp, i64, vp, i64, vp, i64, i32, i64, i64, i64,
                                         ctypes.c_float, i32, vp, sz, vp]
    lib.thanos_dense_product.restype = i32
    lib.thanos_dense_product_workspace.argtypes = [i64, i64, i64]
    lib.thanos_dense_product_workspace.restype = sz
    f32 = ctypes.c_float
    lib.thanos_adapter_forward.argtypes = [vp, i64, vp, vp, i64, vp, i64, vp, vp, vp, vp, i32, i64,
                                           i64, i64, i64, i32, vp, sz, vp]
    lib.thanos_adapter_forward.restype = i32
    lib.thanos_adapter_backward.argtypes = [vp, i64, vp, vp, i32, vp, i64, vp, i64, vp, vp, i64, vp,
                                            vp, vp, vp, i32, i64, i64, i64, i64, i32, vp, sz, vp]
    lib.thanos_adapter_backward.restype = i32
    lib.thanos_adapter_workspace_bytes.argtypes = [i32, i64, i64, i64, i64, i32, i32]
    lib.thanos_adapter_workspace_bytes.restype = sz
    lib.thanos_adapter_forward_packed.argtypes = [vp, i64, vp, vp, i64, vp, i64, vp, i32, vp, vp, vp,
                                                  vp, i32, i64, i64, i64, i64, i32, vp, sz, vp]
    lib.thanos_adapter_forward_packed.restype = i32
    lib.thanos_adapter_backward_packed.argtypes = [vp, i64, vp, vp, i32, vp, i64, vp, i64, vp, i64, vp,
                                                   vp, i64, vp, i32, vp, vp, vp, vp, i32, i64, i64, i64,
                                                   i64, i32, vp, sz, vp]
    lib.thanos_adapter_backward_packed.restype = i32
    lib.thanos_adapter_packed_workspace_bytes.argtypes = [i32, i32, i32, i64, i64, i64, i64, i32, i32]
    lib.thanos_adapter_packed_workspace_bytes.restype = sz
    lib.thanos_pack_weights.argtypes = [vp, i64, vp, vp, i64, i32, i64, i64, i32, vp]
    lib.thanos_pack_weights.restype = i32
    lib.thanos_unpack_weights.argtypes = [vp, i64, i32, vp, i64, vp, i64, i64, i32, vp]
    lib.thanos_unpack_weights.restype = i32
    lib.thanos_pack_activations.argtypes = [vp, i64, vp, i64, vp, i64, i32, i64, i64, vp]
    lib.thanos_pack_activations.restype = i32
    lib.thanos_unpack_activations.argtypes = [vp, i64, i32, vp, i64, vp, i64, i64, i64, vp]
    lib.thanos_unpack_activations.restype = i32
    lib.thanos_orthogonalise.argtypes = [vp, vp, i32, i64, i64, i64, vp, i32, f32, vp, sz, vp]
    lib.thanos_orthogonalise.restype = i32
    lib.thanos_orthogonal_step.argtypes = [vp, vp, i32, vp, vp, vp, i32, vp, i64, i64, i64, f32, f32,
                                           f32, i32, f32, vp, i32, f32, vp, sz, vp]
    lib.thanos_orthogonal_step.restype = i32
    lib.thanos_orthogonal_workspace_bytes.argtypes = [i64, i64, i64]
    lib.thanos_orthogonal_workspace_bytes.restype = sz
    lib.thanos_token_logprobs.argtypes = [vp, vp, vp, vp, vp, vp, i64, i32, vp, i64, i64, i32, vp]
    lib.thanos_token_logprobs.restype = i32
    lib.thanos_token_logprobs_backward.argtypes = [vp, i64, vp, i64, i32, vp, vp, vp, vp, vp, vp, vp,
                                                   i64, i64, i32, vp]
    lib.thanos_token_logprobs_backward.restype = i32
    lib.thanos_fp32_fma_probe.argtypes = [vp, i64, i32, i32, ctypes.POINTER(ctypes.c_double), vp]
    lib.thanos_fp32_fma_probe.restype = i32
    lib.thanos_workspace_bytes.argtypes = [i32, i64, i64, i32, i32]
    lib.thanos_workspace_bytes.restype = sz
    lib.thanos_status_string.argtypes = [i32]
    lib.thanos_status_string.restype = ctypes.c_char_p
    lib.thanos_version.argtypes = []
    lib.thanos_version.restype = i32
    lib.thanos_launch_count.argtypes = []
    lib.thanos_launch_count.restype = i64
    _lib = lib
    _bind_calls(lib)
    return lib


def _bind_calls(lib):
    """Loads _calls.so beside the library.  It only makes calls shorter: without it, or with one that
    was built for another torch or Python, they go the long way."""
    global _calls
    try:
        from . import _calls as module
    except ImportError:
        return
    here = "torch %s, python %d.%d" % ((torch.__version__,) + sys.version_info[:2])
    if getattr(module, "built_for", None) != here:
        return
    names = ["thanos_" + n for n in (
        "token_logprobs", "token_logprobs_backward", "pack_weights", "unpack_weights",
        "pack_activations", "unpack_activations", "adapter_forward", "adapter_backward",
        "adapter_forward_packed", "adapter_backward_packed", "adapter_workspace_bytes",
        "adapter_packed_workspace_bytes")]
    module.bind(PackedWeights, PackedActivations,
                {n: ctypes.cast(getattr(lib, n), ctypes.c_void_p).value for n in names})
    _calls = module


def status_string(code: int) -> str:
    return load_library().thanos_status_string(int(code)).decode()


def version() -> int:
    return int(load_library().thanos_version())


def launch_count() -> int:
    return int(load_library().thanos_launch_count())


def workspace_bytes(which: int, c: int, b: int, B: int, dtype: int) -> int:
    return int(load_library().thanos_workspace_bytes(which, c, b, B, dtype))


def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.float32:
        return F32
    if t.dtype == torch.bfloat16:
        return BF16
    raise TypeError("unsupported dtype %s (float32 or bfloat16)" % t.dtype)


def _stream_ptr(stream) -> int:
    if stream is not None:
        return int(stream.cuda_stream)
    return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())


def _check_dev(*ts):
    for t in ts:
        if not t.is_cuda or not t.is_contiguous():
            raise ValueError("expected contiguous CUDA tensors")


def _ws(nbytes: int, device) -> torch.Tensor:
    return torch.empty(max(int(nbytes), 256), dtype=torch.uint8, device=device)


def _check(code: int, where: str):
    if code != 0:
        raise ThanosError(code, where)


def _on(t: torch.Tensor):
    """Makes the tensor's device current for the duration of a library call (kernels are
    launched on, and per-device state is looked up for, the current device)."""
    if t.get_device() == torch.cuda.current_device():
        return _NO_SCOPE
    return torch.cuda.device(t.device)


def hessian_status(workspace: torch.Tensor) -> int:
    """Device status word of the last thanos_hessian_accumulate call that used `workspace`
    (synchronises): 0, or THANOS_ERR_TIMEOUT (7) if a bounded wait inside the kernel ran out."""
    return int(workspace[:4].view(torch.int32).item())


def hessian_accumulate(H: torch.Tensor, X: torch.Tensor, stream=None,
                       workspace: Optional[torch.Tensor] = None, check: bool = False,
                       ordered: bool = False) -> None:
    """H += 2 X^T X for tokens-major X [n_tok, b] (float32 or bfloat16); H float32 [b, b].
    With check=True the call's device status word is read back (this waits for the call) and a
    non-zero status raises.  ordered=True calls thanos_hessian_accumulate_ordered (fixed
    summation order: bit-reproducible results)."""
    lib = load_library()
    if not X.is_cuda or X.stride(-1) != 1:
        raise ValueError("X must be a CUDA tensor with unit inner stride")
    _check_dev(H)
    b = H.shape[0]
    n_tok = X.shape[0]
    ldx = X.stride(0) if n_tok > 1 else b
    dt = _dtype_code(X)
    if workspace is None:
        workspace = _ws(workspace_bytes(WS_HESSIAN, 0, b, 0, dt), H.device)
    with _on(H):
        fn = lib.thanos_hessian_accumulate_ordered if ordered else lib.thanos_hessian_accumulate
        _check(fn(H.data_ptr(), b, X.data_ptr(), dt, n_tok, ldx, workspace.data_ptr(),
                  workspace.numel(), _stream_ptr(stream)), "thanos_hessian_accumulate")
        if check and n_tok > 0:
            st = hessian_status(workspace)
            if st != 0:
                raise ThanosError(st, "thanos_hessian_accumulate (device)")


def prepare_inverse(H: torch.Tensor, damp_rel: float, stream=None,
                    workspace: Optional[torch.Tensor] = None, check: bool = True,
                    factor: Optional[torch.Tensor] = None,
                    xnorm: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, torch.Tensor]:
    """Returns (factor U [b, b] upper-triangular with U^T U = (H + damp I)^-1, xnorm [b]);
    pass `factor` / `xnorm` to have them written into existing buffers."""
    lib = load_library()
    _check_dev(H)
    b = H.shape[0]
    if factor is None:
        factor = torch.empty((b, b), dtype=torch.float32, device=H.device)
    if xnorm is None:
        xnorm = torch.empty((b,), dtype=torch.float32, device=H.device)
    _check_dev(factor, xnorm)
    status = torch.zeros(4, dtype=torch.int32, device=H.device)
    if workspace is None:
        workspace = _ws(workspace_bytes(WS_PREPARE, 0, b, 0, F32), H.device)
    with _on(H):
        _check(lib.thanos_prepare_inverse(H.data_ptr(), b, float(damp_rel), factor.data_ptr(),
                                          xnorm.data_ptr(), workspace.data_ptr(),
                                          workspace.numel(), status.data_ptr(),
                                          _stream_ptr(stream)), "thanos_prepare_inverse")
    if check:
        st = status.cpu()
        if int(st[0]) != 0:
            raise ThanosError(int(st[0]), "thanos_prepare_inverse (column %d)" % int(st[1]))
    return factor, xnorm


def _read_stats(stats_dev: torch.Tensor) -> PruneStats:
    return PruneStats.from_bytes(bytes(stats_dev.cpu().numpy().tobytes()))


def prune_layer(W: torch.Tensor, factor: torch.Tensor, xnorm: torch.Tensor, mode: int,
                p: float = 0.0, n: int = 0, m: int = 0, B: int = 128, stream=None,
                workspace: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None,
                mask: Optional[torch.Tensor] = None, read_stats: bool = True):
    """Block sweep over one layer.  Returns (W_pruned, mask uint8, PruneStats | stats tensor)."""
    lib = load_library()
    _check_dev(W, factor, xnorm)
    c, b = W.shape
    dt = _dtype_code(W)
    if out is None:
        out = torch.empty_like(W)
    if mask is None:
        mask = torch.empty((c, b), dtype=torch.uint8, device=W.device)
    stats = torch.zeros(64, dtype=torch.uint8, device=W.device)
    if workspace is None:
        workspace = _ws(workspace_bytes(WS_PRUNE, c, b, B, dt), W.device)
    with _on(W):
        _check(lib.thanos_prune_layer(W.data_ptr(), out.data_ptr(), mask.data_ptr(), dt, c, b,
                                      factor.data_ptr(), xnorm.data_ptr(), mode, float(p), n, m, B,
                                      workspace.data_ptr(), workspace.numel(), stats.data_ptr(),
                                      _stream_ptr(stream)), "thanos_prune_layer")
    if not read_stats:
        return out, mask, stats
    st = _read_stats(stats)
    if st.status != 0:
        raise ThanosError(st.status, "thanos_prune_layer (row %d)" % st.err_index)
    return out, mask, st


def prune_block(Wc: torch.Tensor, mask: torch.Tensor, factor: torch.Tensor, xnorm: torch.Tensor,
                mode: int, n: int, m: int, B: int, j1: int, r: Optional[torch.Tensor],
                stats: torch.Tensor, stream=None, workspace: Optional[torch.Tensor] = None):
    """One block step in place on the float32 working weights Wc (and r, a 1-element int64)."""
    lib = load_library()
    _check_dev(Wc, mask, factor, xnorm)
    c, b = Wc.shape
    if workspace is None:
        workspace = _ws(workspace_bytes(WS_PRUNE, c, b, B, F32), Wc.device)
    with _on(Wc):
        _check(lib.thanos_prune_block(Wc.data_ptr(), mask.data_ptr(), c, b, factor.data_ptr(),
                                      xnorm.data_ptr(), mode, n, m, B, j1,
                                      r.data_ptr() if r is not None else None,
                                      workspace.data_ptr(), workspace.numel(), stats.data_ptr(),
                                      _stream_ptr(stream)), "thanos_prune_block")


def prune_layer_host(W_host: torch.Tensor, X_host: Optional[torch.Tensor], damp_rel: float,
                     mode: int, p: float = 0.0, n: int = 0, m: int = 0, B: int = 128,
                     arena: Optional[torch.Tensor] = None, reuse_factor: bool = False,
                     out: Optional[torch.Tensor] = None, mask: Optional[torch.Tensor] = None,
                     a: Optional[int] = None, stream=None, device="cuda"):
    """Whole path for one layer from HOST tensors (pinned or pageable); returns host tensors."""
    lib = load_library()
    if W_host.is_cuda or (X_host is not None and X_host.is_cuda):
        raise ValueError("prune_layer_host takes host tensors")
    c, b = W_host.shape
    dt = _dtype_code(W_host)
    if X_host is not None:
        if _dtype_code(X_host) != dt or not X_host.is_contiguous():
            raise ValueError("X must be contiguous and share W's dtype")
        a = X_host.shape[0]
    if a is None:
        a = 0
    if out is None:
        out = torch.empty_like(W_host)
    if mask is None:
        mask = torch.empty((c, b), dtype=torch.uint8)
    if arena is None:
        arena = _ws(workspace_bytes(WS_HOST_LAYER, c, b, B, dt), device)
    stats = _Stats()
    with _on(arena):
        code = lib.thanos_prune_layer_host(W_host.data_ptr(),
                                           X_host.data_ptr() if X_host is not None else None,
                                           out.data_ptr(), mask.data_ptr(), dt, c, b, a,
                                           float(damp_rel), mode, float(p), n, m, B,
                                           1 if reuse_factor else 0, arena.data_ptr(),
                                           arena.numel(), ctypes.byref(stats),
                                           _stream_ptr(stream))
    _check(code, "thanos_prune_layer_host")
    st = PruneStats(stats.status, stats.err_index, stats.n_pruned, stats.r_left, stats.max_s,
                    stats.n_blocks, stats.n_tied, stats.last_threshold_bits, stats.select_misses,
                    stats.select_rescans)
    if st.status != 0:
        raise ThanosError(st.status, "thanos_prune_layer_host (index %d)" % st.err_index)
    return out, mask, st


def prune_layer_noalloc(W: torch.Tensor, factor: torch.Tensor, xnorm: torch.Tensor, mode: int,
                        p: float = 0.0, n: int = 0, m: int = 0, B: int = 128, stream=None,
                        out: Optional[torch.Tensor] = None, mask: Optional[torch.Tensor] = None,
                        stats: Optional[torch.Tensor] = None):
    """thanos_prune_layer_noalloc: the sweep with the library's built-in 4 MiB scratch, for
    callers that cannot allocate a workspace.  Only the outputs are created here; pass `out`,
    `mask` and `stats` (64 bytes, uint8) and this function creates no device tensor at all.
    Calls on one device must not overlap."""
    lib = load_library()
    _check_dev(W, factor, xnorm)
    c, b = W.shape
    dt = _dtype_code(W)
    if out is None:
        out = torch.empty_like(W)
    if mask is None:
        mask = torch.empty((c, b), dtype=torch.uint8, device=W.device)
    if stats is None:
        stats = torch.zeros(64, dtype=torch.uint8, device=W.device)
    with _on(W):
        _check(lib.thanos_prune_layer_noalloc(W.data_ptr(), out.data_ptr(), mask.data_ptr(), dt, c,
                                              b, factor.data_ptr(), xnorm.data_ptr(), mode,
                                              float(p), n, m, B, stats.data_ptr(),
                                              _stream_ptr(stream)), "thanos_prune_layer_noalloc")
    st = _read_stats(stats)
    if st.status != 0:
        raise ThanosError(st.status, "thanos_prune_layer_noalloc (row %d)" % st.err_index)
    return out, mask, st


def fp32_fma_probe(out: torch.Tensor, ctas: int, iters: int, stream=None) -> float:
    """thanos_fp32_fma_probe: enqueues the FMA-chain kernel; returns its floating-point
    operation count (time it with CUDA events around this call)."""
    lib = load_library()
    _check_dev(out)
    flop = ctypes.c_double(0.0)
    with _on(out):
        _check(lib.thanos_fp32_fma_probe(out.data_ptr(), out.numel(), ctas, iters,
                                         ctypes.byref(flop), _stream_ptr(stream)),
               "thanos_fp32_fma_probe")
    return float(flop.value)


def dense_product(A: torch.Tensor, B: torch.Tensor, b_transposed: bool = False, alpha: float = 1.0,
                  out: Optional[torch.Tensor] = None, accumulate: bool = False, stream=None,
                  check: bool = True):
    """thanos_dense_product: out = (accumulate ? out : 0) + alpha * A @ (B^T if b_transposed
    else B), fp32 device matrices (rows may be strided: the last dimension is contiguous)."""
    lib = load_library()
    _check_dev(A, B)
    assert A.dtype == torch.float32 and B.dtype == torch.float32
    assert A.stride(1) == 1 and B.stride(1) == 1
    M, K = A.shape
    N = B.shape[0] if b_transposed else B.shape[1]
    assert (B.shape[1] if b_transposed else B.shape[0]) == K
    if out is None:
        out = torch.empty((M, N), dtype=torch.float32, device=A.device)
        assert not accumulate
    assert out.stride(1) == 1
    nbytes = lib.thanos_dense_product_workspace(M, N, K)
    ws = torch.empty(max(nbytes, 256), dtype=torch.uint8, device=A.device)
    with _on(A):
        _check(lib.thanos_dense_product(out.data_ptr(), out.stride(0), A.data_ptr(), A.stride(0),
                                        B.data_ptr(), B.stride(0), 1 if b_transposed else 0, M, N, K,
                                        float(alpha), 1 if accumulate else 0, ws.data_ptr(), nbytes,
                                        _stream_ptr(stream)), "thanos_dense_product")
    if check:
        st = int(ws[:4].view(torch.int32).item())
        if st != 0:
            raise ThanosError(st, "thanos_dense_product (device)")
    return out


def prune_layer_outliers(W: torch.Tensor, factor: torch.Tensor, xnorm: torch.Tensor,
                         H: torch.Tensor, n: int, m: int, alpha: float, B: int = 128, stream=None,
                         workspace: Optional[torch.Tensor] = None,
                         out: Optional[torch.Tensor] = None, mask: Optional[torch.Tensor] = None):
    """thanos_prune_layer_outliers: n:m sweep that leaves the ceil(alpha c) rows with the largest
    h_i = 1/2 W_i H W_i^T untouched.  Returns (W_pruned, mask, outlier flags uint8 [c], stats)."""
    lib = load_library()
    _check_dev(W, factor, xnorm, H)
    c, b = W.shape
    dt = _dtype_code(W)
    if out is None:
        out = torch.empty_like(W)
    if mask is None:
        mask = torch.empty((c, b), dtype=torch.uint8, device=W.device)
    flags = torch.empty((c,), dtype=torch.uint8, device=W.device)
    stats = torch.zeros(64, dtype=torch.uint8, device=W.device)
    if workspace is None:
        workspace = _ws(workspace_bytes(WS_PRUNE_OUTLIERS, c, b, B, dt), W.device)
    with _on(W):
        _check(lib.thanos_prune_layer_outliers(W.data_ptr(), out.data_ptr(), mask.data_ptr(), dt, c, b,
                                               factor.data_ptr(), xnorm.data_ptr(), H.data_ptr(), n, m,
                                               B, float(alpha), flags.data_ptr(), workspace.data_ptr(),
                                               workspace.numel(), stats.data_ptr(),
                                               _stream_ptr(stream)), "thanos_prune_layer_outliers")
    st = _read_stats(stats)
    if st.status != 0:
        raise ThanosError(st.status, "thanos_prune_layer_outliers (row %d)" % st.err_index)
    return out, mask, flags, st


def prune_layer_structured(W: torch.Tensor, factor: torch.Tensor, xnorm: torch.Tensor, p: float,
                           alpha: float = 0.0, H: Optional[torch.Tensor] = None, stream=None,
                           workspace: Optional[torch.Tensor] = None,
                           out: Optional[torch.Tensor] = None):
    """thanos_prune_layer_structured: removes the ceil(p b / (1 - alpha)) columns of smallest loss
    from all but the ceil(alpha c) outlier rows and updates the kept weights (Algorithm 2).
    Returns (W_pruned, removed columns uint8 [b], outlier rows uint8 [c], stats)."""
    lib = load_library()
    _check_dev(W, factor, xnorm)
    if alpha > 0.0:
        if H is None:
            raise ValueError("alpha > 0 needs the Hessian H")
        _check_dev(H)
    c, b = W.shape
    dt = _dtype_code(W)
    if out is None:
        out = torch.empty_like(W)
    colrm = torch.empty((b,), dtype=torch.uint8, device=W.device)
    flags = torch.empty((c,), dtype=torch.uint8, device=W.device)
    stats = torch.zeros(64, dtype=torch.uint8, device=W.device)
    if workspace is None:
        need = int(lib.thanos_structured_workspace_bytes(c, b, float(p), float(alpha), dt))
        if need == 0:
            raise ThanosError(1, "thanos_structured_workspace_bytes rejected the arguments")
        workspace = _ws(need, W.device)
    with _on(W):
        _check(lib.thanos_prune_layer_structured(W.data_ptr(), out.data_ptr(), colrm.data_ptr(),
                                                 flags.data_ptr(), dt, c, b, factor.data_ptr(),
                                                 xnorm.data_ptr(),
                                                 H.data_ptr() if H is not None else None, float(p),
                                                 float(alpha), workspace.data_ptr(), workspace.numel(),
                                                 stats.data_ptr(), _stream_ptr(stream)),
               "thanos_prune_layer_structured")
    st = _read_stats(stats)
    if st.status != 0:
        raise ThanosError(st.status, "thanos_prune_layer_structured (index %d)" % st.err_index)
    return out, colrm, flags, st


# ------------------------------------------------------------------ recovery of a pruned layer
def _alloc_scope(stream):
    """Buffers made for a call on another stream come from that stream's pool: the caching
    allocator then neither hands out memory that the current stream still uses nor takes it back
    before the call is done."""
    return _NO_SCOPE if stream is None else torch.cuda.stream(stream)


# The checks below run in front of calls that take a dozen microseconds on the device, so they ask
# each tensor for as little as they can.
def _rows(t: torch.Tensor, cols: int, device: int, name: str) -> int:
    """Leading dimension of a matrix on `device` with `cols` columns and unit inner stride."""
    if t.get_device() != device or t.dim() != 2 or t.shape[1] != cols:
        raise ValueError("%s must be a matrix of %d columns on CUDA device %d" % (name, cols, device))
    ld, inner = t.stride()
    if inner != 1 and cols > 1:
        raise ValueError("%s must have unit inner stride" % name)
    return ld if t.shape[0] > 1 else (cols + 7) // 8 * 8   # one row: its stride is never used


def _dense(t: torch.Tensor, shape, dtype, device: int, name: str) -> None:
    if (t.get_device() != device or t.dtype != dtype or t.shape != shape
            or not t.is_contiguous()):
        raise ValueError("%s must be a contiguous %s tensor of shape %s on CUDA device %d"
                         % (name, dtype, tuple(shape), device))


def _device_of(t: torch.Tensor, name: str) -> int:
    if not t.is_cuda:
        raise ValueError("%s must be a CUDA tensor" % name)
    return t.get_device()


class PackedWeights(NamedTuple):
    """Weights [c, cols] in 4 bits, from pack_weights: codes uint8 [c, ldq] (two a byte, the even
    column in the low half, each as code + 8; rows of whole 64-column blocks), scales bfloat16
    [ceil(cols / group), c] of five significant bits.  Takes the place of W."""

    codes: torch.Tensor
    scales: torch.Tensor
    group: int
    cols: int


class PackedActivations(NamedTuple):
    """Activations in 8 bits, from pack_activations: codes int8 [n_tok, b] (leading dimension a
    multiple of 16), exps uint8 [n_tok, ceil(b / 32)] (leading dimension a multiple of 4):
    x = code 2^(e - 127).  Takes the place of X in adapter_backward."""

    codes: torch.Tensor
    exps: torch.Tensor


def _packed_weights(W: PackedWeights, dev: int):
    """Checked (c, b, ldq) of packed weights."""
    codes, scales, group, b = W
    if codes.get_device() != dev or codes.dtype != torch.uint8 or codes.dim() != 2:
        raise ValueError("the weights' codes must be a uint8 matrix on CUDA device %d" % dev)
    (c, wide), (ldq, inner) = codes.shape, codes.stride()
    if inner != 1 or wide < -(-b // 64) * 32:
        raise ValueError("the weights' codes must have unit inner stride and whole 64-column blocks")
    if group not in (64, 128):
        raise ValueError("the weights' group must be 64 or 128")
    _dense(scales, (-(-b // group), c), torch.bfloat16, dev, "the weights' scales")
    return c, b, ldq if c > 1 else -(-wide // 16) * 16


def _packed_activations(X: PackedActivations, b: int, dev: int):
    """Checked (T, ldc, lde) of packed activations."""
    codes, exps = X
    if codes.dtype != torch.int8 or exps.dtype != torch.uint8 or exps.dim() != 2 \
            or exps.shape[0] != codes.shape[0]:
        raise ValueError("packed activations are int8 codes [n_tok, b] and uint8 exps [n_tok, b / 32]")
    ldc = _rows(codes, b, dev, "the activations' codes")
    lde = _rows(exps, -(-b // 32), dev, "the activations' exps")
    if codes.shape[0] <= 1:       # one row: its strides are never used
        ldc, lde = -(-b // 16) * 16, -(-lde // 4) * 4
    return codes.shape[0], ldc, lde


def _adapters(X, W, A, B, index, scale, dev):
    """Checked sizes (T, c, b, n, r), W's leading dimension and dtype code of an adapted projection."""
    dtype = X.dtype
    dt = _dtype_code(X)
    if type(W) is PackedWeights:
        c, b, ldw = _packed_weights(W, dev)
    else:
        if W.dim() != 2 or W.dtype != dtype:
            raise ValueError("W must be a matrix of X's dtype")
        c, b = W.shape
        ldw = _rows(W, b, dev, "W")
    T = X.shape[0]
    if A is None:
        if not (B is None and index is None and scale is None):
            raise ValueError("without A there is no B, index or scale either")
        return T, c, b, 0, 0, ldw, dt
    if A.dim() != 3:
        raise ValueError("A must have the shape [n_adapters, r, b]")
    n, r, _ = A.shape
    _dense(A, (n, r, b), dtype, dev, "A")
    _dense(B, (n, c, r), dtype, dev, "B")
    _dense(index, (T,), torch.int32, dev, "index")
    _dense(scale, (n,), torch.float32, dev, "scale")
    return T, c, b, n, r, ldw, dt


@functools.lru_cache(maxsize=256)
def _adapter_workspace(backward, T, c, b, n, r, dt):
    return max(int(load_library().thanos_adapter_workspace_bytes(backward, T, c, b, n, r, dt)), 256)


@functools.lru_cache(maxsize=256)
def _packed_workspace(backward, packed_w, packed_x, T, c, b, n, r, dt):
    return max(int(load_library().thanos_adapter_packed_workspace_bytes(
        backward, packed_w, packed_x, T, c, b, n, r, dt)), 256)


@functools.lru_cache(maxsize=256)
def _orthogonal_workspace(k, m, n):
    return max(int(load_library().thanos_orthogonal_workspace_bytes(k, m, n)), 256)


def _scratch(workspace: Optional[torch.Tensor], nbytes: int, like: torch.Tensor) -> torch.Tensor:
    """The caller's workspace, or a new one."""
    if workspace is None:
        return like.new_empty(nbytes, dtype=torch.uint8)
    if workspace.get_device() != like.get_device() or workspace.dtype != torch.uint8 \
            or not workspace.is_contiguous():
        raise ValueError("workspace must be a contiguous uint8 tensor on the call's device")
    return workspace


def _ptr(t):
    return None if t is None else t.data_ptr()


def _status(workspace: torch.Tensor, where: str, stream) -> None:
    with _alloc_scope(stream):   # behind the call, on the stream that it runs on
        st = int(workspace[:4].view(torch.int32).item())
    if st != 0:
        raise ThanosError(st, where + " (device)")


def adapter_forward(X: torch.Tensor, W: Union[torch.Tensor, PackedWeights], A: Optional[torch.Tensor] = None,
                    B: Optional[torch.Tensor] = None, index: Optional[torch.Tensor] = None,
                    scale: Optional[torch.Tensor] = None, stream=None,
                    workspace: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None,
                    V: Optional[torch.Tensor] = None, check: bool = False):
    """thanos_adapter_forward: Y[t] = X[t] W^T + scale[i] (X[t] A[i]^T) B[i]^T with i = index[t],
    -1 for a token without adapter.  X [T, b], W [c, b], A [n, r, b], B [n, c, r] share a dtype
    (float32 or bfloat16); index int32 [T], scale float32 [n].  Returns (Y, V): V float32 [T, r]
    holds X[t] A[i]^T for adapter_backward (None without adapters).  W may be PackedWeights
    (thanos_adapter_forward_packed).  With check=True the call's device status word is read back (this
    waits for the call)."""
    lib = _lib or load_library()
    if _calls is not None and stream is workspace is out is V is None and not check:
        done = _calls.adapter_forward(X, W, A, B, index, scale)
        if done is not None:
            return done
    dev = _device_of(X, "X")
    T, c, b, n, r, ldw, dt = _adapters(X, W, A, B, index, scale, dev)
    packed = type(W) is PackedWeights
    ldx = _rows(X, b, dev, "X")
    with _on(X):
        with _alloc_scope(stream):
            if out is None:
                out = X.new_empty((T, c))
            elif out.dtype != X.dtype or out.shape[0] != T:
                raise ValueError("out must be a [T, c] tensor of X's dtype")
            if n > 0:
                if V is None:
                    V = scale.new_empty((T, r))
                else:
                    _dense(V, (T, r), torch.float32, dev, "V")
            else:
                V = None     # a buffer that was passed in is not written
            workspace = _scratch(workspace, _packed_workspace(0, 1, 0, T, c, b, n, r, dt) if packed
                                 else _adapter_workspace(0, T, c, b, n, r, dt), X)
        ldy = _rows(out, c, dev, "out")
        if packed:
            _check(lib.thanos_adapter_forward_packed(
                out.data_ptr(), ldy, _ptr(V), X.data_ptr(), ldx, W.codes.data_ptr(), ldw,
                W.scales.data_ptr(), W.group, _ptr(A), _ptr(B), _ptr(index), _ptr(scale), dt, T, c, b,
                n, r, workspace.data_ptr(), workspace.numel(), _stream_ptr(stream)),
                "thanos_adapter_forward_packed")
        else:
            _check(lib.thanos_adapter_forward(out.data_ptr(), ldy, _ptr(V), X.data_ptr(), ldx,
                                              W.data_ptr(), ldw, _ptr(A), _ptr(B), _ptr(index),
                                              _ptr(scale), dt, T, c, b, n, r, workspace.data_ptr(),
                                              workspace.numel(), _stream_ptr(stream)),
                   "thanos_adapter_forward")
        if check:
            _status(workspace, "thanos_adapter_forward", stream)
    return out, V


def adapter_backward(dY: torch.Tensor, X: Union[torch.Tensor, PackedActivations, None],
                     V: Optional[torch.Tensor], W: Union[torch.Tensor, PackedWeights],
                     A: Optional[torch.Tensor] = None,
                     B: Optional[torch.Tensor] = None, index: Optional[torch.Tensor] = None,
                     scale: Optional[torch.Tensor] = None, need_dx: bool = True,
                     dA: Optional[torch.Tensor] = None, dB: Optional[torch.Tensor] = None,
                     accumulate: bool = False, need_grads: bool = True, stream=None,
                     workspace: Optional[torch.Tensor] = None, dX: Optional[torch.Tensor] = None,
                     check: bool = False):
    """thanos_adapter_backward: (dX, dA, dB) of adapter_forward for the output gradient dY [T, c].
    V is what adapter_forward returned.  dA, dB are float32, shaped like A and B; with
    accumulate=True they are added to (pass them in).  need_dx=False / need_grads=False leave a
    part out (None is returned for it; X and V may then be None without gradients).  X may be
    PackedActivations and W PackedWeights, one or both (thanos_adapter_backward_packed)."""
    lib = _lib or load_library()
    if _calls is not None and stream is workspace is dA is dB is dX is None and not (check or accumulate):
        done = _calls.adapter_backward(dY, X, V, W, A, B, index, scale, bool(need_dx),
                                       bool(need_grads))
        if done is not None:
            return done
    dev = _device_of(dY, "dY")
    T, c, b, n, r, ldw, dt = _adapters(dY, W, A, B, index, scale, dev)
    packed_w = type(W) is PackedWeights
    lddy = _rows(dY, c, dev, "dY")
    need_grads = need_grads and n > 0
    ldx = lde = 0
    packed_x = need_grads and type(X) is PackedActivations
    if need_grads:
        if X is None or V is None:
            raise ValueError("the adapters' gradients need X and V")
        if packed_x:
            rows, ldx, lde = _packed_activations(X, b, dev)
            if rows != T:
                raise ValueError("X must have n_tok rows")
            X, exps = X
        elif X.dtype != dY.dtype or X.shape[0] != T:
            raise ValueError("X must be a [T, b] tensor of dY's dtype")
        if not packed_x:
            ldx = _rows(X, b, dev, "X")
        _dense(V, (T, r), torch.float32, dev, "V")
        if accumulate and (dA is None or dB is None):
            raise ValueError("accumulate=True needs dA and dB")
    else:
        X = V = dA = dB = None
    with _on(dY):
        lddx = 0
        with _alloc_scope(stream):
            if not need_dx:
                dX = None
            elif dX is None:
                dX = dY.new_empty((T, b))
            elif dX.dtype != dY.dtype or dX.shape[0] != T:
                raise ValueError("dX must be a [T, b] tensor of dY's dtype")
            if need_grads:
                if dA is None:
                    dA = scale.new_empty((n, r, b))
                else:
                    _dense(dA, (n, r, b), torch.float32, dev, "dA")
                if dB is None:
                    dB = scale.new_empty((n, c, r))
                else:
                    _dense(dB, (n, c, r), torch.float32, dev, "dB")
            workspace = _scratch(workspace,
                                 _packed_workspace(1, int(packed_w and (need_dx or dt == F32)),
                                                   int(packed_x), T, c, b, n, r, dt)
                                 if packed_w or packed_x else _adapter_workspace(1, T, c, b, n, r, dt),
                                 dY)
        if need_dx:
            lddx = _rows(dX, b, dev, "dX")
        if packed_w or packed_x:
            _check(lib.thanos_adapter_backward_packed(
                _ptr(dX), lddx, _ptr(dA), _ptr(dB), 1 if accumulate else 0, dY.data_ptr(), lddy,
                _ptr(X), ldx, exps.data_ptr() if packed_x else None, lde, _ptr(V),
                W.codes.data_ptr() if packed_w else W.data_ptr(), ldw,
                W.scales.data_ptr() if packed_w else None, W.group if packed_w else 0, _ptr(A),
                _ptr(B), _ptr(index), _ptr(scale), dt, T, c, b, n, r, workspace.data_ptr(),
                workspace.numel(), _stream_ptr(stream)), "thanos_adapter_backward_packed")
        else:
            _check(lib.thanos_adapter_backward(
                _ptr(dX), lddx, _ptr(dA), _ptr(dB), 1 if accumulate else 0, dY.data_ptr(), lddy,
                _ptr(X), ldx, _ptr(V), W.data_ptr(), ldw, _ptr(A), _ptr(B), _ptr(index), _ptr(scale),
                dt, T, c, b, n, r, workspace.data_ptr(), workspace.numel(), _stream_ptr(stream)),
                "thanos_adapter_backward")
        if check:
            _status(workspace, "thanos_adapter_backward", stream)
    return dX, dA, dB


NEWTON_SCHULZ = (3.4445, -4.7750, 2.0315)  # quintic with a steep slope at zero, five steps


def _matrices(G: torch.Tensor):
    if G.dim() not in (2, 3) or not G.is_contiguous():
        raise ValueError("expected a contiguous matrix or batch of matrices")
    return (1 if G.dim() == 2 else G.shape[0]), G.shape[-2], G.shape[-1]


def orthogonalise(G: torch.Tensor, steps: int = 5, coef=NEWTON_SCHULZ, eps: float = 1e-7,
                  stream=None, workspace: Optional[torch.Tensor] = None,
                  out: Optional[torch.Tensor] = None, check: bool = False) -> torch.Tensor:
    """thanos_orthogonalise: Newton-Schulz iteration on G [m, n] or [batch, m, n] (float32 or
    bfloat16, contiguous); returns bfloat16 of the same shape."""
    lib = load_library()
    dev = _device_of(G, "G")
    k, m, n = _matrices(G)
    dt = _dtype_code(G)
    with _on(G):
        with _alloc_scope(stream):
            if out is None:
                out = torch.empty(G.shape, dtype=torch.bfloat16, device=G.device)
            else:
                _dense(out, G.shape, torch.bfloat16, dev, "out")
            workspace = _scratch(workspace, _orthogonal_workspace(k, m, n), G)
        abc = (ctypes.c_float * 3)(*coef)
        _check(lib.thanos_orthogonalise(out.data_ptr(), G.data_ptr(), dt, k, m, n, abc, steps,
                                        float(eps), workspace.data_ptr(), workspace.numel(),
                                        _stream_ptr(stream)), "thanos_orthogonalise")
        if check and k > 0:   # nothing runs for an empty batch, and nothing writes the word
            _status(workspace, "thanos_orthogonalise", stream)
    return out


def orthogonal_step(W: torch.Tensor, M: torch.Tensor, G: torch.Tensor,
                    mask: Optional[torch.Tensor] = None, lr: float = 2e-4, gain: float = 1.0,
                    momentum: float = 0.95, nesterov: bool = True, weight_decay: float = 0.0,
                    steps: int = 5, coef=NEWTON_SCHULZ, eps: float = 1e-7, stream=None,
                    workspace: Optional[torch.Tensor] = None, W_out: Optional[torch.Tensor] = None,
                    M_out: Optional[torch.Tensor] = None, check: bool = False):
    """thanos_orthogonal_step: momentum, orthogonalised update and new weights in one call; weights
    that `mask` (uint8, non-zero = removed) marks stay exact zeros and take no part.  W, G float32
    or bfloat16, M float32, all [m, n] or [batch, m, n] and contiguous.  Returns (W_out, M_out);
    pass W_out=W, M_out=M to update in place."""
    lib = load_library()
    dev = _device_of(G, "G")
    k, m, n = _matrices(G)
    wdt, gdt = _dtype_code(W), _dtype_code(G)
    _dense(W, G.shape, W.dtype, dev, "W")
    _dense(M, G.shape, torch.float32, dev, "M")
    if mask is not None:
        _dense(mask, G.shape, torch.uint8, dev, "mask")
    with _on(G):
        with _alloc_scope(stream):
            if W_out is None:
                W_out = torch.empty_like(W)
            else:
                _dense(W_out, G.shape, W.dtype, dev, "W_out")
            if M_out is None:
                M_out = torch.empty_like(M)
            else:
                _dense(M_out, G.shape, torch.float32, dev, "M_out")
            workspace = _scratch(workspace, _orthogonal_workspace(k, m, n), G)
        abc = (ctypes.c_float * 3)(*coef)
        _check(lib.thanos_orthogonal_step(W_out.data_ptr(), W.data_ptr(), wdt, M_out.data_ptr(),
                                          M.data_ptr(), G.data_ptr(), gdt, _ptr(mask), k, m, n,
                                          float(lr), float(gain), float(momentum),
                                          1 if nesterov else 0, float(weight_decay), abc, steps,
                                          float(eps), workspace.data_ptr(), workspace.numel(),
                                          _stream_ptr(stream)), "thanos_orthogonal_step")
        if check and k > 0:   # nothing runs for an empty batch, and nothing writes the word
            _status(workspace, "thanos_orthogonal_step", stream)
    return W_out, M_out
