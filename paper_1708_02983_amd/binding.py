"""Thin ctypes binding of libeasgd_hip.so: argument marshalling only.

Every function takes torch tensors that already live on the GPU, checks their
dtype / device / contiguity / size on the host, and passes raw device pointers
and the current HIP stream through the C ABI declared in ``include/easgd.h``.
All arithmetic of the round runs inside the library's kernels; there is no
fallback: if the shared library is missing, importing this module raises.
"""
from __future__ import annotations

import ctypes
import functools
import os
from typing import NamedTuple, Optional, Sequence

import torch

_PKG_DIR = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG_DIR, "libeasgd_hip.so")

EASGD_OK = 0
OPT_UPDATE_BLOCKS_PER_CU = 1
OPT_UPDATE_NONTEMPORAL = 2
OPT_UPDATE_GROUPS = 3
OPT_GEMM_TILE = 4
OPT_ROUND_OVERLAP = 5
OPT_GEMM_XCD = 6
OPT_GEMM_PAIR = 7
OPT_MLP_HEAD = 8
OPT_UPDATE_LAYOUT = 9
OPT_ROUND_SINGLE_LAUNCH = 10
OPT_ROUND_SPIN_LIMIT = 11


class EasgdError(RuntimeError):
    def __init__(self, code: int, message: str):
        super().__init__(f"easgd error {code}: {message}")
        self.code = code


def _load() -> ctypes.CDLL:
    if not os.path.exists(LIB_PATH):
        raise ImportError(
            f"{LIB_PATH} not found: build the HIP library first "
            "(python -m paper_1708_02983_amd.build); there is no CPU fallback")
    lib = ctypes.CDLL(LIB_PATH)
    vp, sz, f, i = ctypes.c_void_p, ctypes.c_size_t, ctypes.c_float, ctypes.c_int
    lib.easgd_sync_round.argtypes = [vp, vp, vp, i, sz, sz, f, f, vp]
    lib.easgd_sync_round.restype = i
    lib.measgd_round.argtypes = [vp, vp, vp, vp, i, sz, sz, f, f, f, vp]
    lib.measgd_round.restype = i
    lib.easgd_sync_round_bf16.argtypes = [vp, vp, vp, i, sz, sz, f, f, vp]
    lib.easgd_sync_round_bf16.restype = i
    lib.measgd_round_bf16.argtypes = [vp, vp, vp, vp, i, sz, sz, f, f, f, vp]
    lib.measgd_round_bf16.restype = i
    lib.measgd_round_bf16v.argtypes = [vp, vp, vp, vp, i, sz, sz, f, f, f, vp]
    lib.measgd_round_bf16v.restype = i
    lib.sync_sgd_round.argtypes = [vp, vp, vp, i, sz, sz, f, f, vp]
    lib.sync_sgd_round.restype = i
    lib.async_easgd_round.argtypes = [vp, vp, vp, vp, i, sz, sz, ctypes.POINTER(ctypes.c_int), i, f, f, f, vp]
    lib.async_easgd_round.restype = i
    lib.hogwild_easgd_round.argtypes = [vp, vp, vp, vp, i, sz, sz, f, f, f, vp]
    lib.hogwild_easgd_round.restype = i
    ip = ctypes.POINTER(ctypes.c_int)
    lib.easgd_grad_workspace_bytes.argtypes = [ip, i, i, i]
    lib.easgd_grad_workspace_bytes.restype = sz
    lib.easgd_grad.argtypes = [ip, i, vp, sz, vp, vp, i, i, vp, vp, vp, sz, vp]
    lib.easgd_grad.restype = i
    lib.easgd_grad_static.argtypes = [ip, i, vp, sz, vp, vp, i, i, vp, vp, vp]
    lib.easgd_grad_static.restype = i
    lib.easgd_grad_bf16.argtypes = [ip, i, vp, sz, vp, vp, i, i, vp, vp, vp, sz, vp]
    lib.easgd_grad_bf16.restype = i
    lib.easgd_mlp_round_workspace_bytes.argtypes = [ip, i, i, i]
    lib.easgd_mlp_round_workspace_bytes.restype = sz
    lib.easgd_mlp_round.argtypes = [ip, i, vp, vp, vp, sz, vp, vp, i, i, vp, vp, f, f, f, vp, sz, vp]
    lib.easgd_mlp_round.restype = i
    lib.easgd_mlp_round_bf16v.argtypes = [ip, i, vp, vp, vp, sz, vp, vp, i, i, vp, vp, f, f, f, vp, sz, vp]
    lib.easgd_mlp_round_bf16v.restype = i
    lib.easgd_layer_product.argtypes = [i, i, i, i, i, vp, vp, sz, vp, vp, sz, i, vp]
    lib.easgd_layer_product.restype = i
    lib.easgd_top_logits_workspace_bytes.argtypes = [sz, i, i]
    lib.easgd_top_logits_workspace_bytes.restype = sz
    lib.easgd_top_logits.argtypes = [vp, i, sz, i, sz, i, f, vp, vp, vp, vp, sz, vp]
    lib.easgd_top_logits.restype = i
    lib.easgd_distill_workspace_bytes.argtypes = [sz, i, i]
    lib.easgd_distill_workspace_bytes.restype = sz
    lib.easgd_distill_loss.argtypes = [vp, i, sz, i, sz, vp, vp, vp, i, vp, f, f, vp, vp, vp, sz, vp]
    lib.easgd_distill_loss.restype = i
    lib.easgd_distill_grad.argtypes = [vp, i, sz, i, sz, vp, vp, vp, i, vp, f, f, vp, vp, f, vp, sz, vp]
    lib.easgd_distill_grad.restype = i
    lib.easgd_distill.argtypes = [vp, i, sz, i, sz, vp, vp, vp, i, vp, f, f, f, vp, vp, sz, vp, sz, vp]
    lib.easgd_distill.restype = i
    lib.easgd_grad_distill.argtypes = [ip, i, vp, sz, vp, vp, vp, vp, i, vp, i, i, f, f, vp, vp, vp, sz, vp]
    lib.easgd_grad_distill.restype = i
    lib.easgd_score_tokens_workspace_bytes.argtypes = [sz, i, i]
    lib.easgd_score_tokens_workspace_bytes.restype = sz
    lib.easgd_score_tokens.argtypes = [vp, i, sz, i, sz, vp, f, vp, vp, vp, i, vp, vp, vp, vp, sz, vp]
    lib.easgd_score_tokens.restype = i
    lib.easgd_score_tokens_grad.argtypes = [vp, i, sz, i, sz, vp, f, vp, vp, vp, f, vp, sz, vp]
    lib.easgd_score_tokens_grad.restype = i
    lib.easgd_token_loss_workspace_bytes.argtypes = [sz, i]
    lib.easgd_token_loss_workspace_bytes.restype = sz
    lib.easgd_token_loss.argtypes = [vp, i, sz, i, sz, vp, vp, f, f, f, vp, vp, vp, vp, sz, vp, sz, vp]
    lib.easgd_token_loss.restype = i
    lib.easgd_grad_token_loss.argtypes = [ip, i, vp, sz, vp, vp, vp, i, i, f, f, vp, vp, vp, vp, vp, sz, vp]
    lib.easgd_grad_token_loss.restype = i
    lib.easgd_grad_norms_workspace_bytes.argtypes = [i, sz]
    lib.easgd_grad_norms_workspace_bytes.restype = sz
    lib.easgd_grad_norms.argtypes = [vp, i, i, sz, sz, f, vp, vp, vp, sz, vp]
    lib.easgd_grad_norms.restype = i
    i64 = ctypes.c_int64
    lib.adamw_round.argtypes = [vp, vp, vp, vp, i, vp, i, sz, sz, vp, vp, vp, i, vp, f, vp, f, f, f, f, f, i64, vp, vp]
    lib.adamw_round.restype = i
    lib.adamw_round_8bit.argtypes = [vp, vp, vp, vp, vp, vp, i, vp, i, sz, sz, vp, vp, vp, i, vp, f, vp, f, f, f, f, f, i64, vp, ctypes.c_uint32, vp]
    lib.adamw_round_8bit.restype = i
    lib.easgd_sample_tokens_workspace_bytes.argtypes = [sz, i]
    lib.easgd_sample_tokens_workspace_bytes.restype = sz
    lib.easgd_sample_tokens.argtypes = [vp, i, sz, i, sz, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.easgd_sample_tokens.restype = i
    lib.easgd_mlp_num_params.argtypes = [ip, i]
    lib.easgd_mlp_num_params.restype = sz
    lib.easgd_stream_copy.argtypes = [vp, vp, sz, vp]
    lib.easgd_stream_copy.restype = i
    lib.easgd_stream_triad.argtypes = [vp, vp, vp, sz, f, vp]
    lib.easgd_stream_triad.restype = i
    lib.easgd_stream_mix32.argtypes = [vp, vp, vp, vp, vp, sz, f, vp]
    lib.easgd_stream_mix32.restype = i
    lib.easgd_mfma_probe.argtypes = [vp, sz, i, i, i, vp, sz, ctypes.POINTER(ctypes.c_uint), vp]
    lib.easgd_mfma_probe.restype = i
    lib.easgd_round_barrier_timeouts.argtypes = [vp]
    lib.easgd_round_barrier_timeouts.restype = ctypes.c_long
    lib.easgd_launch_count.argtypes = []
    lib.easgd_launch_count.restype = ctypes.c_ulonglong
    lib.easgd_set_option.argtypes = [i, ctypes.c_long]
    lib.easgd_set_option.restype = i
    lib.easgd_get_option.argtypes = [i]
    lib.easgd_get_option.restype = ctypes.c_long
    lib.easgd_last_error.restype = ctypes.c_char_p
    lib.easgd_version.restype = i
    return lib


_lib = _load()


def lib() -> ctypes.CDLL:
    """The loaded C-ABI library (for callers that want the raw entry points)."""
    return _lib


def _check(code: int) -> None:
    if code != EASGD_OK:
        raise EasgdError(code, _lib.easgd_last_error().decode())


_raw_current_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream(stream) -> ctypes.c_void_p:
    # the current stream of the current device; torch.cuda.current_stream() builds a Stream object through several
    # layers of Python (8 us per call here, more than the library's own share of a small round), the raw query does not
    if stream is None:
        if _raw_current_stream is not None:
            return ctypes.c_void_p(_raw_current_stream(torch.cuda.current_device()))
        stream = torch.cuda.current_stream()
    device = getattr(stream, "device", None)
    if isinstance(device, torch.device) and device.index not in (None, torch.cuda.current_device()):
        raise ValueError(f"stream is on {device}, the current device is cuda:{torch.cuda.current_device()}")
    return ctypes.c_void_p(stream.cuda_stream)


def _stream_on(stream, device: int):
    """_stream for calls whose tensors are known to be on the current device, `device`."""
    if stream is None and _raw_current_stream is not None:
        return _raw_current_stream(device)
    return _stream(stream)


def _dev(name: str, t: torch.Tensor, dtype, min_numel: int) -> int:
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a CUDA/HIP tensor")
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if t.numel() < min_numel:
        raise ValueError(f"{name} holds {t.numel()} elements, needs {min_numel}")
    return t.data_ptr()


def _stream_object(stream):
    return stream if isinstance(stream, torch.cuda.Stream) else torch.cuda.ExternalStream(stream.cuda_stream)


def _new(shape, dtype, like, stream):
    """A tensor for a result or for scratch, from the memory of the stream that works on it first: what the current stream's
    memory holds free may still be in use by that stream's work, which another stream does not wait for.  The current
    stream, whose program gets the tensor, is noted as a user: the memory goes back to `stream` after its work, too."""
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=like.device)
    stream, caller = _stream_object(stream), torch.cuda.current_stream(like.device)
    with torch.cuda.stream(stream):
        t = torch.empty(shape, dtype=dtype, device=like.device)
    if stream != caller:
        t.record_stream(caller)
    return t


def _replica_shape(W: torch.Tensor, N: Optional[int]):
    if W.dim() != 2:
        raise ValueError("replica matrices must be [P][ld]")
    P, ld = W.shape
    return P, ld, (ld if N is None else int(N))


def easgd_sync_round(W, G, Wc, eta: float, rho: float, N: Optional[int] = None, stream=None) -> None:
    """Steps (2)-(5) of a Sync EASGD round, in place on W[P][ld] and Wc[N] (Eq. (1), Eq. (2))."""
    P, ld, N = _replica_shape(W, N)
    need = (P - 1) * ld + N
    _check(_lib.easgd_sync_round(_dev("W", W, torch.float32, need), _dev("G", G, torch.float32, need),
                                 _dev("Wc", Wc, torch.float32, N), P, N, ld, eta, rho, _stream(stream)))


def measgd_round(W, V, G, Wc, eta: float, rho: float, delta: float, N: Optional[int] = None,
                 stream=None) -> None:
    """The same round with the momentum worker rule, in place on W, V and Wc (Eq. (5), (6), (2))."""
    P, ld, N = _replica_shape(W, N)
    need = (P - 1) * ld + N
    _check(_lib.measgd_round(_dev("W", W, torch.float32, need), _dev("V", V, torch.float32, need),
                             _dev("G", G, torch.float32, need), _dev("Wc", Wc, torch.float32, N),
                             P, N, ld, eta, rho, delta, _stream(stream)))


def easgd_sync_round_bf16(W, G16, Wc, eta: float, rho: float, N: Optional[int] = None, stream=None) -> None:
    """easgd_sync_round with the gradients stored as bfloat16 (torch.bfloat16 tensor [P][ld]); an extension."""
    P, ld, N = _replica_shape(W, N)
    need = (P - 1) * ld + N
    _check(_lib.easgd_sync_round_bf16(_dev("W", W, torch.float32, need), _dev("G16", G16, torch.bfloat16, need),
                                      _dev("Wc", Wc, torch.float32, N), P, N, ld, eta, rho, _stream(stream)))


def measgd_round_bf16(W, V16, G16, Wc, eta: float, rho: float, delta: float, N: Optional[int] = None,
                      stream=None) -> None:
    """measgd_round with gradients and momentum buffers stored as bfloat16 (torch.bfloat16 tensors [P][ld]);
    an extension."""
    P, ld, N = _replica_shape(W, N)
    need = (P - 1) * ld + N
    _check(_lib.measgd_round_bf16(_dev("W", W, torch.float32, need), _dev("V16", V16, torch.bfloat16, need),
                                  _dev("G16", G16, torch.bfloat16, need), _dev("Wc", Wc, torch.float32, N),
                                  P, N, ld, eta, rho, delta, _stream(stream)))


def measgd_round_bf16v(W, V16, G, Wc, eta: float, rho: float, delta: float, N: Optional[int] = None,
                       stream=None) -> None:
    """measgd_round with only the momentum buffers stored as bfloat16; the gradients are fp32; an extension."""
    P, ld, N = _replica_shape(W, N)
    need = (P - 1) * ld + N
    _check(_lib.measgd_round_bf16v(_dev("W", W, torch.float32, need), _dev("V16", V16, torch.bfloat16, need),
                                   _dev("G", G, torch.float32, need), _dev("Wc", Wc, torch.float32, N),
                                   P, N, ld, eta, rho, delta, _stream(stream)))


def sync_sgd_round(W, G, eta: float, V=None, delta: float = 0.0, N: Optional[int] = None, stream=None) -> None:
    """Synchronous data-parallel SGD on the replicas: every replica moves by the sum of all gradients
    (Section 2.3, Section 6.2); V selects the momentum rule Eq. (3),(4)."""
    P, ld, N = _replica_shape(W, N)
    need = (P - 1) * ld + N
    _check(_lib.sync_sgd_round(_dev("W", W, torch.float32, need),
                               None if V is None else _dev("V", V, torch.float32, need),
                               _dev("G", G, torch.float32, need), P, N, ld, eta, delta, _stream(stream)))


def async_easgd_round(W, G, Wc, order: Sequence[int], eta: float, rho: float, V=None, delta: float = 0.0,
                      N: Optional[int] = None, stream=None) -> None:
    """The master serving one worker at a time in the sequence `order` (Algorithm 1 in rank order; Async EASGD /
    Async MEASGD in arrival order), one launch for the whole schedule; V selects Eq. (5),(6)."""
    P, ld, N = _replica_shape(W, N)
    need = (P - 1) * ld + N
    seq = (ctypes.c_int * len(order))(*[int(j) for j in order])
    _check(_lib.async_easgd_round(_dev("W", W, torch.float32, need),
                                  None if V is None else _dev("V", V, torch.float32, need),
                                  _dev("G", G, torch.float32, need), _dev("Wc", Wc, torch.float32, N),
                                  P, N, ld, seq, len(order), eta, rho, delta, _stream(stream)))


def hogwild_easgd_round(W, G, Wc, eta: float, rho: float, V=None, delta: float = 0.0, N: Optional[int] = None,
                        stream=None) -> None:
    """Hogwild EASGD: all workers exchange with the center at once, lock-free (atomic adds into the center);
    W and Wc are not reproducible from run to run."""
    P, ld, N = _replica_shape(W, N)
    need = (P - 1) * ld + N
    _check(_lib.hogwild_easgd_round(_dev("W", W, torch.float32, need),
                                    None if V is None else _dev("V", V, torch.float32, need),
                                    _dev("G", G, torch.float32, need), _dev("Wc", Wc, torch.float32, N),
                                    P, N, ld, eta, rho, delta, _stream(stream)))


# What the marshalling derives from the layer widths alone is kept per tuple of widths: a round of a small network
# takes some 15 us on the device, and rebuilding the C array and asking the library for N and the workspace size on
# every call cost more than that on the host.
@functools.lru_cache(maxsize=256)
def _dims_cached(dims: tuple):
    arr = (ctypes.c_int * len(dims))(*dims)
    return arr, len(dims) - 1


def _dims(dims: Sequence[int]):
    return _dims_cached(tuple(int(d) for d in dims))


@functools.lru_cache(maxsize=256)
def _num_params_cached(dims: tuple) -> int:
    arr, L = _dims_cached(dims)
    return int(_lib.easgd_mlp_num_params(arr, L))


def easgd_mlp_num_params(dims: Sequence[int]) -> int:
    return _num_params_cached(tuple(int(d) for d in dims))


@functools.lru_cache(maxsize=256)
def _workspace_cached(dims: tuple, P: int, b: int, whole_round: bool) -> int:
    arr, L = _dims_cached(dims)
    fn = _lib.easgd_mlp_round_workspace_bytes if whole_round else _lib.easgd_grad_workspace_bytes
    return int(fn(arr, L, P, b))


def easgd_grad_workspace_bytes(dims: Sequence[int], P: int, b: int) -> int:
    return _workspace_cached(tuple(int(d) for d in dims), int(P), int(b), False)


def easgd_grad(dims: Sequence[int], W, X, y, G, loss=None, workspace=None, stream=None):
    """Step (1): gradients of all P workers into G[P][ld]; returns the workspace used.
    A torch.bfloat16 G selects the form that stores the gradients in 16 bits (an extension)."""
    arr, L = _dims(dims)
    if W.dim() != 2 or X.dim() != 3 or y.dim() != 2:
        raise ValueError("expected W[P][ld], X[P][b][d_in], y[P][b]")
    P, ld = W.shape
    b = X.shape[1]
    N = easgd_mlp_num_params(dims)
    if N == 0:
        raise ValueError(f"invalid layer widths {list(dims)}")
    if X.shape[0] != P or X.shape[2] != dims[0] or tuple(y.shape) != (P, b):
        raise ValueError("X / y shapes do not match W and dims")
    need = (P - 1) * ld + N
    nbytes = easgd_grad_workspace_bytes(dims, P, b)
    if workspace is None:
        workspace = _new(nbytes, torch.uint8, W, stream)
    g16 = G.dtype == torch.bfloat16
    entry = _lib.easgd_grad_bf16 if g16 else _lib.easgd_grad
    _check(entry(arr, L, _dev("W", W, torch.float32, need), ld,
                           _dev("X", X, torch.float32, P * b * dims[0]),
                           _dev("y", y, torch.int32, P * b), P, b,
                           _dev("G", G, torch.bfloat16 if g16 else torch.float32, need),
                           None if loss is None else _dev("loss", loss, torch.float32, P),
                           _dev("workspace", workspace, torch.uint8, nbytes), workspace.numel(),
                           _stream(stream)))
    return workspace


def easgd_layer_product(kind: int, d_in: int, d_out: int, A, out, Wl=None, dZ=None, ld: int = 0, out_ws: int = 0,
                        relu: bool = False, stream=None) -> None:
    """One product of forward / backward propagation alone (a testing aid): kind 0 forward, 1 weight gradient,
    2 input gradient; A[P][b][d_in], Wl[P][ld], dZ[P][b][d_out], out[P][out_ws]."""
    P, b = A.shape[0], A.shape[1]
    _check(_lib.easgd_layer_product(kind, d_in, d_out, P, b, _dev("A", A, torch.float32, P * b * d_in),
                                    None if Wl is None else _dev("Wl", Wl, torch.float32, (P - 1) * ld + (d_in + 1) * d_out),
                                    ld, None if dZ is None else _dev("dZ", dZ, torch.float32, P * b * d_out),
                                    _dev("out", out, torch.float32, (P - 1) * out_ws + 1), out_ws, int(relu),
                                    _stream(stream)))


STATIC_SCRATCH_BYTES = 64 << 20    # EASGD_STATIC_SCRATCH_BYTES of include/easgd.h


def easgd_grad_static(dims: Sequence[int], W, X, y, G, loss=None, stream=None) -> None:
    """easgd_grad on the library's own static workspace: nothing is allocated, here or in the library
    (for callers that cannot allocate; shapes beyond STATIC_SCRATCH_BYTES of workspace are rejected)."""
    arr, L = _dims(dims)
    if W.dim() != 2 or X.dim() != 3 or y.dim() != 2:
        raise ValueError("expected W[P][ld], X[P][b][d_in], y[P][b]")
    P, ld = W.shape
    b = X.shape[1]
    N = easgd_mlp_num_params(dims)
    if N == 0:
        raise ValueError(f"invalid layer widths {list(dims)}")
    if X.shape[0] != P or X.shape[2] != dims[0] or tuple(y.shape) != (P, b):
        raise ValueError("X / y shapes do not match W and dims")
    need = (P - 1) * ld + N
    _check(_lib.easgd_grad_static(arr, L, _dev("W", W, torch.float32, need), ld,
                                  _dev("X", X, torch.float32, P * b * dims[0]),
                                  _dev("y", y, torch.int32, P * b), P, b,
                                  _dev("G", G, torch.float32, need),
                                  None if loss is None else _dev("loss", loss, torch.float32, P),
                                  _stream(stream)))


def easgd_mlp_round_workspace_bytes(dims: Sequence[int], P: int, b: int) -> int:
    return _workspace_cached(tuple(int(d) for d in dims), int(P), int(b), True)


def easgd_mlp_round(dims: Sequence[int], W, Wc, X, y, eta: float, rho: float, V=None, delta: float = 0.0,
                    G=None, loss=None, workspace=None, stream=None):
    """Steps (1)-(5) in one call, the update fused into backward propagation; V selects Eq. (5),(6)
    (a torch.bfloat16 V selects the form that stores the momentum buffers in 16 bits, an extension);
    the gradients are stored only when G is given.  Returns the workspace used."""
    arr, L = _dims(dims)
    if W.dim() != 2 or X.dim() != 3 or y.dim() != 2:
        raise ValueError("expected W[P][ld], X[P][b][d_in], y[P][b]")
    P, ld = W.shape
    b = X.shape[1]
    N = easgd_mlp_num_params(dims)
    if N == 0:
        raise ValueError(f"invalid layer widths {list(dims)}")
    if X.shape[0] != P or X.shape[2] != dims[0] or tuple(y.shape) != (P, b):
        raise ValueError("X / y shapes do not match W and dims")
    if V is not None and tuple(V.shape) != (P, ld):
        raise ValueError("V must have the shape of W")
    need = (P - 1) * ld + N
    nbytes = easgd_mlp_round_workspace_bytes(dims, P, b)
    if workspace is None:
        workspace = _new(nbytes, torch.uint8, W, stream)
    v16 = V is not None and V.dtype == torch.bfloat16
    entry = _lib.easgd_mlp_round_bf16v if v16 else _lib.easgd_mlp_round
    _check(entry(arr, L, _dev("W", W, torch.float32, need),
                                None if V is None else _dev("V", V, torch.bfloat16 if v16 else torch.float32, need),
                                _dev("Wc", Wc, torch.float32, N), ld,
                                _dev("X", X, torch.float32, P * b * dims[0]),
                                _dev("y", y, torch.int32, P * b), P, b,
                                None if G is None else _dev("G", G, torch.float32, need),
                                None if loss is None else _dev("loss", loss, torch.float32, P),
                                eta, rho, delta,
                                _dev("workspace", workspace, torch.uint8, nbytes), workspace.numel(),
                                _stream(stream)))
    return workspace


# ---- rows of logits ----------------------------------------------------------------------------------------------

MAX_TOP = 256                       # EASGD_MAX_TOP of include/easgd.h
_LOGIT_TYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}     # easgd_dtype


def _logit_rows(name: str, t: torch.Tensor):
    """Address, element type, rows, row length and stride of a matrix of logits (rows may be strided, a row's elements not)
    on the current device, where the kernels run."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a CUDA/HIP tensor")
    code = _LOGIT_TYPES.get(t.dtype)
    if code is None:
        raise TypeError(f"{name} must be torch.float32, torch.bfloat16 or torch.float16, got {t.dtype}")
    if t.dim() != 2:
        raise ValueError(f"{name} must be [rows][V]")
    rows, V = t.shape
    ld, step = t.stride()
    if V > 1 and step != 1:
        raise ValueError(f"{name}: a row's elements must follow one another")
    if rows <= 1 or V == 0:
        ld = max(V, 1)
    elif ld < V:
        raise ValueError(f"{name}: rows must not overlap (stride {ld}, length {V})")
    here = torch.cuda.current_device()
    if t.get_device() != here:
        raise ValueError(f"{name} is on {t.device}, the current device is cuda:{here}")
    return t.data_ptr(), code, rows, V, ld


def _given(name: str, t, dtype, shape: tuple, device: int):
    """Address of a tensor of this type and shape on the device with this number; None for None."""
    if t is None:
        return None
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a CUDA/HIP tensor")
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if t.shape != shape or not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous and {list(shape)}, got {list(t.shape)}")
    if t.get_device() != device:
        raise ValueError(f"{name} must be on cuda:{device}, is on {t.device}")
    return t.data_ptr()


def _scratch(nbytes: int, workspace, like, stream):
    """The workspace (kept by the caller until the call is made), its address and size."""
    if workspace is None:
        if nbytes == 0:
            return None, None, 0
        workspace = _new(nbytes, torch.uint8, like, stream)
    elif workspace.device != like.device:
        raise ValueError(f"workspace must be on {like.device}, is on {workspace.device}")
    return workspace, _dev("workspace", workspace, torch.uint8, nbytes), workspace.numel()


@functools.lru_cache(maxsize=256)
def easgd_top_logits_workspace_bytes(rows: int, V: int, k: int) -> int:
    return int(_lib.easgd_top_logits_workspace_bytes(rows, V, k))


@functools.lru_cache(maxsize=256)
def easgd_distill_workspace_bytes(rows: int, V: int, k: int) -> int:
    return int(_lib.easgd_distill_workspace_bytes(rows, V, k))


@functools.lru_cache(maxsize=256)
def easgd_sample_tokens_workspace_bytes(rows: int, V: int) -> int:
    return int(_lib.easgd_sample_tokens_workspace_bytes(rows, V))


_F32, _I32 = torch.float32, torch.int32


def easgd_top_logits(logits, k: int, temperature: float = 1.0, values=None, indices=None, lse=None, workspace=None, stream=None):
    """The k first logits of every row's order and the row's log-sum-exp at `temperature`: what a teacher hands on.
    logits [rows][V] (fp32, bf16 or fp16, rows may be strided) -> values [rows][k] fp32, indices [rows][k] int32,
    lse [rows] fp32; places left over hold -inf and -1."""
    ptr, code, rows, V, ld = _logit_rows("logits", logits)
    k, on = int(k), logits.get_device()
    if k < 1 or k > MAX_TOP:
        raise ValueError(f"k must be in [1, {MAX_TOP}], got {k}")
    if values is None:
        values = _new((rows, k), _F32, logits, stream)
    if indices is None:
        indices = _new((rows, k), _I32, logits, stream)
    if lse is None:
        lse = _new((rows,), _F32, logits, stream)
    keep, ws, nbytes = _scratch(easgd_top_logits_workspace_bytes(rows, V, k), workspace, logits, stream)
    _check(_lib.easgd_top_logits(ptr, code, rows, V, ld, k, temperature, _given("values", values, _F32, (rows, k), on),
                                 _given("indices", indices, _I32, (rows, k), on), _given("lse", lse, _F32, (rows,), on),
                                 ws, nbytes, _stream(stream)))
    return values, indices, lse


def _distill_args(logits, indices, values, temperature, teacher_lse, labels, hard):
    ptr, code, rows, V, ld = _logit_rows("logits", logits)
    if not isinstance(indices, torch.Tensor) or indices.dim() != 2:
        raise ValueError("indices must be [rows][k]")
    k, on = indices.shape[1], logits.get_device()
    return rows, V, k, on, (ptr, code, rows, V, ld, _given("indices", indices, _I32, (rows, k), on), _given("values", values, _F32, (rows, k), on),
                            _given("teacher_lse", teacher_lse, _F32, (rows,), on), k, _given("labels", labels, _I32, (rows,), on),
                            temperature, hard)


def _gradient_rows(logits, dlogits, rows: int, V: int, stream):
    if dlogits is None:
        dlogits = _new((rows, V), logits.dtype, logits, stream)
    ptr, code, drows, dV, dld = _logit_rows("dlogits", dlogits)
    if dlogits.dtype != logits.dtype or drows != rows or dV != V:
        raise ValueError(f"dlogits must be [{rows}][{V}] {logits.dtype}, got {list(dlogits.shape)} {dlogits.dtype}")
    return dlogits, ptr, dld


def easgd_distill_loss(logits, indices, values, temperature: float = 1.0, teacher_lse=None, labels=None, hard: float = 0.0,
                       loss=None, state=None, workspace=None, stream=None):
    """Forward pass of distillation: the loss of every row of student logits [rows][V] against the teacher's top logits
    (indices, values [rows][k]; teacher_lse [rows] turns what they leave over into one more outcome), mixed with the
    cross-entropy of labels [rows] by `hard`.  Returns loss [rows] and state [rows][4], which easgd_distill_grad takes."""
    rows, V, k, on, args = _distill_args(logits, indices, values, temperature, teacher_lse, labels, hard)
    if loss is None:
        loss = _new((rows,), _F32, logits, stream)
    if state is None:
        state = _new((rows, 4), _F32, logits, stream)
    keep, ws, nbytes = _scratch(easgd_distill_workspace_bytes(rows, V, k), workspace, logits, stream)
    _check(_lib.easgd_distill_loss(*args, _given("loss", loss, _F32, (rows,), on), _given("state", state, _F32, (rows, 4), on),
                                   ws, nbytes, _stream(stream)))
    return loss, state


def easgd_distill_grad(logits, indices, values, state, temperature: float = 1.0, teacher_lse=None, labels=None, hard: float = 0.0,
                       scale: float = 1.0, dloss=None, dlogits=None, stream=None):
    """Backward pass of easgd_distill_loss: the gradient of scale * sum(dloss * loss) (dloss None: all ones) with respect to
    the student's logits, in their type."""
    rows, V, k, on, args = _distill_args(logits, indices, values, temperature, teacher_lse, labels, hard)
    dlogits, dptr, dld = _gradient_rows(logits, dlogits, rows, V, stream)
    _check(_lib.easgd_distill_grad(*args, _given("state", state, _F32, (rows, 4), on), _given("dloss", dloss, _F32, (rows,), on),
                                   scale, dptr, dld, _stream(stream)))
    return dlogits


def easgd_distill(logits, indices, values, temperature: float = 1.0, teacher_lse=None, labels=None, hard: float = 0.0,
                  scale: float = 1.0, loss=None, dlogits=None, workspace=None, stream=None):
    """Loss and gradient of distillation in one call: easgd_distill_loss, and the gradient of scale * sum(loss)."""
    rows, V, k, on, args = _distill_args(logits, indices, values, temperature, teacher_lse, labels, hard)
    if loss is None:
        loss = _new((rows,), _F32, logits, stream)
    dlogits, dptr, dld = _gradient_rows(logits, dlogits, rows, V, stream)
    keep, ws, nbytes = _scratch(easgd_distill_workspace_bytes(rows, V, k), workspace, logits, stream)
    _check(_lib.easgd_distill(*args, scale, _given("loss", loss, _F32, (rows,), on), dptr, dld, ws, nbytes, _stream(stream)))
    return loss, dlogits


def easgd_grad_distill(dims: Sequence[int], W, X, indices, values, G, loss=None, temperature: float = 1.0, teacher_lse=None, labels=None,
                       hard: float = 0.0, workspace=None, stream=None):
    """Step (1) with distillation in the place of the softmax cross-entropy: gradients of all P workers into G[P][ld] from the
    teacher's top logits (indices, values [P][b][k]; teacher_lse, labels [P][b]); returns the workspace used."""
    arr, L = _dims(dims)
    if W.dim() != 2 or X.dim() != 3 or indices.dim() != 3:
        raise ValueError("expected W[P][ld], X[P][b][d_in], indices[P][b][k]")
    P, ld = W.shape
    b, k, on = X.shape[1], indices.shape[2], torch.cuda.current_device()
    N = easgd_mlp_num_params(dims)
    if N == 0:
        raise ValueError(f"invalid layer widths {list(dims)}")
    need = (P - 1) * ld + N
    nbytes = easgd_grad_workspace_bytes(dims, P, b)
    for name, t in (("W", W), ("G", G)):
        _dev(name, t, _F32, need)
        if t.get_device() != on:
            raise ValueError(f"{name} must be on cuda:{on}, is on {t.device}")
    workspace, ws, size = _scratch(nbytes, workspace, W, stream)
    _check(_lib.easgd_grad_distill(arr, L, W.data_ptr(), ld, _given("X", X, _F32, (P, b, dims[0]), on),
                                   _given("indices", indices, _I32, (P, b, k), on), _given("values", values, _F32, (P, b, k), on),
                                   _given("teacher_lse", teacher_lse, _F32, (P, b), on), k, _given("labels", labels, _I32, (P, b), on),
                                   P, b, temperature, hard, G.data_ptr(), _given("loss", loss, _F32, (P,), on), ws, size, _stream(stream)))
    return workspace


def easgd_sample_tokens(logits, u, temperature=None, top_k=None, top_p=None, min_p=None, tokens=None, logprob=None,
                        workspace=None, stream=None):
    """One token of every row of logits [rows][V], drawn with the random numbers u [rows] in [0, 1); temperature, top_p,
    min_p (fp32) and top_k (int32) are [rows] tensors on the GPU or None.  Returns tokens [rows] int32 (-1: every logit
    masked) and the logarithm of the probability with which each was drawn."""
    ptr, code, rows, V, ld = _logit_rows("logits", logits)
    if u is None:
        raise TypeError("u must be a CUDA/HIP tensor")
    on, shape = logits.get_device(), (rows,)
    if tokens is None:
        tokens = _new(shape, _I32, logits, stream)
    if logprob is None:
        logprob = _new(shape, _F32, logits, stream)
    keep, ws, nbytes = _scratch(easgd_sample_tokens_workspace_bytes(rows, V), workspace, logits, stream)
    _check(_lib.easgd_sample_tokens(ptr, code, rows, V, ld, _given("u", u, _F32, shape, on), _given("temperature", temperature, _F32, shape, on),
                                    _given("top_k", top_k, _I32, shape, on), _given("top_p", top_p, _F32, shape, on),
                                    _given("min_p", min_p, _F32, shape, on), _given("tokens", tokens, _I32, shape, on),
                                    _given("logprob", logprob, _F32, shape, on), ws, nbytes, _stream(stream)))
    return tokens, logprob


class TokenScores(NamedTuple):
    """What easgd_score_tokens says about the rows; None for what was not asked for."""
    logprob: Optional[torch.Tensor]
    entropy: Optional[torch.Tensor]
    rank: Optional[torch.Tensor]
    top_logprob: Optional[torch.Tensor]
    top_indices: Optional[torch.Tensor]
    state: Optional[torch.Tensor]


@functools.lru_cache(maxsize=256)
def easgd_score_tokens_workspace_bytes(rows: int, V: int, k: int) -> int:
    return int(_lib.easgd_score_tokens_workspace_bytes(rows, V, k))


@functools.lru_cache(maxsize=256)
def easgd_token_loss_workspace_bytes(rows: int, V: int) -> int:
    return int(_lib.easgd_token_loss_workspace_bytes(rows, V))


def _asked(what, shape, dtype, like, stream):
    """An optional result: None or False (not asked for), True (a new tensor) or the caller's tensor."""
    if what is None or what is False:
        return None
    return _new(shape, dtype, like, stream) if what is True else what


def easgd_score_tokens(logits, tokens=None, temperature: float = 1.0, k: int = 0, logprob=None, entropy=True, rank=None,
                       top_logprob=None, top_indices=None, state=None, workspace=None, stream=None) -> TokenScores:
    """Log probabilities of given tokens [rows] int32 under the rows of logits [rows][V] (fp32, bf16 or fp16, rows may be strided) at a
    temperature, the rows' entropies, the tokens' ranks, and the k first alternatives as log probabilities with their places.
    entropy, rank and state (for easgd_score_tokens_grad) are a tensor to fill, True for a new one, or None where they are not
    wanted.  A token outside [0, V) marks a padded row; without tokens there are no logprob and no rank."""
    ptr, code, rows, V, ld = _logit_rows("logits", logits)
    k, on, shape = int(k), logits.get_device(), (rows,)
    if k < 0 or k > MAX_TOP:
        raise ValueError(f"k must be in [0, {MAX_TOP}], got {k}")
    if logprob is None and tokens is not None:
        logprob = _new(shape, _F32, logits, stream)
    entropy = _asked(entropy, shape, _F32, logits, stream)
    rank = _asked(rank, shape, _I32, logits, stream)
    state = _asked(state, (rows, 4), _F32, logits, stream)
    if k == 0 and (top_logprob is not None or top_indices is not None):
        raise ValueError("top_logprob and top_indices need k > 0")
    if k and top_logprob is None:
        top_logprob = _new((rows, k), _F32, logits, stream)
    if k and top_indices is None:
        top_indices = _new((rows, k), _I32, logits, stream)
    keep, ws, nbytes = _scratch(easgd_score_tokens_workspace_bytes(rows, V, k), workspace, logits, stream)
    _check(_lib.easgd_score_tokens(ptr, code, rows, V, ld, _given("tokens", tokens, _I32, shape, on), temperature,
                                   _given("logprob", logprob, _F32, shape, on), _given("entropy", entropy, _F32, shape, on),
                                   _given("rank", rank, _I32, shape, on), k, _given("top_logprob", top_logprob, _F32, (rows, k), on),
                                   _given("top_indices", top_indices, _I32, (rows, k), on), _given("state", state, _F32, (rows, 4), on),
                                   ws, nbytes, _stream_on(stream, on)))
    return TokenScores(logprob, entropy, rank, top_logprob, top_indices, state)


def easgd_score_tokens_grad(logits, tokens, state, temperature: float = 1.0, dlogprob=None, dentropy=None, scale: float = 1.0,
                            dlogits=None, stream=None):
    """Backward pass of easgd_score_tokens: the gradient of scale * sum(dlogprob * logprob + dentropy * entropy) with respect to the
    logits, in their type; either of dlogprob and dentropy [rows] may be None."""
    ptr, code, rows, V, ld = _logit_rows("logits", logits)
    on, shape = logits.get_device(), (rows,)
    dlogits, dptr, dld = _gradient_rows(logits, dlogits, rows, V, stream)
    _check(_lib.easgd_score_tokens_grad(ptr, code, rows, V, ld, _given("tokens", tokens, _I32, shape, on), temperature,
                                        _given("state", state, _F32, (rows, 4), on), _given("dlogprob", dlogprob, _F32, shape, on),
                                        _given("dentropy", dentropy, _F32, shape, on), scale, dptr, dld, _stream_on(stream, on)))
    return dlogits


def easgd_token_loss(logits, tokens, weight=None, bonus: float = 0.0, temperature: float = 1.0, scale: float = 1.0, loss=None, logprob=None,
                     entropy=None, dlogits=None, workspace=None, stream=None):
    """Loss and gradient of given tokens in one call: loss = -weight * logprob - bonus * entropy of every row, and the gradient of
    scale * sum(loss).  Returns loss, logprob, entropy (None unless it is a tensor or True) and dlogits."""
    ptr, code, rows, V, ld = _logit_rows("logits", logits)
    on, shape = logits.get_device(), (rows,)
    if loss is None:
        loss = _new(shape, _F32, logits, stream)
    if logprob is None:
        logprob = _new(shape, _F32, logits, stream)
    entropy = _asked(entropy, shape, _F32, logits, stream)
    dlogits, dptr, dld = _gradient_rows(logits, dlogits, rows, V, stream)
    keep, ws, nbytes = _scratch(easgd_token_loss_workspace_bytes(rows, V), workspace, logits, stream)
    _check(_lib.easgd_token_loss(ptr, code, rows, V, ld, _given("tokens", tokens, _I32, shape, on), _given("weight", weight, _F32, shape, on),
                                 bonus, temperature, scale, _given("loss", loss, _F32, shape, on), _given("logprob", logprob, _F32, shape, on),
                                 _given("entropy", entropy, _F32, shape, on), dptr, dld, ws, nbytes, _stream_on(stream, on)))
    return loss, logprob, entropy, dlogits


def easgd_grad_token_loss(dims: Sequence[int], W, X, tokens, G, loss=None, weight=None, bonus: float = 0.0, temperature: float = 1.0, logprob=None,
                          entropy=None, workspace=None, stream=None):
    """Step (1) with the loss of given tokens in the place of the softmax cross-entropy: gradients of all P workers into G[P][ld] from
    tokens [P][b] and weight [P][b]; logprob and entropy [P][b] are filled where they are given.  Returns the workspace used."""
    arr, L = _dims(dims)
    if W.dim() != 2 or X.dim() != 3:
        raise ValueError("expected W[P][ld], X[P][b][d_in]")
    P, ld = W.shape
    b, on = X.shape[1], torch.cuda.current_device()
    N = easgd_mlp_num_params(dims)
    if N == 0:
        raise ValueError(f"invalid layer widths {list(dims)}")
    need = (P - 1) * ld + N
    for name, t in (("W", W), ("G", G)):
        _dev(name, t, _F32, need)
        if t.get_device() != on:
            raise ValueError(f"{name} must be on cuda:{on}, is on {t.device}")
    workspace, ws, size = _scratch(easgd_grad_workspace_bytes(dims, P, b), workspace, W, stream)
    shape = (P, b)
    _check(_lib.easgd_grad_token_loss(arr, L, W.data_ptr(), ld, _given("X", X, _F32, (P, b, dims[0]), on), _given("tokens", tokens, _I32, shape, on),
                                      _given("weight", weight, _F32, shape, on), P, b, bonus, temperature, G.data_ptr(),
                                      _given("loss", loss, _F32, (P,), on), _given("logprob", logprob, _F32, shape, on),
                                      _given("entropy", entropy, _F32, shape, on), ws, size, _stream_on(stream, on)))
    return workspace


# ---- AdamW on the replicas ---------------------------------------------------------------------------------------

def _replica_rows(name: str, t, N: Optional[int]):
    """Address, element type, P, N and ld of a matrix of replicas or gradients on the current device."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a CUDA/HIP tensor")
    code = _LOGIT_TYPES.get(t.dtype)
    if code is None:
        raise TypeError(f"{name} must be torch.float32, torch.bfloat16 or torch.float16, got {t.dtype}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    P, ld, N = _replica_shape(t, N)
    if N < 1 or N > ld:
        raise ValueError(f"N must be in [1, {ld}], got {N}")
    here = torch.cuda.current_device()
    if t.get_device() != here:
        raise ValueError(f"{name} is on {t.device}, the current device is cuda:{here}")
    return t.data_ptr(), code, P, N, ld, here


@functools.lru_cache(maxsize=256)
def easgd_grad_norms_workspace_bytes(P: int, N: int) -> int:
    return int(_lib.easgd_grad_norms_workspace_bytes(P, N))


def easgd_grad_norms(G, max_norm: float = float("inf"), N: Optional[int] = None, norm=None, clip=None, workspace=None, stream=None):
    """The L2 norm of every worker's gradient G[P][ld] (fp32, bf16 or fp16) and the factor min(1, max_norm / norm) that clips it (0 where the
    norm is infinite or NaN).  Returns norm [P] and clip [P], which adamw_round takes."""
    ptr, code, P, N, ld, on = _replica_rows("G", G, N)
    if norm is None:
        norm = _new((P,), _F32, G, stream)
    if clip is None:
        clip = _new((P,), _F32, G, stream)
    keep, ws, nbytes = _scratch(easgd_grad_norms_workspace_bytes(P, N), workspace, G, stream)
    _check(_lib.easgd_grad_norms(ptr, code, P, N, ld, max_norm, _given("norm", norm, _F32, (P,), on), _given("clip", clip, _F32, (P,), on),
                                 ws, nbytes, _stream_on(stream, on)))
    return norm, clip


ADAMW_BLOCK = 256                   # parameters that share the scales of their moments in 8 bits


def adamw_round(W, M, S, G, step, eta, Wc=None, rho: float = 0.0, beta1: float = 0.9, beta2: float = 0.999, eps: float = 1e-8,
                decay: float = 0.01, tensors=None, clip=None, M_scale=None, S_scale=None, seed: int = 0, N: Optional[int] = None, stream=None) -> None:
    """An AdamW step of all replicas, in place on W[P][ld], M, S (and Wc[N]): with a center the elastic exchange (Eq. (1) with AdamW's
    move in the place of the gradient, Eq. (2)), without one every worker's own step.

    G[P][ld] is fp32, bf16 or fp16.  tensors = (ends int64, rates fp32, decays fp32), all [n] on the GPU, gives the tensors of a replica their own rate
    and decay.  clip [P] fp32 scales every worker's gradient (0: the worker sits the step out).  step is a whole number from 1 on, or a tensor [1] int64,
    eta a number or a tensor [1] fp32, read when the kernel runs (for captured calls).  M of torch.float8_e4m3fn and S of torch.float8_e5m2
    select moments in 8 bits, with M_scale and S_scale [P][ceil(N/256)] fp32 and a seed for their random rounding."""
    wptr, _, P, N, ld, on = _replica_rows("W", W, N)
    if W.dtype != _F32:
        raise TypeError(f"W must be torch.float32, got {W.dtype}")
    shape = (P, ld)
    code = _LOGIT_TYPES.get(getattr(G, "dtype", None))
    if code is None:
        raise TypeError("G must be a torch.float32, torch.bfloat16 or torch.float16 tensor")
    gptr = _given("G", G, G.dtype, shape, on)
    eight = getattr(M, "dtype", None) == torch.float8_e4m3fn
    mptr = _given("M", M, torch.float8_e4m3fn if eight else _F32, shape, on)
    sptr = _given("S", S, torch.float8_e5m2 if eight else _F32, shape, on)
    n, ends, rates, decays = 0, None, None, None
    if tensors is not None:
        ends, rates, decays = tensors
        n = len(ends)
        ends, rates, decays = _given("ends", ends, torch.int64, (n,), on), _given("rates", rates, _F32, (n,), on), _given("decays", decays, _F32, (n,), on)
    step_at = eta_at = None
    if isinstance(step, torch.Tensor):
        step, step_at = 1, _given("step", step, torch.int64, (1,), on)
    if isinstance(eta, torch.Tensor):
        eta, eta_at = 0.0, _given("eta", eta, _F32, (1,), on)
    center = _given("Wc", Wc, _F32, (N,), on)
    clip = _given("clip", clip, _F32, (P,), on)
    if eight:
        blocks = (P, (N + ADAMW_BLOCK - 1) // ADAMW_BLOCK)
        if M_scale is None or S_scale is None:
            raise ValueError("moments in 8 bits need M_scale and S_scale")
        _check(_lib.adamw_round_8bit(wptr, mptr, sptr, _given("M_scale", M_scale, _F32, blocks, on), _given("S_scale", S_scale, _F32, blocks, on), gptr, code,
                                     center, P, N, ld, ends, rates, decays, n, clip, eta, eta_at, rho, beta1, beta2, eps, decay, step, step_at,
                                     seed & 0xFFFFFFFF, _stream_on(stream, on)))
        return
    if M_scale is not None or S_scale is not None:
        raise ValueError("M_scale and S_scale belong to moments in 8 bits")
    _check(_lib.adamw_round(wptr, mptr, sptr, gptr, code, center, P, N, ld, ends, rates, decays, n, clip, eta, eta_at, rho, beta1, beta2, eps, decay,
                            step, step_at, _stream_on(stream, on)))


def stream_copy(dst, src, stream=None) -> None:
    """Measurement aid: dst[:] = src with the library's streaming copy kernel."""
    n = src.numel()
    _check(_lib.easgd_stream_copy(_dev("dst", dst, torch.float32, n), _dev("src", src, torch.float32, n), n, _stream(stream)))


def stream_triad(a, b, c, s: float, stream=None) -> None:
    """Measurement aid: a[:] = b + s*c (two reads, one write per element)."""
    n = a.numel()
    _check(_lib.easgd_stream_triad(_dev("a", a, torch.float32, n), _dev("b", b, torch.float32, n),
                                   _dev("c", c, torch.float32, n), n, s, _stream(stream)))


def stream_mix32(a, b, c, d, e, s: float, stream=None) -> None:
    """Measurement aid: a[:] = c + s*d, b[:] = d + s*e (three reads, two writes per element)."""
    n = a.numel()
    _check(_lib.easgd_stream_mix32(_dev("a", a, torch.float32, n), _dev("b", b, torch.float32, n),
                                   _dev("c", c, torch.float32, n), _dev("d", d, torch.float32, n),
                                   _dev("e", e, torch.float32, n), n, s, _stream(stream)))


def mfma_probe(out, iters: int, mode, blocks_per_cu: int = 2, src=None, stream=None) -> int:
    """Measurement aid: the bare fp32 matrix-instruction loop (see include/easgd.h; mode 0, 1 or 2, a bool counts as
    0 or 1; mode 2 reads `src`).  Returns the flops of the launch."""
    blocks = ctypes.c_uint(0)
    mode = int(mode)
    src_ptr, src_len = (None, 0) if src is None else (_dev("src", src, torch.float32, 4096), src.numel())
    _check(_lib.easgd_mfma_probe(_dev("out", out, torch.float32, out.numel()), out.numel(), int(iters), mode,
                                 int(blocks_per_cu), src_ptr, src_len, ctypes.byref(blocks), _stream(stream)))
    return blocks.value * 4 * int(iters) * 16 * 4096


def round_barrier_timeouts(stream=None) -> int:
    """Blocks that ever gave up waiting at the barrier of a single-launch round on `stream` (synchronises it)."""
    n = int(_lib.easgd_round_barrier_timeouts(_stream(stream)))
    if n < 0:
        _check(n)
    return n


def launch_count() -> int:
    """Measurement aid: kernel launches issued by the library in this process so far."""
    return int(_lib.easgd_launch_count())


def set_option(option: int, value: int) -> None:
    _check(_lib.easgd_set_option(option, value))


def get_option(option: int) -> int:
    return int(_lib.easgd_get_option(option))


def version() -> int:
    return int(_lib.easgd_version())
