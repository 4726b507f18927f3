"""Python binding of the MI355X batched HDC inference library (``libhd.so``).

Argument marshalling only: every step of inference runs in the library's HIP
kernels, called through the C ABI declared in ``include/hd.h``. PyTorch is
used for device memory and streams. There is no fallback: if the compiled
library is missing, importing a function raises.

Operation (ScalableHD, Alg. 1): H = HardSign(X B) (Eq. 7, Eq. 1),
S = H C^T (Eq. 8), labels = argmax_k S (Eq. 9). Single-pass training
(Sec. II-C): C = HardSign of the per-class sums of HardSign(X B).

Behind an answer: products with 4-bit weights (``nibble_*``) and log
probabilities with entropy and alternatives (``logprobs``). Behind learning:
their gradient (``logprobs_grad``) and encodings kept in 8 bits, from which the
class vectors' gradient is read (``ckpt_*``).

Many classes and layers in 8 bits: the cross entropy of encodings and class vectors without the
scores, with its gradient (``class_loss``, ``class_loss_grad``), products in 8-bit integers
(``byte_*``), and dropout without a stored mask (``dropout``).
"""
from __future__ import annotations

import ctypes
import functools
import os
import threading
from typing import NamedTuple

PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(PKG, "libhd.so")

HD_OK, HD_ERR_ARG, HD_ERR_UNSUPPORTED, HD_ERR_WORKSPACE, HD_ERR_HIP = range(5)
HD_F32, HD_BF16, HD_I8 = 0, 1, 2
HD_DETERMINISTIC = 0x100  # flag OR-ed into act: bit-identical results from call to call
ACTS = {"hardsign": 0, "identity": 1}

SYMBOLS = (
    "hd_status_str",
    "hd_encode",
    "hd_similarity",
    "hd_infer_workspace_bytes",
    "hd_infer",
    "hd_model_packed_bytes",
    "hd_pack_model",
    "hd_infer_packed_workspace_bytes",
    "hd_infer_packed",
    "hd_infer_kernel",
    "hd_noalloc_scratch_bytes",
    "hd_infer_packed_noalloc",
    "hd_infer_stream_workspace_bytes",
    "hd_infer_stream",
    "hd_bundle_classes",
    "hd_class_hardsign",
    "hd_bundle_classes_packed",
    "hd_bundle_kernel",
    "hd_nibble_bytes",
    "hd_nibble_pack",
    "hd_nibble_quantize",
    "hd_nibble_unpack",
    "hd_nibble_workspace_bytes",
    "hd_nibble_product",
    "hd_logprobs_workspace_bytes",
    "hd_logprobs",
    "hd_logprobs_grad",
    "hd_ckpt_bytes",
    "hd_ckpt_store",
    "hd_ckpt_load",
    "hd_ckpt_class_grad_workspace_bytes",
    "hd_ckpt_class_grad",
    "hd_byte_bytes",
    "hd_byte_pack",
    "hd_byte_quantize",
    "hd_byte_unpack",
    "hd_byte_rows",
    "hd_byte_workspace_bytes",
    "hd_byte_product",
    "hd_class_loss_workspace_bytes",
    "hd_class_loss",
    "hd_class_loss_grad_workspace_bytes",
    "hd_class_loss_grad_workspace_bytes_of",
    "hd_class_loss_grad",
    "hd_dropout",
)

_lib = None
_lock = threading.Lock()


class HDError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        msg = lib().hd_status_str(status).decode() if _lib is not None else str(status)
        super().__init__(f"{where}: {msg}")


def lib():
    """The loaded ``libhd.so`` with argument types set (raises if absent)."""
    global _lib
    if _lib is not None:
        return _lib
    with _lock:
        if _lib is not None:
            return _lib
        if not os.path.exists(LIB_PATH):
            raise ImportError(
                f"{LIB_PATH} is not built; run paper_2506_09282_amd/build.py "
                "(or __graft_entry__.build()) first")
        L = ctypes.CDLL(LIB_PATH)
        vp, i64, i32, sz = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int, ctypes.c_size_t
        L.hd_status_str.argtypes = [i32]
        L.hd_status_str.restype = ctypes.c_char_p
        L.hd_encode.argtypes = [vp, vp, vp, i64, i64, i64, i32, i32, vp]
        L.hd_encode.restype = i32
        L.hd_similarity.argtypes = [vp, vp, vp, vp, i64, i64, i64, i32, vp]
        L.hd_similarity.restype = i32
        L.hd_infer_workspace_bytes.argtypes = [i64, i64, i64, i64, i32]
        L.hd_infer_workspace_bytes.restype = sz
        L.hd_infer.argtypes = [vp, vp, vp, vp, vp, i64, i64, i64, i64, i32, i32, vp, sz, vp]
        L.hd_infer.restype = i32
        L.hd_model_packed_bytes.argtypes = [i64, i64, i64, i32]
        L.hd_model_packed_bytes.restype = sz
        L.hd_pack_model.argtypes = [vp, vp, i64, i64, i64, i32, vp, sz, vp]
        L.hd_pack_model.restype = i32
        L.hd_infer_packed_workspace_bytes.argtypes = [i64, i64, i64, i64, i32]
        L.hd_infer_packed_workspace_bytes.restype = sz
        L.hd_infer_packed.argtypes = [vp, vp, vp, vp, i64, i64, i64, i64, i32, i32, vp, sz, vp]
        L.hd_infer_packed.restype = i32
        L.hd_infer_kernel.argtypes = [i64, i64, i64, i64, i32, i32]
        L.hd_infer_kernel.restype = ctypes.c_char_p
        L.hd_noalloc_scratch_bytes.argtypes = []
        L.hd_noalloc_scratch_bytes.restype = sz
        L.hd_infer_packed_noalloc.argtypes = [vp, vp, vp, vp, i64, i64, i64, i64, i32, i32, vp]
        L.hd_infer_packed_noalloc.restype = i32
        L.hd_infer_stream_workspace_bytes.argtypes = [i64, i64, i64, i64, i64, i32]
        L.hd_infer_stream_workspace_bytes.restype = sz
        L.hd_infer_stream.argtypes = [vp, vp, vp, vp, vp, vp, i64, i64, i64, i64, i64, i32, i32,
                                      vp, sz, vp]
        L.hd_infer_stream.restype = i32
        L.hd_bundle_classes.argtypes = [vp, vp, vp, vp, i64, i64, i64, i64, i32, vp]
        L.hd_bundle_classes.restype = i32
        L.hd_class_hardsign.argtypes = [vp, vp, i64, i64, vp]
        L.hd_class_hardsign.restype = i32
        L.hd_bundle_classes_packed.argtypes = [vp, vp, vp, vp, i64, i64, i64, i64, i32, vp]
        L.hd_bundle_classes_packed.restype = i32
        L.hd_bundle_kernel.argtypes = [i64, i64, i64, i64, i32, i32]
        L.hd_bundle_kernel.restype = ctypes.c_char_p
        f32 = ctypes.c_float
        L.hd_nibble_bytes.argtypes = [i64, i64, i64]
        L.hd_nibble_bytes.restype = sz
        L.hd_nibble_pack.argtypes = [vp, vp, vp, i64, i64, i64, vp, sz, vp]
        L.hd_nibble_pack.restype = i32
        L.hd_nibble_quantize.argtypes = [vp, i64, i32, i32, i64, i64, i64, i32, vp, sz, vp]
        L.hd_nibble_quantize.restype = i32
        L.hd_nibble_unpack.argtypes = [vp, i32, vp, i64, i64, i64, vp]
        L.hd_nibble_unpack.restype = i32
        L.hd_nibble_workspace_bytes.argtypes = [i64, i64, i32]
        L.hd_nibble_workspace_bytes.restype = sz
        L.hd_nibble_product.argtypes = [vp, i64, vp, i32, vp, i64, i64, i64, i64, i64, i32, i32,
                                        i32, vp, sz, vp]
        L.hd_nibble_product.restype = i32
        L.hd_logprobs_workspace_bytes.argtypes = [i64, i64, i32]
        L.hd_logprobs_workspace_bytes.restype = sz
        L.hd_logprobs.argtypes = [vp, i64, vp, i64, vp, f32, vp, vp, vp, vp, vp, i64, i64, i64,
                                  i32, vp, sz, vp]
        L.hd_logprobs.restype = i32
        L.hd_logprobs_grad.argtypes = [vp, i64, vp, i64, vp, f32, vp, vp, vp, vp, vp, i64, i64,
                                       i64, i32, vp]
        L.hd_logprobs_grad.restype = i32
        L.hd_ckpt_bytes.argtypes = [i64, i64]
        L.hd_ckpt_bytes.restype = sz
        L.hd_ckpt_store.argtypes = [vp, i64, i64, i64, i32, vp, sz, vp]
        L.hd_ckpt_store.restype = i32
        L.hd_ckpt_load.argtypes = [vp, vp, i64, i64, i64, i32, vp]
        L.hd_ckpt_load.restype = i32
        L.hd_ckpt_class_grad_workspace_bytes.argtypes = [i64, i64, i64, i32]
        L.hd_ckpt_class_grad_workspace_bytes.restype = sz
        L.hd_ckpt_class_grad.argtypes = [vp, i64, vp, vp, i64, i64, i64, i32, i32, vp, sz, vp]
        L.hd_ckpt_class_grad.restype = i32
        L.hd_byte_bytes.argtypes = [i64, i64]
        L.hd_byte_bytes.restype = sz
        L.hd_byte_pack.argtypes = [vp, vp, i64, i64, vp, sz, vp]
        L.hd_byte_pack.restype = i32
        L.hd_byte_quantize.argtypes = [vp, i64, i32, i64, i64, i32, vp, sz, vp]
        L.hd_byte_quantize.restype = i32
        L.hd_byte_unpack.argtypes = [vp, vp, i64, i64, vp]
        L.hd_byte_unpack.restype = i32
        L.hd_byte_rows.argtypes = [vp, i64, i64, i64, i32, vp, vp, vp]
        L.hd_byte_rows.restype = i32
        L.hd_byte_workspace_bytes.argtypes = [i64, i64, i64, i32]
        L.hd_byte_workspace_bytes.restype = sz
        L.hd_byte_product.argtypes = [vp, i64, vp, vp, vp, i64, i64, i64, i64, i32, i32, i32, vp,
                                      sz, vp]
        L.hd_byte_product.restype = i32
        L.hd_class_loss_workspace_bytes.argtypes = [i64, i64, i64, i32]
        L.hd_class_loss_workspace_bytes.restype = sz
        L.hd_class_loss.argtypes = [vp, i64, vp, i64, vp, vp, f32, vp, vp, i64, i64, i64, i32, vp,
                                    sz, vp]
        L.hd_class_loss.restype = i32
        L.hd_class_loss_grad_workspace_bytes.argtypes = [i64, i64, i64, i32]
        L.hd_class_loss_grad_workspace_bytes.restype = sz
        L.hd_class_loss_grad_workspace_bytes_of.argtypes = [i64, i64, i64, i32, i32, i32]
        L.hd_class_loss_grad_workspace_bytes_of.restype = sz
        L.hd_class_loss_grad.argtypes = [vp, i64, vp, i64, vp, vp, f32, vp, vp, vp, vp, i64, i64,
                                         i64, i32, vp, sz, vp]
        L.hd_class_loss_grad.restype = i32
        u64, f64 = ctypes.c_uint64, ctypes.c_double
        L.hd_dropout.argtypes = [vp, i64, vp, i64, i64, i64, f64, u64, u64, vp, i32, vp]
        L.hd_dropout.restype = i32
        _lib = L
        return L


def _torch():
    import torch
    return torch


def _dt_of(dtype) -> int:
    torch = _torch()
    if dtype == torch.float32:
        return HD_F32
    if dtype == torch.bfloat16:
        return HD_BF16
    if dtype == torch.int8:
        return HD_I8
    raise TypeError(f"unsupported dtype {dtype}; use float32, bfloat16 or int8")


def _dt(t) -> int:
    return _dt_of(t.dtype)


def _check_dev(*ts):
    for t in ts:
        if not t.is_cuda:
            raise ValueError("tensors must be on the GPU")
        if not t.is_contiguous():
            raise ValueError("tensors must be contiguous (row-major)")


def _stream_ptr(device) -> int:
    torch = _torch()
    if device.index is None:
        return torch.cuda.current_stream(device).cuda_stream
    return torch._C._cuda_getCurrentRawStream(device.index)  # (without a Stream object)


def _raise(st: int, where: str):
    if st != HD_OK:
        raise HDError(st, where)


# Workspaces are cached per (device, stream, size); the library leaves the
# parts that must start at zero zeroed after every call of the same shape,
# so a cached buffer is only zeroed when first allocated for that key. A call that is
# captured into a graph has a workspace of that graph's instead, zeroed by each replay: a
# graph's memory holds nothing before its first replay, and replays may run beside
# eager calls and other graphs.
_ws_cache: dict = {}


@functools.lru_cache(maxsize=1024)
def _need(query: str, device: int, *sizes) -> int:
    """A workspace size query's answer (a function of the sizes and the device)."""
    return int(getattr(lib(), query)(*sizes))


def _workspace(device, nbytes: int, key, grows: bool = False):
    """A zeroed workspace of ``nbytes``, or with ``grows`` (for calls that leave all of it
    zeroed, so that one serves every shape) of at least that."""
    torch = _torch()
    if nbytes == 0:
        return None
    if torch.cuda.is_current_stream_capturing():
        return torch.zeros(nbytes, dtype=torch.uint8, device=device)
    k = (device.index, _stream_ptr(device), key, 0 if grows else nbytes)
    ws = _ws_cache.get(k)
    if ws is None or ws.numel() < nbytes:
        ws = torch.zeros(nbytes, dtype=torch.uint8, device=device)
        _ws_cache[k] = ws
    return ws


def encode(X, B, act: str = "hardsign"):
    """Stage I alone: H[N, D] float32 = act(X B)."""
    torch = _torch()
    _check_dev(X, B)
    if X.dtype != B.dtype:
        raise TypeError("X and B must have the same dtype")
    N, F = X.shape
    F2, D = B.shape
    if F2 != F:
        raise ValueError("shape mismatch")
    H = torch.empty((N, D), dtype=torch.float32, device=X.device)
    st = lib().hd_encode(X.data_ptr(), B.data_ptr(), H.data_ptr(), N, F, D, _dt(X), ACTS[act],
                         _stream_ptr(X.device))
    _raise(st, "hd_encode")
    return H


def similarity(H, C, return_scores: bool = False):
    """Stage II alone: labels[N] int32 (and scores[N, K] float32)."""
    torch = _torch()
    _check_dev(H, C)
    if H.dtype != torch.float32:
        raise TypeError("H must be float32")
    N, D = H.shape
    K, D2 = C.shape
    if D2 != D:
        raise ValueError("shape mismatch")
    labels = torch.empty(N, dtype=torch.int32, device=H.device)
    scores = torch.empty((N, K), dtype=torch.float32, device=H.device) if return_scores else None
    st = lib().hd_similarity(H.data_ptr(), C.data_ptr(), labels.data_ptr(),
                             scores.data_ptr() if scores is not None else None, N, D, K, _dt(C),
                             _stream_ptr(H.device))
    _raise(st, "hd_similarity")
    return (labels, scores) if return_scores else labels


def infer_workspace_bytes(N: int, F: int, D: int, K: int, dtype) -> int:
    dt = _dt_of(dtype)
    return int(lib().hd_infer_workspace_bytes(N, F, D, K, dt))


def infer_kernel(N: int, F: int, D: int, K: int, dtype, packed: bool = True) -> str:
    """Name of the main kernel hd_infer / hd_infer_packed launches for these sizes."""
    dt = _dt_of(dtype)
    return lib().hd_infer_kernel(N, F, D, K, dt, 1 if packed else 0).decode()


def _act(act: str, deterministic: bool) -> int:
    return ACTS[act] | (HD_DETERMINISTIC if deterministic else 0)


def infer(X, B, C, act: str = "hardsign", return_scores: bool = False, out=None,
          workspace=None, deterministic: bool = False):
    """Alg. 1 fused: labels[N] int32 (and scores[N, K] float32).

    ``deterministic``: bit-identical scores and labels from call to call
    (fixed-order reduction of the partial scores).

    ``out`` may be a (labels, scores-or-None) pair of preallocated tensors.
    ``workspace`` may be a zeroed uint8 device tensor of at least
    ``infer_workspace_bytes(...)`` bytes; otherwise a cached one is used.
    """
    torch = _torch()
    _check_dev(X, B, C)
    if not (X.dtype == B.dtype == C.dtype):
        raise TypeError("X, B and C must share a dtype")
    N, F = X.shape
    F2, D = B.shape
    K, D2 = C.shape
    if F2 != F or D2 != D:
        raise ValueError("shape mismatch")
    dt = _dt(X)
    L = lib()
    if out is not None:
        labels, scores = out
    else:
        labels = torch.empty(N, dtype=torch.int32, device=X.device)
        scores = (torch.empty((N, K), dtype=torch.float32, device=X.device)
                  if return_scores else None)
    need = _need("hd_infer_workspace_bytes", X.device.index, N, F, D, K, dt)
    ws = workspace if workspace is not None else _workspace(X.device, need, ("infer", N, F, D, K, dt))
    st = L.hd_infer(X.data_ptr(), B.data_ptr(), C.data_ptr(), labels.data_ptr(),
                    scores.data_ptr() if scores is not None else None, N, F, D, K, dt,
                    _act(act, deterministic),
                    ws.data_ptr() if ws is not None else None,
                    ws.numel() if ws is not None else 0, _stream_ptr(X.device))
    _raise(st, "hd_infer")
    return (labels, scores) if (return_scores or out is not None) else labels


class PackedModel:
    """A model tiled once by ``hd_pack_model`` (opaque device image)."""

    def __init__(self, image, F: int, D: int, K: int, dt: int):
        self.image, self.F, self.D, self.K, self.dt = image, F, D, K, dt


def pack_model(B, C=None, K: int = 1) -> PackedModel:
    """Tile B and C once (Sec. III-D). ``C=None`` packs B alone (the class
    part of the image is zero, sized for ``K`` classes): a model for
    ``bundle_classes_packed`` before the class hypervectors exist."""
    torch = _torch()
    _check_dev(B)
    F, D = B.shape
    if C is not None:
        _check_dev(C)
        if B.dtype != C.dtype:
            raise TypeError("B and C must share a dtype")
        K, D2 = C.shape
        if D2 != D:
            raise ValueError("shape mismatch")
    dt = _dt(B)
    L = lib()
    nbytes = int(L.hd_model_packed_bytes(F, D, K, dt))
    image = torch.empty(nbytes, dtype=torch.uint8, device=B.device)
    st = L.hd_pack_model(B.data_ptr(), C.data_ptr() if C is not None else None, F, D, K, dt,
                         image.data_ptr(), nbytes, _stream_ptr(B.device))
    _raise(st, "hd_pack_model")
    return PackedModel(image, F, D, K, dt)


def infer_packed(X, model: PackedModel, act: str = "hardsign", return_scores: bool = False,
                 out=None, workspace=None, deterministic: bool = False):
    """Alg. 1 fused from a packed model: labels[N] (and scores[N, K])."""
    torch = _torch()
    _check_dev(X)
    if _dt(X) != model.dt:
        raise TypeError("X dtype differs from the packed model's")
    N, F = X.shape
    if F != model.F:
        raise ValueError("shape mismatch")
    D, K, dt = model.D, model.K, model.dt
    L = lib()
    if out is not None:
        labels, scores = out
    else:
        labels = torch.empty(N, dtype=torch.int32, device=X.device)
        scores = (torch.empty((N, K), dtype=torch.float32, device=X.device)
                  if return_scores else None)
    need = _need("hd_infer_packed_workspace_bytes", X.device.index, N, F, D, K, dt)
    ws = workspace if workspace is not None else _workspace(X.device, need,
                                                            ("packed", N, F, D, K, dt))
    st = L.hd_infer_packed(X.data_ptr(), model.image.data_ptr(), labels.data_ptr(),
                           scores.data_ptr() if scores is not None else None, N, F, D, K, dt,
                           _act(act, deterministic), ws.data_ptr() if ws is not None else None,
                           ws.numel() if ws is not None else 0, _stream_ptr(X.device))
    _raise(st, "hd_infer_packed")
    return (labels, scores) if (return_scores or out is not None) else labels


def infer_packed_noalloc(X, model: PackedModel, act: str = "hardsign", return_scores: bool = False,
                         out=None, deterministic: bool = False):
    """``infer_packed`` on the library's fixed scratch (no workspace argument;
    calls on one GPU must not overlap in time)."""
    torch = _torch()
    _check_dev(X)
    if _dt(X) != model.dt:
        raise TypeError("X dtype differs from the packed model's")
    N, F = X.shape
    if F != model.F:
        raise ValueError("shape mismatch")
    D, K, dt = model.D, model.K, model.dt
    if out is not None:
        labels, scores = out
    else:
        labels = torch.empty(N, dtype=torch.int32, device=X.device)
        scores = (torch.empty((N, K), dtype=torch.float32, device=X.device)
                  if return_scores else None)
    st = lib().hd_infer_packed_noalloc(X.data_ptr(), model.image.data_ptr(), labels.data_ptr(),
                                       scores.data_ptr() if scores is not None else None, N, F, D,
                                       K, dt, _act(act, deterministic), _stream_ptr(X.device))
    _raise(st, "hd_infer_packed_noalloc")
    return (labels, scores) if (return_scores or out is not None) else labels


def stream_workspace_bytes(nbatch: int, N: int, F: int, D: int, K: int, dtype) -> int:
    dt = _dt_of(dtype)
    return int(lib().hd_infer_stream_workspace_bytes(nbatch, N, F, D, K, dt))


def infer_stream(X, model: PackedModel, act: str = "hardsign", return_scores: bool = False,
                 ready=None, done=None, out=None, workspace=None):
    """Streaming inference: ``X`` is [nbatch, N, F] (a queue of batches); one
    persistent launch returns labels [nbatch, N] (and scores [nbatch, N, K]).

    ``ready``/``done``: optional int32 tensors of one element (device memory
    or pinned host memory) for the queue counter and the batches-done counter.
    ``workspace``: a zeroed uint8 device tensor of at least
    ``stream_workspace_bytes(...)`` bytes; otherwise a cached one is used."""
    torch = _torch()
    _check_dev(X)
    if _dt(X) != model.dt:
        raise TypeError("X dtype differs from the packed model's")
    if X.dim() != 3:
        raise ValueError("X must be [nbatch, N, F]")
    nbatch, N, F = X.shape
    if F != model.F:
        raise ValueError("shape mismatch")
    D, K, dt = model.D, model.K, model.dt
    L = lib()
    if out is not None:
        labels, scores = out
    else:
        labels = torch.empty((nbatch, N), dtype=torch.int32, device=X.device)
        scores = (torch.empty((nbatch, N, K), dtype=torch.float32, device=X.device)
                  if return_scores else None)
    need = _need("hd_infer_stream_workspace_bytes", X.device.index, nbatch, N, F, D, K, dt)
    if need == 0 and nbatch > 0:
        raise HDError(HD_ERR_UNSUPPORTED, "hd_infer_stream")
    ws = workspace if workspace is not None else _workspace(X.device, need,
                                                            ("stream", nbatch, N, F, D, K, dt))
    st = L.hd_infer_stream(X.data_ptr(), model.image.data_ptr(),
                           ready.data_ptr() if ready is not None else None, labels.data_ptr(),
                           scores.data_ptr() if scores is not None else None,
                           done.data_ptr() if done is not None else None, nbatch, N, F, D, K, dt,
                           ACTS[act], ws.data_ptr() if ws is not None else None,
                           ws.numel() if ws is not None else 0, _stream_ptr(X.device))
    _raise(st, "hd_infer_stream")
    return (labels, scores) if (return_scores or out is not None) else labels


def bundle_classes(X, B, y, K: int, counts=None):
    """Single-pass training, accumulation step (Sec. II-C): adds
    HardSign(X_n B) into ``counts[y[n]]`` for every sample with 0 <= y[n] < K
    and returns ``counts`` ([K, D] int32; a new zeroed tensor when None).
    Calls with the same ``counts`` accumulate, so a training set can be fed
    in chunks."""
    torch = _torch()
    _check_dev(X, B, y)
    if X.dtype != B.dtype:
        raise TypeError("X and B must have the same dtype")
    if y.dtype != torch.int32:
        raise TypeError("y must be int32")
    N, F = X.shape
    F2, D = B.shape
    if F2 != F or y.shape != (N,):
        raise ValueError("shape mismatch")
    if counts is None:
        counts = torch.zeros((K, D), dtype=torch.int32, device=X.device)
    else:
        _check_dev(counts)
        if counts.dtype != torch.int32 or tuple(counts.shape) != (K, D):
            raise ValueError("counts must be int32 [K, D]")
    st = lib().hd_bundle_classes(X.data_ptr(), B.data_ptr(), y.data_ptr(), counts.data_ptr(), N,
                                 F, D, K, _dt(X), _stream_ptr(X.device))
    _raise(st, "hd_bundle_classes")
    return counts


def bundle_classes_packed(X, model: PackedModel, y, K: int, counts=None):
    """``bundle_classes`` on the matrix cores, reading B from a packed model
    (``pack_model(B)`` or ``pack_model(B, C)``; the class part is not read)."""
    torch = _torch()
    _check_dev(X, y)
    if _dt(X) != model.dt:
        raise TypeError("X dtype differs from the packed model's")
    if y.dtype != torch.int32:
        raise TypeError("y must be int32")
    N, F = X.shape
    if F != model.F or y.shape != (N,):
        raise ValueError("shape mismatch")
    D = model.D
    if counts is None:
        counts = torch.zeros((K, D), dtype=torch.int32, device=X.device)
    else:
        _check_dev(counts)
        if counts.dtype != torch.int32 or tuple(counts.shape) != (K, D):
            raise ValueError("counts must be int32 [K, D]")
    st = lib().hd_bundle_classes_packed(X.data_ptr(), model.image.data_ptr(), y.data_ptr(),
                                        counts.data_ptr(), N, F, D, K, model.dt,
                                        _stream_ptr(X.device))
    _raise(st, "hd_bundle_classes_packed")
    return counts


def bundle_kernel(N: int, F: int, D: int, K: int, dtype, packed: bool = True) -> str:
    """Name of the kernel bundle_classes(_packed) launches for these sizes."""
    dt = _dt_of(dtype)
    return lib().hd_bundle_kernel(N, F, D, K, dt, 1 if packed else 0).decode()


def class_hardsign(counts, out=None):
    """Normalisation step (Eq. 1): the class hypervectors M [K, D] float32,
    +1 where counts >= 0 (ties and empty classes) and -1 elsewhere."""
    torch = _torch()
    _check_dev(counts)
    if counts.dtype != torch.int32 or counts.dim() != 2:
        raise ValueError("counts must be int32 [K, D]")
    K, D = counts.shape
    M = out if out is not None else torch.empty((K, D), dtype=torch.float32,
                                                device=counts.device)
    _check_dev(M)
    if M.dtype != torch.float32 or tuple(M.shape) != (K, D):
        raise ValueError("out must be float32 [K, D]")
    st = lib().hd_class_hardsign(counts.data_ptr(), M.data_ptr(), K, D,
                                 _stream_ptr(counts.device))
    _raise(st, "hd_class_hardsign")
    return M


def train(X, B, y, K: int):
    """Single-pass training in one call: M [K, D] float32 = class_hardsign(
    bundle_classes(X, B, y, K))."""
    return class_hardsign(bundle_classes(X, B, y, K))


# ---- Operators behind answers and learning ------------------------------------------------
#
# A call here takes a few microseconds on the GPU at the smallest sizes, so the binding
# looks each property up once and asks for the stream by its device's index.

_codes: dict = {}  # torch dtype -> hd_dtype, of the matrices these operators take


def _float_codes() -> dict:
    if not _codes:
        torch = _torch()
        _codes.update({torch.float32: HD_F32, torch.bfloat16: HD_BF16})
    return _codes


def _raw_stream(index: int) -> int:
    return _torch()._C._cuda_getCurrentRawStream(index)


def _rows(t, name: str):
    """A float32 or bfloat16 matrix on the GPU whose rows are contiguous:
    (rows, columns, row stride, hd_dtype, device index)."""
    index = t.get_device()
    if index < 0:
        raise ValueError("tensors must be on the GPU")
    code = (_codes or _float_codes()).get(t.dtype)
    if code is None:
        raise TypeError(f"{name} must be float32 or bfloat16")
    if t.dim() != 2:
        raise ValueError(f"{name} must be a matrix")
    rows, cols = t.shape
    ld, step = t.stride()
    if step != 1 and cols > 1:
        raise ValueError(f"{name} must have contiguous rows")
    if ld < cols:
        # (the stride of a single row or of none is not used, and may be anything)
        if rows > 1:
            raise ValueError(f"{name} must not have overlapping rows")
        ld = cols
    return rows, cols, ld, code, index


def _vec(t, name: str, dtype, n: int, index: int) -> int:
    """The address of a contiguous vector of n on the device ``index``."""
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}")
    if t.get_device() != index or t.shape != (n,) or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous vector of {n} on GPU {index}")
    return t.data_ptr()


def _ptr(t):
    return t.data_ptr() if t is not None else None


class NibbleWeights:
    """A matrix in 4 bits with group scales, laid out once (opaque device image)."""

    def __init__(self, image, outer: int, inner: int, group: int, zeros: bool):
        self.image, self.outer, self.inner = image, outer, inner
        self.group, self.zeros = group, zeros


def _nibble_image(outer: int, inner: int, group: int, device):
    torch = _torch()
    nbytes = int(lib().hd_nibble_bytes(outer, inner, group))
    return torch.empty(nbytes, dtype=torch.uint8, device=device), nbytes


def nibble_pack(codes, scales, zeros=None, inner: int = 0, group: int = 64) -> NibbleWeights:
    """4-bit weights from given codes: ``codes`` [outer, ceil(inner/2)] uint8 (input
    2j in the low half of byte j), ``scales`` [outer, ceil(inner/group)] bfloat16,
    ``zeros`` the same shape uint8 (0..15) or None (8 everywhere). ``inner`` 0
    stands for twice the bytes of a row."""
    torch = _torch()
    _check_dev(codes, scales)
    if codes.dtype != torch.uint8 or scales.dtype != torch.bfloat16:
        raise TypeError("codes must be uint8 and scales bfloat16")
    if codes.dim() != 2 or scales.dim() != 2:
        raise ValueError("codes and scales must be matrices")
    outer, half = codes.shape
    inner = inner or 2 * half
    if group not in (32, 64, 128):
        raise ValueError("group must be 32, 64 or 128")
    groups = -(-inner // group)
    if half != -(-inner // 2) or tuple(scales.shape) != (outer, groups):
        raise ValueError("shape mismatch")
    if zeros is not None:
        _check_dev(zeros)
        if zeros.dtype != torch.uint8:
            raise TypeError("zeros must be uint8")
        if tuple(zeros.shape) != (outer, groups):
            raise ValueError("shape mismatch")
    image, nbytes = _nibble_image(outer, inner, group, codes.device)
    st = lib().hd_nibble_pack(codes.data_ptr(), scales.data_ptr(), _ptr(zeros), outer, inner,
                              group, image.data_ptr(), nbytes, _stream_ptr(codes.device))
    _raise(st, "hd_nibble_pack")
    return NibbleWeights(image, outer, inner, group, zeros is not None)


def nibble_quantize(W, group: int = 64, inner_rows: bool = False,
                    zeros: bool = False) -> NibbleWeights:
    """4-bit weights from numbers: ``W`` [outer, inner] (class hypervectors), or with
    ``inner_rows`` [inner, outer] (base hypervectors B[F, D]); float32 or bfloat16.
    ``zeros``: min-max codes with zero points instead of symmetric ones."""
    outer, inner, ld, dt, index = _rows(W, "W")
    if inner_rows:
        outer, inner = inner, outer
    image, nbytes = _nibble_image(outer, inner, group, W.device)
    st = lib().hd_nibble_quantize(W.data_ptr(), ld, int(inner_rows), int(zeros), outer, inner,
                                  group, dt, image.data_ptr(), nbytes, _raw_stream(index))
    _raise(st, "hd_nibble_quantize")
    return NibbleWeights(image, outer, inner, group, bool(zeros))


def nibble_unpack(w: NibbleWeights):
    """The weights that ``w`` stands for: [outer, inner] float32."""
    torch = _torch()
    W = torch.empty((w.outer, w.inner), dtype=torch.float32, device=w.image.device)
    st = lib().hd_nibble_unpack(w.image.data_ptr(), int(w.zeros), W.data_ptr(), w.outer, w.inner,
                                w.group, _stream_ptr(w.image.device))
    _raise(st, "hd_nibble_unpack")
    return W


def nibble_product(X, w: NibbleWeights, act: str = "identity", dtype=None, out=None):
    """Y[N, outer] = act(X w^T) for X [N, inner] float32 or bfloat16; ``dtype`` of Y
    defaults to X's. ``act`` "hardsign" encodes (Stage I on 4-bit base vectors)."""
    N, inner, ldx, x_dt, index = _rows(X, "X")
    outer, image = w.outer, w.image
    if inner != w.inner:
        raise ValueError("shape mismatch")
    if image.get_device() != index:
        raise ValueError("X and the weights must be on one device")
    if out is None:
        if dtype is None or dtype == X.dtype:
            y_dt = x_dt
        else:
            y_dt = _codes.get(dtype)
            if y_dt is None:
                raise TypeError("dtype must be float32 or bfloat16")
        out, ldy = _torch().empty(N, outer, dtype=dtype or X.dtype, device=X.device), outer
    else:
        _, _, ldy, y_dt, out_index = _rows(out, "out")
        if out_index != index or out.shape != (N, outer):
            raise ValueError("out must be [N, outer] on X's device")
        if dtype is not None and out.dtype != dtype:
            raise TypeError("out has another dtype")
    need = _need("hd_nibble_workspace_bytes", index, N, inner, x_dt)
    ws = None
    if need:
        torch = _torch()
        ws = torch.empty(need, dtype=torch.uint8, device=X.device)
    st = lib().hd_nibble_product(X.data_ptr(), ldx, image.data_ptr(), w.zeros, out.data_ptr(),
                                 ldy, N, outer, inner, w.group, x_dt, y_dt, ACTS[act], _ptr(ws),
                                 need, _raw_stream(index))
    _raise(st, "hd_nibble_product")
    return out


class LogProbs(NamedTuple):
    """What ``logprobs`` gives for N rows: ``logp`` [N] (None without ``y``),
    ``entropy`` [N], ``stats`` [N, 2] (the largest score m, and log sum exp
    scale (s - m)), ``ids`` and ``top_logp`` [N, top] (None for top 0). They are
    parts of one allocation."""
    logp: object
    entropy: object
    stats: object
    ids: object
    top_logp: object


def _mask_arg(mask, N: int, K: int, index: int):
    """Address and row stride of a mask [K] or [N, K] (bool or uint8)."""
    torch = _torch()
    if mask is None:
        return None, 0
    if mask.get_device() != index:
        raise ValueError("mask must be on the scores' device")
    if mask.dtype not in (torch.bool, torch.uint8):
        raise TypeError("mask must be bool or uint8")
    if mask.shape == (K,):
        if K > 1 and mask.stride(0) != 1:
            raise ValueError("mask must be contiguous")
        return mask.data_ptr(), 0
    if mask.shape != (N, K):
        raise ValueError("mask must be [K] or [N, K]")
    ldm, step = mask.stride()
    if K > 1 and step != 1:
        raise ValueError("mask must have contiguous rows")
    if N == 1 or ldm == 0:  # one row, or one row expanded
        return mask.data_ptr(), 0
    if ldm < K:
        raise ValueError("mask must not have overlapping rows")
    return mask.data_ptr(), ldm


def logprobs_workspace_bytes(N: int, K: int, dtype) -> int:
    return int(lib().hd_logprobs_workspace_bytes(N, K, _dt_of(dtype)))


def logprobs(scores, y=None, top: int = 0, scale: float = 1.0, mask=None,
             workspace=None) -> LogProbs:
    """Log probabilities of the classes ``y`` [N] int32 (outside [0, K): none asked
    for) under softmax(scale * scores), scores [N, K] float32 or bfloat16, with
    the entropy and the ``top`` (up to 32) best alternatives. ``mask`` [K] or [N, K]:
    classes that are False take no part. ``workspace`` may be a zeroed uint8
    device tensor of ``logprobs_workspace_bytes(...)`` bytes."""
    torch = _torch()
    N, K, ld, dt, index = _rows(scores, "scores")
    device = scores.device
    yptr = _vec(y, "y", torch.int32, N, index) if y is not None else None
    mptr, ldm = (None, 0) if mask is None else _mask_arg(mask, N, K, index)
    each = N * top if top > 0 else 0
    buf = torch.empty(4 * N + 2 * each, dtype=torch.float32, device=device)
    at = buf.data_ptr()  # stats, entropy, logp, ids, top_logp
    ws = workspace
    if ws is None:
        need = _need("hd_logprobs_workspace_bytes", index, N, K, dt)
        if need:
            ws = _workspace(device, need, "logprobs", grows=True)
    elif ws.dtype != torch.uint8 or ws.get_device() != index or not ws.is_contiguous():
        raise ValueError("workspace must be a contiguous uint8 tensor on the scores' device")
    st = lib().hd_logprobs(scores.data_ptr(), ld, mptr, ldm, yptr, scale,
                           at + 12 * N if yptr is not None else None, at + 8 * N, at,
                           at + 16 * N if each else None, at + 16 * N + 4 * each if each else None,
                           N, K, top, dt, _ptr(ws), ws.numel() if ws is not None else 0,
                           _raw_stream(index))
    _raise(st, "hd_logprobs")
    if each:
        stats, entropy, logp, ids, best = buf.split_with_sizes((2 * N, N, N, each, each))
        ids, best = ids.view(torch.int32).view(N, top), best.view(N, top)
    else:
        stats, entropy, logp = buf.split_with_sizes((2 * N, N, N))
        ids = torch.empty((N, top), dtype=torch.int32, device=device) if top > 0 else None
        best = torch.empty((N, top), dtype=torch.float32, device=device) if top > 0 else None
    return LogProbs(logp if yptr is not None else None, entropy, stats.view(N, 2), ids, best)


def logprobs_grad(scores, y, lp: LogProbs, g_logp=None, g_entropy=None, scale: float = 1.0,
                  mask=None, out=None):
    """The gradient of sum(g_logp * logp + g_entropy * entropy) with respect to the
    scores, [N, K] of their dtype; ``lp`` is what ``logprobs`` gave for the same
    scores, scale and mask. ``out`` may be the scores themselves."""
    torch = _torch()
    f32 = torch.float32
    N, K, ld, dt, index = _rows(scores, "scores")
    yptr = _vec(y, "y", torch.int32, N, index) if y is not None else None
    glp = _vec(g_logp, "g_logp", f32, N, index) if g_logp is not None else None
    gep = _vec(g_entropy, "g_entropy", f32, N, index) if g_entropy is not None else None
    entropy, stats = _vec(lp.entropy, "entropy", f32, N, index), lp.stats
    if (stats.shape != (N, 2) or stats.dtype != f32 or not stats.is_contiguous()
            or stats.get_device() != index):
        raise ValueError("stats must be float32 [N, 2] on the scores' device")
    mptr, ldm = (None, 0) if mask is None else _mask_arg(mask, N, K, index)
    if out is None:
        out, ldd = torch.empty(N, K, dtype=scores.dtype, device=scores.device), K
    else:
        _, _, ldd, out_dt, out_index = _rows(out, "out")
        if out.shape != (N, K) or out_dt != dt or out_index != index:
            raise ValueError("out must have the scores' shape, dtype and device")
    st = lib().hd_logprobs_grad(scores.data_ptr(), ld, mptr, ldm, yptr, scale, stats.data_ptr(),
                                entropy, glp, gep, out.data_ptr(), ldd, N, K, dt,
                                _raw_stream(index))
    _raise(st, "hd_logprobs_grad")
    return out


class Checkpoint:
    """Activations [N, D] kept in 8 bits (opaque device image)."""

    def __init__(self, image, N: int, D: int):
        self.image, self.N, self.D = image, N, D


def ckpt_store(H, out=None) -> Checkpoint:
    """Keeps activations ``H`` [N, D] (float32 or bfloat16) in 8 bits, 64 rows of a
    column sharing a scale. ``out``: a Checkpoint of the same sizes to overwrite."""
    N, D, ld, dt, index = _rows(H, "H")
    nbytes = _need("hd_ckpt_bytes", index, N, D)
    if out is None:
        torch = _torch()
        out = Checkpoint(torch.empty(nbytes, dtype=torch.uint8, device=H.device), N, D)
    elif (out.N, out.D) != (N, D) or out.image.get_device() != index:
        raise ValueError("out must be a checkpoint of H's sizes on its device")
    st = lib().hd_ckpt_store(H.data_ptr(), ld, N, D, dt, out.image.data_ptr(), nbytes,
                             _raw_stream(index))
    _raise(st, "hd_ckpt_store")
    return out


def ckpt_load(kept: Checkpoint, dtype=None, out=None):
    """The activations a checkpoint stands for, [N, D] (float32 unless ``dtype`` or
    ``out`` says bfloat16)."""
    N, D, image = kept.N, kept.D, kept.image
    if out is None:
        torch = _torch()
        dtype = dtype or torch.float32
        dt, ld = (_codes or _float_codes()).get(dtype), D
        if dt is None:
            raise TypeError("dtype must be float32 or bfloat16")
        out = torch.empty(N, D, dtype=dtype, device=image.device)
    else:
        _, _, ld, dt, index = _rows(out, "out")
        if out.shape != (N, D) or index != image.get_device():
            raise ValueError("out must be [N, D] on the checkpoint's device")
        if dtype is not None and out.dtype != dtype:
            raise TypeError("out has another dtype")
    st = lib().hd_ckpt_load(image.data_ptr(), out.data_ptr(), ld, N, D, dt,
                            _raw_stream(image.get_device()))
    _raise(st, "hd_ckpt_load")
    return out


def ckpt_class_grad(dS, kept: Checkpoint, out=None, accumulate: bool = False):
    """The class vectors' gradient dC[K, D] float32 = dS^T H from the scores' gradient
    ``dS`` [N, K] (float32 or bfloat16) and the checkpoint of the encodings H.
    ``out`` receives it, or with ``accumulate`` has it added."""
    torch = _torch()
    N, K, ld, dt, index = _rows(dS, "dS")
    D, image = kept.D, kept.image
    if N != kept.N:
        raise ValueError("shape mismatch")
    if image.get_device() != index:
        raise ValueError("dS and the checkpoint must be on one device")
    if out is None:
        if accumulate:
            raise ValueError("accumulate needs out")
        out = torch.empty(K, D, dtype=torch.float32, device=dS.device)
    else:
        _check_dev(out)
        if out.dtype != torch.float32 or out.shape != (K, D) or out.get_device() != index:
            raise ValueError("out must be float32 [K, D] on dS's device")
    need = _need("hd_ckpt_class_grad_workspace_bytes", index, N, D, K, dt)
    ws = torch.empty(need, dtype=torch.uint8, device=dS.device) if need else None
    st = lib().hd_ckpt_class_grad(dS.data_ptr(), ld, image.data_ptr(), out.data_ptr(), N, D, K,
                                  dt, accumulate, ws.data_ptr() if need else None, need,
                                  _raw_stream(index))
    _raise(st, "hd_ckpt_class_grad")
    return out


class ByteWeights:
    """A matrix in 8 bits with a scale for each output, laid out once (opaque device image)."""

    def __init__(self, image, outer: int, inner: int):
        self.image, self.outer, self.inner = image, outer, inner


def _byte_image(outer: int, inner: int, device):
    torch = _torch()
    nbytes = int(lib().hd_byte_bytes(outer, inner))
    return torch.empty(nbytes, dtype=torch.uint8, device=device), nbytes


def byte_pack(codes, scales) -> ByteWeights:
    """8-bit weights from given ``codes`` [outer, inner] int8 and ``scales`` [outer] float32."""
    torch = _torch()
    _check_dev(codes)
    if codes.dtype != torch.int8:
        raise TypeError("codes must be int8")
    if codes.dim() != 2:
        raise ValueError("codes must be a matrix")
    outer, inner = codes.shape
    index = codes.get_device()
    sptr = _vec(scales, "scales", torch.float32, outer, index)
    image, nbytes = _byte_image(outer, inner, codes.device)
    st = lib().hd_byte_pack(codes.data_ptr(), sptr, outer, inner, image.data_ptr(), nbytes,
                            _raw_stream(index))
    _raise(st, "hd_byte_pack")
    return ByteWeights(image, outer, inner)


def byte_quantize(W, inner_rows: bool = False) -> ByteWeights:
    """8-bit weights from numbers: ``W`` [outer, inner] (class hypervectors), or with
    ``inner_rows`` [inner, outer] (base hypervectors B[F, D]); float32 or bfloat16."""
    outer, inner, ld, dt, index = _rows(W, "W")
    if inner_rows:
        outer, inner = inner, outer
    image, nbytes = _byte_image(outer, inner, W.device)
    st = lib().hd_byte_quantize(W.data_ptr(), ld, int(inner_rows), outer, inner, dt,
                                image.data_ptr(), nbytes, _raw_stream(index))
    _raise(st, "hd_byte_quantize")
    return ByteWeights(image, outer, inner)


def byte_unpack(w: ByteWeights):
    """The weights that ``w`` stands for: [outer, inner] float32."""
    torch = _torch()
    W = torch.empty((w.outer, w.inner), dtype=torch.float32, device=w.image.device)
    st = lib().hd_byte_unpack(w.image.data_ptr(), W.data_ptr(), w.outer, w.inner,
                              _raw_stream(w.image.get_device()))
    _raise(st, "hd_byte_unpack")
    return W


def byte_rows(X):
    """Rows of ``X`` [N, inner] (float32 or bfloat16) as codes [N, inner] int8 and scales [N]
    float32: what ``byte_product`` does to them, for rows that several products take."""
    torch = _torch()
    N, inner, ld, dt, index = _rows(X, "X")
    codes = torch.empty(N, inner, dtype=torch.int8, device=X.device)
    scales = torch.empty(N, dtype=torch.float32, device=X.device)
    st = lib().hd_byte_rows(X.data_ptr(), ld, N, inner, dt, codes.data_ptr(), scales.data_ptr(),
                            _raw_stream(index))
    _raise(st, "hd_byte_rows")
    return codes, scales


def byte_product(X, w: ByteWeights, act: str = "identity", dtype=None, out=None, row_scales=None):
    """Y[N, outer] = act(X w^T) in 8-bit integers. ``X`` [N, inner] float32 or bfloat16 is taken
    to codes with a scale for each row; int8 ``X`` holds codes, with ``row_scales`` [N] float32
    (None: 1). ``dtype`` of Y defaults to X's (float32 for int8). ``act`` "hardsign" encodes."""
    torch = _torch()
    if X.dtype == torch.int8:
        index = X.get_device()
        if index < 0:
            raise ValueError("tensors must be on the GPU")
        if X.dim() != 2:
            raise ValueError("X must be a matrix")
        N, inner = X.shape
        ldx, step = X.stride()
        if step != 1 and inner > 1:
            raise ValueError("X must have contiguous rows")
        if ldx < inner:
            if N > 1:
                raise ValueError("X must not have overlapping rows")
            ldx = inner
        x_dt = HD_I8
    else:
        N, inner, ldx, x_dt, index = _rows(X, "X")
        if row_scales is not None:
            raise ValueError("row_scales are for X in int8")
    sptr = _vec(row_scales, "row_scales", torch.float32, N, index) if row_scales is not None else None
    outer, image = w.outer, w.image
    if inner != w.inner:
        raise ValueError("shape mismatch")
    if image.get_device() != index:
        raise ValueError("X and the weights must be on one device")
    if out is None:
        if dtype is None:
            dtype = torch.float32 if x_dt == HD_I8 else X.dtype
        y_dt = (_codes or _float_codes()).get(dtype)
        if y_dt is None:
            raise TypeError("dtype must be float32 or bfloat16")
        out, ldy = torch.empty(N, outer, dtype=dtype, device=X.device), outer
    else:
        _, _, ldy, y_dt, out_index = _rows(out, "out")
        if out_index != index or out.shape != (N, outer):
            raise ValueError("out must be [N, outer] on X's device")
        if dtype is not None and out.dtype != dtype:
            raise TypeError("out has another dtype")
    need = _need("hd_byte_workspace_bytes", index, N, outer, inner, x_dt)
    ws = torch.empty(need, dtype=torch.uint8, device=X.device) if need else None
    st = lib().hd_byte_product(X.data_ptr(), ldx, sptr, image.data_ptr(), out.data_ptr(), ldy, N,
                               outer, inner, x_dt, y_dt, ACTS[act], _ptr(ws), need,
                               _raw_stream(index))
    _raise(st, "hd_byte_product")
    return out


class ClassLoss(NamedTuple):
    """What ``class_loss`` gives for N rows: ``loss`` [N] and ``stats`` [N, 2] (the largest score m,
    and log sum exp scale (s - m)). They are parts of one allocation."""
    loss: object
    stats: object


def _class_args(H, C, y, mask):
    torch = _torch()
    N, D, ldh, dt, index = _rows(H, "H")
    K, D2, ldc, c_dt, c_index = _rows(C, "C")
    if c_dt != dt:
        raise TypeError("H and C must share a dtype")
    if D2 != D:
        raise ValueError("shape mismatch")
    if c_index != index:
        raise ValueError("H and C must be on one device")
    yptr = _vec(y, "y", torch.int32, N, index)
    mptr = None
    if mask is not None:
        if mask.dtype not in (torch.bool, torch.uint8):
            raise TypeError("mask must be bool or uint8")
        mptr = _vec(mask, "mask", mask.dtype, K, index)
    return N, D, K, ldh, ldc, dt, index, yptr, mptr


def class_loss(H, C, y, scale: float = 1.0, mask=None) -> ClassLoss:
    """Softmax cross entropy of the classes ``y`` [N] int32 (outside [0, K): none asked for, loss 0)
    under softmax(scale * H C^T), for encodings ``H`` [N, D] and class vectors ``C`` [K, D], both
    float32 or both bfloat16, without the scores being kept. ``mask`` [K]: classes that are False
    take no part. Nothing here is recorded by autograd: gradients are ``class_loss_grad``'s."""
    torch = _torch()
    N, D, K, ldh, ldc, dt, index, yptr, mptr = _class_args(H, C, y, mask)
    buf = torch.empty(3 * N, dtype=torch.float32, device=H.device)
    at = buf.data_ptr()  # stats, loss
    need = _need("hd_class_loss_workspace_bytes", index, N, D, K, dt)
    ws = torch.empty(need, dtype=torch.uint8, device=H.device) if need else None
    st = lib().hd_class_loss(H.data_ptr(), ldh, C.data_ptr(), ldc, mptr, yptr, scale, at + 8 * N,
                             at, N, D, K, dt, _ptr(ws), need, _raw_stream(index))
    _raise(st, "hd_class_loss")
    stats, loss = buf.split_with_sizes((2 * N, N))
    return ClassLoss(loss, stats.view(N, 2))


def class_loss_grad(H, C, y, cl: ClassLoss, g_loss, scale: float = 1.0, mask=None,
                    wrt: str = "both"):
    """The gradient of sum(g_loss * loss) (``g_loss`` [N] float32): (dH [N, D], dC [K, D]) of H's
    dtype; ``cl`` is what ``class_loss`` gave for the same H, C, y, scale and mask. ``wrt``: "both",
    "encodings" or "classes"; what is not asked for is None and costs nothing."""
    torch = _torch()
    if wrt not in ("both", "encodings", "classes"):
        raise ValueError('wrt must be "both", "encodings" or "classes"')
    N, D, K, ldh, ldc, dt, index, yptr, mptr = _class_args(H, C, y, mask)
    gptr, stats = _vec(g_loss, "g_loss", torch.float32, N, index), cl.stats
    if (stats.shape != (N, 2) or stats.dtype != torch.float32 or not stats.is_contiguous()
            or stats.get_device() != index):
        raise ValueError("stats must be float32 [N, 2] on the encodings' device")
    dH = torch.empty(N, D, dtype=H.dtype, device=H.device) if wrt != "classes" else None
    dC = torch.empty(K, D, dtype=H.dtype, device=H.device) if wrt != "encodings" else None
    need = _need("hd_class_loss_grad_workspace_bytes_of", index, N, D, K, dt, dH is not None,
                 dC is not None)
    ws = torch.empty(need, dtype=torch.uint8, device=H.device) if need else None
    st = lib().hd_class_loss_grad(H.data_ptr(), ldh, C.data_ptr(), ldc, mptr, yptr, scale,
                                  stats.data_ptr(), gptr, _ptr(dH), _ptr(dC), N, D, K, dt,
                                  _ptr(ws), need, _raw_stream(index))
    _raise(st, "hd_class_loss_grad")
    return dH, dC


def dropout(X, p: float, seed: int, step=0, out=None):
    """``X`` [N, D] (float32 or bfloat16) with values dropped with probability ``p`` and the others
    times 1 / (1 - p). Which ones is a function of ``seed`` and ``step`` (64 bits each) and a
    value's place: the same call on the gradient is the backward pass (autograd records none).
    ``step`` may be an int64 tensor of one element on the GPU, which a graph's replays read. ``out``
    may be X itself."""
    torch = _torch()
    N, D, ldx, dt, index = _rows(X, "X")
    at = None
    if isinstance(step, torch.Tensor):
        if step.dtype != torch.int64 or step.numel() != 1:
            raise TypeError("step must be a number or an int64 tensor of one element")
        if step.get_device() != index:
            raise ValueError("step must be on X's device")
        at, step = step.data_ptr(), 0
    if not (0 <= seed < 1 << 64 and 0 <= step < 1 << 64):
        raise ValueError("seed and step must be in [0, 2^64)")
    if out is None:
        out, ldy = torch.empty(N, D, dtype=X.dtype, device=X.device), D
    else:
        _, _, ldy, out_dt, out_index = _rows(out, "out")
        if out.shape != (N, D) or out_dt != dt or out_index != index:
            raise ValueError("out must have X's shape, dtype and device")
    st = lib().hd_dropout(X.data_ptr(), ldx, out.data_ptr(), ldy, N, D, p, seed, step, at, dt,
                          _raw_stream(index))
    _raise(st, "hd_dropout")
    return out
