"""ctypes binding of libattt (include/attt.h), argument marshalling only.

Each function has the name of the C entry point it calls and takes torch
tensors (device memory) plus an optional torch.cuda.Stream; every step of the
computation runs in the library's CUDA kernels.  There is no fallback: if
libattt.so is missing or the device is not a GB300-class part, the call
raises.
"""
from __future__ import annotations

import ctypes
import os
import threading
from typing import Optional, Sequence, Tuple

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libattt.so")
# ATTT_CHECKED=1 selects the checked build (device-side bounds checks)
LIB_CHECKED_PATH = os.path.join(_HERE, "libattt_checked.so")

ATTT_OK = 0
ATTT_ERR_INVALID_ARG = 1
ATTT_ERR_TABLE_FULL = 2
ATTT_ERR_TOKEN_RANGE = 3
ATTT_ERR_TIMEOUT = 4
ATTT_ERR_WORKSPACE = 5
ATTT_ERR_CUDA = 6
ATTT_ERR_UNSUPPORTED = 7
ATTT_ERR_CAPACITY = 8
ATTT_ERR_CHECK = 9
STATUS_NAMES = {
    0: "ATTT_OK", 1: "ATTT_ERR_INVALID_ARG", 2: "ATTT_ERR_TABLE_FULL", 3: "ATTT_ERR_TOKEN_RANGE",
    4: "ATTT_ERR_TIMEOUT", 5: "ATTT_ERR_WORKSPACE", 6: "ATTT_ERR_CUDA", 7: "ATTT_ERR_UNSUPPORTED",
    8: "ATTT_ERR_CAPACITY", 9: "ATTT_ERR_CHECK",
}

_lock = threading.Lock()
_lib = None


class AtttError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = int(code)
        super().__init__(f"{where}: {STATUS_NAMES.get(int(code), code)}")


class EpisodeConfig(ctypes.Structure):
    """attt_episode_config (field order and types as in attt.h)."""
    _fields_ = [("n", ctypes.c_int), ("w_min", ctypes.c_float), ("max_history", ctypes.c_int64),
                ("max_update", ctypes.c_int64), ("din", ctypes.c_int64), ("d", ctypes.c_int64),
                ("V", ctypes.c_int64), ("r", ctypes.c_int), ("scale", ctypes.c_float), ("lr", ctypes.c_float),
                ("grad_steps", ctypes.c_int), ("cadence", ctypes.c_int), ("optimizer", ctypes.c_int),
                ("beta1", ctypes.c_double), ("beta2", ctypes.c_double), ("eps", ctypes.c_double),
                ("weight_decay", ctypes.c_double)]


class BatchConfig(ctypes.Structure):
    """attt_batch_config (field order and types as in attt.h)."""
    _fields_ = [("episodes", ctypes.c_int), ("n", ctypes.c_int), ("w_min", ctypes.c_float),
                ("max_history", ctypes.c_int64), ("max_update", ctypes.c_int64), ("din", ctypes.c_int64),
                ("d", ctypes.c_int64), ("V", ctypes.c_int64), ("r", ctypes.c_int), ("scale", ctypes.c_float),
                ("lr", ctypes.c_float), ("grad_steps", ctypes.c_int)]


def load_library(path: Optional[str] = None) -> ctypes.CDLL:
    """Loads libattt.so (raises if it has not been built)."""
    global _lib
    with _lock:
        if _lib is not None:
            return _lib
        p = path or (LIB_CHECKED_PATH if os.environ.get("ATTT_CHECKED") == "1" else LIB_PATH)
        if not os.path.exists(p):
            raise RuntimeError(f"libattt.so not found at {p}; run paper_2607_03441_gb300.build.build()")
        lib = ctypes.CDLL(p)
        P, i64, i32, f32, sz = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int, ctypes.c_float, ctypes.c_size_t
        f64 = ctypes.c_double
        sig = {
            "attt_status_string": (ctypes.c_char_p, [i32]),
            "attt_abi_version": (i32, []),
            "attt_kernel_launches": (ctypes.c_uint64, []),
            "attt_device_status": (i32, [P]),
            "attt_selftest_wait_timeout": (i32, [P]),
            "attt_fault_inject": (i32, [ctypes.c_char_p]),
            "attt_history_create": (i32, [i32, i64, ctypes.POINTER(P)]),
            "attt_history_destroy": (i32, [P]),
            "attt_history_reset": (i32, [P, P]),
            "attt_history_insert": (i32, [P, P, i64, P]),
            "attt_history_length": (i64, [P]),
            "attt_history_ngram": (i32, [P]),
            "attt_history_status": (i32, [P, P]),
            "attt_history_count": (i32, [P, P, i64, P, P]),
            "attt_ngram_weights": (i32, [P, P, i64, f32, P, P]),
            "attt_ce_workspace_bytes": (sz, [i64, i64, i64]),
            "attt_ce_workspace_max_bytes": (sz, [i64, i64, i64]),
            "attt_weighted_ce_fwd_bwd": (i32, [P, P, P, P, i64, i64, i64, P, P, P, P, sz, P]),
            "attt_lora_workspace_bytes": (sz, [i64, i64, i32, P, i32]),
            "attt_lora_grad": (i32, [P, i64, i64, i32, P, P, P, P, i32, f32, P, P, P, sz, P]),
            "attt_lora_step": (i32, [P, P, P, P, i64, i64, i32, f32, P, P, P]),
            "attt_lora_grad_noalloc": (i32, [P, i64, i64, i32, P, P, P, P, i32, f32, P, P, P]),
            "attt_lora_forward_workspace_bytes": (sz, [i64, i64, i64, i32]),
            "attt_lora_input_grad_workspace_bytes": (sz, [i64, i64, i64, i32]),
            "attt_lora_forward": (i32, [P, P, P, P, i64, i64, i64, i32, f32, P, P, sz, P]),
            "attt_lora_input_grad": (i32, [P, P, P, P, i64, i64, i64, i32, f32, P, P, sz, P]),
            "attt_cast_bf16": (i32, [P, P, i64, P]),
            "attt_lora_adamw_step": (i32, [P, P, P, P, P, P, P, P, i64, i64, i32, f32, f64, f64, f64, f64, i32, P,
                                           P, P]),
            "attt_episode_create": (i32, [ctypes.POINTER(EpisodeConfig), P, P, P, P, ctypes.POINTER(P)]),
            "attt_episode_destroy": (i32, [P]),
            "attt_episode_reset": (i32, [P, P]),
            "attt_episode_update": (i32, [P, P, P, i64, P, P, P]),
            "attt_episode_agent_step": (i32, [P, P, P, i64, P, P, ctypes.POINTER(i32), P]),
            "attt_episode_read_adapter": (i32, [P, P, P, P]),
            "attt_episode_drift": (i32, [P, P, i64, P, P, P]),
            "attt_episode_checkpoint_bytes": (sz, [P]),
            "attt_episode_save": (i32, [P, P, sz, P]),
            "attt_episode_load": (i32, [P, P, sz, P]),
            "attt_history_save": (i32, [P, P, P]),
            "attt_history_restore": (i32, [P, P, i64, P]),
            "attt_episode_history": (P, [P]),
            "attt_episode_pending_tokens": (i64, [P]),
            "attt_kl_workspace_bytes": (sz, [i64, i64, i64]),
            "attt_kl_drift": (i32, [P, P, P, i64, i64, i64, P, P, P, sz, P]),
            "attt_lora_muon_workspace_bytes": (sz, [i32, P, P, i32]),
            "attt_lora_muon_step": (i32, [i32, P, P, P, P, P, P, P, P, i32, f32, f32, i32, f32, f32, f32, i32, P, P, P,
                                          sz, P]),
            "attt_layer_norm_forward": (i32, [P, i64, P, P, i64, i64, f32, i32, P, i64, P, P, P]),
            "attt_layer_norm_workspace_bytes": (sz, [i64, i64]),
            "attt_layer_norm_backward": (i32, [P, i64, P, i64, P, P, P, i64, i64, i32, P, i64, P, P, P, sz, P]),
            "attt_logprob_workspace_bytes": (sz, [i64, i64, i64, i32]),
            "attt_logprob_grad_workspace_bytes": (sz, [i64, i64, i64]),
            "attt_logprob_forward": (i32, [P, i64, P, P, i64, i64, i64, f32, i32, P, P, P, P, P, P, sz, P]),
            "attt_logprob_input_grad": (i32, [P, i64, P, P, P, P, P, P, i64, i64, i64, f32, P, P, sz, P]),
            "attt_batch_create": (i32, [ctypes.POINTER(BatchConfig), P, P, P, P, ctypes.POINTER(P)]),
            "attt_batch_destroy": (i32, [P]),
            "attt_batch_reset": (i32, [P, i32, P]),
            "attt_batch_update": (i32, [P, P, P, P, P, P, P]),
            "attt_batch_read_adapter": (i32, [P, i32, P, P, P]),
            "attt_batch_history": (P, [P, i32]),
            "attt_wordsets_create": (i32, [i32, i64, ctypes.POINTER(P)]),
            "attt_wordsets_destroy": (i32, [P]),
            "attt_wordsets_reset": (i32, [P, P]),
            "attt_repetition": (i32, [P, P, i64, f32, P, P, P, P]),
            "attt_wordsets_updates": (i32, [P]),
            "attt_wordsets_status": (i32, [P, P]),
        }
        for name, (res, args) in sig.items():
            fn = getattr(lib, name)
            fn.restype = res
            fn.argtypes = args
        _lib = lib
        return lib


def _check(code: int, where: str) -> None:
    if code != ATTT_OK:
        raise AtttError(code, where)


# torch's own way to a stream's handle; not public, so it may be missing
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_raw_device = getattr(torch._C, "_cuda_getDevice", None)


def _stream(stream: Optional[torch.cuda.Stream]) -> int:
    """The cudaStream_t of `stream`, or of the current stream (asked for by its
    handle where torch has that: building a torch Stream object takes longer
    than a launch)."""
    if stream is not None:
        return stream.cuda_stream
    if _raw_stream is None or _raw_device is None or not torch.cuda.is_initialized():
        return torch.cuda.current_stream().cuda_stream
    return _raw_stream(_raw_device())


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    if t is None:
        return None
    if not t.is_cuda:
        raise ValueError("expected a CUDA tensor")
    if not t.is_contiguous():
        raise ValueError("expected a contiguous tensor")
    return t.data_ptr()


def _bf16(t: torch.Tensor) -> int:
    if t.dtype != torch.bfloat16:
        raise ValueError(f"expected bfloat16, got {t.dtype}")
    return _ptr(t)


def _expect(t: Optional[torch.Tensor], shape, dtype, name: str) -> None:
    """Raises ValueError unless t (when given) has this shape (a tuple of ints)
    and dtype: the C ABI takes sizes on trust, so a smaller tensor would be read
    or written past its end."""
    if t is None:
        return
    if t.shape != shape:
        raise ValueError(f"{name}: expected shape {tuple(shape)}, got {tuple(t.shape)}")
    if t.dtype != dtype:
        raise ValueError(f"{name}: expected {dtype}, got {t.dtype}")


def _rows_ptr(t: torch.Tensor, name: str) -> Tuple[int, int]:
    """(address, row pitch in elements) of a 2-D CUDA tensor whose rows are
    contiguous and do not overlap (a slice of a wider tensor's columns, say)."""
    if not t.is_cuda:
        raise ValueError("expected a CUDA tensor")
    rows, cols = t.shape
    if t.is_contiguous():
        return t.data_ptr(), max(cols, 1)
    ld = t.stride(0) if rows > 1 else max(cols, 1)
    if (cols > 1 and t.stride(1) != 1) or ld < cols:
        raise ValueError(f"{name}: expected rows that are contiguous and do not overlap")
    return t.data_ptr(), ld


def _rows_of(t: torch.Tensor, shape, dtype, name: str) -> Tuple[int, int]:
    """_expect and _rows_ptr in one (each call of Python costs a tenth of a launch)."""
    if t.shape != shape or t.dtype != dtype:
        _expect(t, shape, dtype, name)
    return _rows_ptr(t, name)


_F32 = torch.float32


def _f32_of(t: Optional[torch.Tensor], shape, name: str) -> Optional[int]:
    """_expect (float32) and _ptr in one."""
    if t is None:
        return None
    if t.shape != shape or t.dtype != _F32:
        _expect(t, shape, _F32, name)
    return t.data_ptr() if t.is_cuda and t.is_contiguous() else _ptr(t)


def _empty(*size, dtype, device, stream) -> torch.Tensor:
    """A new tensor that a call on `stream` (None: the current one) writes.  Of another
    stream's memory: what the caller's stream frees or takes next is not what the
    call still waits to use, a workspace among it; a result that the caller's stream
    has read is not given away before that."""
    if stream is None:
        return torch.empty(*size, dtype=dtype, device=device)
    with torch.cuda.stream(stream):
        t = torch.empty(*size, dtype=dtype, device=device)
    t.record_stream(torch.cuda.current_stream())
    return t


def _out_f32(t: Optional[torch.Tensor], shape, name: str, dev, stream) -> torch.Tensor:
    """`t`, checked, or a new float32 tensor of that shape."""
    if t is None:
        return _empty(shape, dtype=torch.float32, device=dev, stream=stream)
    _expect(t, shape, torch.float32, name)
    return t


# --------------------------------------------------------------------------
# status
# --------------------------------------------------------------------------

def attt_status_string(code: int) -> str:
    return load_library().attt_status_string(int(code)).decode()


def attt_abi_version() -> int:
    return int(load_library().attt_abi_version())


def attt_kernel_launches() -> int:
    """Kernels launched by libattt in this process so far."""
    return int(load_library().attt_kernel_launches())


def attt_selftest_wait_timeout(stream=None) -> None:
    """Launches the bounded-wait self-test (a wait that runs out after 2 s)."""
    _check((_lib or load_library()).attt_selftest_wait_timeout(_stream(stream)), "attt_selftest_wait_timeout")


def attt_fault_inject(site: str) -> None:
    """One pending host-side fault: "alloc", "table_full" or "none"."""
    _check((_lib or load_library()).attt_fault_inject(site.encode()), "attt_fault_inject")


def attt_device_status(stream=None) -> int:
    """Synchronises and returns (and clears) the device-side status word."""
    return int(load_library().attt_device_status(_stream(stream)))


# --------------------------------------------------------------------------
# history
# --------------------------------------------------------------------------

class History:
    """Owning handle of an attt_history (destroyed with the object)."""

    def __init__(self, n: int, max_tokens: int):
        self._lib = load_library()
        h = ctypes.c_void_p()
        _check(self._lib.attt_history_create(int(n), int(max_tokens), ctypes.byref(h)), "attt_history_create")
        self.handle = h
        self.n = int(n)
        self.max_tokens = int(max_tokens)
        self._owned = True

    @classmethod
    def _view(cls, handle: int, n: int, max_tokens: int, owner) -> "History":
        """Non-owning handle of a history that another object owns."""
        self = cls.__new__(cls)
        self._lib = load_library()
        self.handle = ctypes.c_void_p(handle)
        self.n = int(n)
        self.max_tokens = int(max_tokens)
        self._owned = False
        self._owner = owner
        return self

    def close(self) -> None:
        if getattr(self, "handle", None):
            if self._owned:
                self._lib.attt_history_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def __len__(self) -> int:
        return int(self._lib.attt_history_length(self.handle))


def attt_history_create(n: int, max_tokens: int) -> History:
    return History(n, max_tokens)


def attt_history_destroy(h: History) -> None:
    h.close()


def attt_history_reset(h: History, stream=None) -> None:
    _check((_lib or load_library()).attt_history_reset(h.handle, _stream(stream)), "attt_history_reset")


def attt_history_insert(h: History, tokens: torch.Tensor, stream=None) -> None:
    if tokens.dtype != torch.int32:
        raise ValueError("tokens must be int32")
    _check((_lib or load_library()).attt_history_insert(h.handle, _ptr(tokens), tokens.numel(), _stream(stream)),
           "attt_history_insert")


def attt_history_save(h: History, stream=None):
    """The history's token stream (int32 numpy array), for a checkpoint."""
    import numpy as np
    n = len(h)
    out = np.empty(n, dtype=np.int32)
    _check(load_library().attt_history_save(h.handle, out.ctypes.data_as(ctypes.c_void_p) if n else None,
                                            _stream(stream)), "attt_history_save")
    return out


def attt_history_restore(h: History, tokens, stream=None) -> None:
    """Makes h the history of `tokens` (int32 numpy array), counts rebuilt exactly."""
    import numpy as np
    t = np.ascontiguousarray(tokens, dtype=np.int32)
    _check(load_library().attt_history_restore(h.handle, t.ctypes.data_as(ctypes.c_void_p) if t.size else None,
                                               t.size, _stream(stream)), "attt_history_restore")


def attt_history_length(h: History) -> int:
    return int(load_library().attt_history_length(h.handle))


def attt_history_status(h: History, stream=None) -> int:
    return int(load_library().attt_history_status(h.handle, _stream(stream)))


def attt_history_count(h: History, ngrams: torch.Tensor, out: Optional[torch.Tensor] = None,
                       stream=None) -> torch.Tensor:
    """count(g, H) for each row g of an int32 [m, n] tensor -> int32 [m]."""
    if ngrams.dtype != torch.int32 or ngrams.dim() != 2 or ngrams.shape[1] != h.n:
        raise ValueError("ngrams must be int32 [m, n]")
    m = ngrams.shape[0]
    _expect(out, (m,), torch.int32, "out")
    if out is None:
        out = _empty(m, dtype=torch.int32, device=ngrams.device, stream=stream)
    _check((_lib or load_library()).attt_history_count(h.handle, _ptr(ngrams), m, _ptr(out), _stream(stream)),
           "attt_history_count")
    return out


def attt_ngram_weights(h: History, tokens: torch.Tensor, w_min: float = 0.05,
                       out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """Eq. 8 / Eq. 9 weights (fp32 [L]) of the update `tokens` (int32 [L])."""
    if tokens.dtype != torch.int32:
        raise ValueError("tokens must be int32")
    L = tokens.numel()
    _expect(out, (L,), torch.float32, "out")
    if out is None:
        out = _empty(L, dtype=torch.float32, device=tokens.device, stream=stream)
    _check((_lib or load_library()).attt_ngram_weights(
        h.handle, _ptr(tokens), L, float(w_min), _ptr(out), _stream(stream)), "attt_ngram_weights")
    return out


# --------------------------------------------------------------------------
# Eq. 10
# --------------------------------------------------------------------------

def attt_ce_workspace_bytes(L: int, d: int, V: int) -> int:
    return int(load_library().attt_ce_workspace_bytes(int(L), int(d), int(V)))


def attt_ce_workspace_max_bytes(Lmax: int, d: int, V: int) -> int:
    """One workspace for every update length 1..Lmax (host-only)."""
    return int(load_library().attt_ce_workspace_max_bytes(int(Lmax), int(d), int(V)))


def attt_weighted_ce_fwd_bwd(h: torch.Tensor, W: torch.Tensor, tgt: torch.Tensor, w: torch.Tensor,
                             loss: Optional[torch.Tensor] = None, dh: Optional[torch.Tensor] = None,
                             lse: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
                             stream=None):
    """Eq. 10 loss (fp32 [1]), dh (fp32 [L, d]) and optionally lse (fp32 [L])."""
    L, d = h.shape
    V = W.shape[0]
    dev = h.device
    _expect(W, (V, d), torch.bfloat16, "W")
    _expect(tgt, (L,), torch.int32, "tgt")
    _expect(w, (L,), torch.float32, "w")
    _expect(dh, (L, d), torch.float32, "dh")
    _expect(lse, (L,), torch.float32, "lse")
    if loss is not None and (loss.numel() < 1 or loss.dtype != torch.float32):
        raise ValueError("loss: expected a float32 tensor of at least one element")
    if loss is None:
        loss = _empty(1, dtype=torch.float32, device=dev, stream=stream)
    if dh is None:
        dh = _empty(L, d, dtype=torch.float32, device=dev, stream=stream)
    if workspace is None:
        workspace = _empty(attt_ce_workspace_bytes(L, d, V), dtype=torch.uint8, device=dev, stream=stream)
    if tgt.dtype != torch.int32 or w.dtype != torch.float32:
        raise ValueError("tgt must be int32 and w float32")
    _check((_lib or load_library()).attt_weighted_ce_fwd_bwd(
        _bf16(h), _bf16(W), _ptr(tgt), _ptr(w), L, d, V, _ptr(loss), _ptr(dh), _ptr(lse),
        _ptr(workspace), workspace.numel(), _stream(stream)), "attt_weighted_ce_fwd_bwd")
    return loss, dh, lse


# --------------------------------------------------------------------------
# LoRA
# --------------------------------------------------------------------------

def attt_lora_workspace_bytes(L: int, din: int, douts: Sequence[int], r: int) -> int:
    arr = (ctypes.c_int64 * len(douts))(*[int(x) for x in douts])
    return int(load_library().attt_lora_workspace_bytes(int(L), int(din), len(douts), arr, int(r)))


def _lora_check(x: torch.Tensor, dys, As, Bs, dAs, dBs):
    """Shapes of one attt_lora_grad group: (L, din, r, douts).  Raises
    ValueError before any launch unless every list has one entry per
    projection and every tensor has its shape and dtype (the C ABI takes the
    sizes on trust, so a smaller or wider-typed tensor would be read or written
    past its end)."""
    if x.dim() != 2:
        raise ValueError(f"x: expected a 2-D [L, din] tensor, got shape {tuple(x.shape)}")
    L, din = x.shape
    k = len(dys)
    if k < 1:
        raise ValueError("at least one projection (dys) is required")
    if not (len(As) == len(Bs) == k) or (dAs is not None and len(dAs) != k) or (dBs is not None and len(dBs) != k):
        raise ValueError("dys, As, Bs (and dAs, dBs) must have one entry per projection")
    bf16, f32 = torch.bfloat16, torch.float32
    _expect(x, (L, din), bf16, "x")
    if As[0].dim() != 2:
        raise ValueError(f"As[0]: expected a 2-D [din, r] tensor, got shape {tuple(As[0].shape)}")
    r = As[0].shape[1]
    a_shape = (din, r)
    douts = []
    for p in range(k):
        dy, A, B = dys[p], As[p], Bs[p]
        if dy.dim() != 2:
            raise ValueError(f"dys[{p}]: expected a 2-D [L, dout] tensor, got shape {tuple(dy.shape)}")
        rows, dout = dy.shape
        douts.append(dout)
        # one test for the usual case; the named checks say what is wrong
        if rows != L or dy.dtype != bf16 or A.shape != a_shape or A.dtype != bf16 or B.shape != (r, dout) \
                or B.dtype != bf16:
            _expect(dy, (L, dout), bf16, f"dys[{p}]")
            _expect(A, a_shape, bf16, f"As[{p}]")
            _expect(B, (r, dout), bf16, f"Bs[{p}]")
        if dAs is not None and dAs[p] is not None and (dAs[p].shape != a_shape or dAs[p].dtype != f32):
            _expect(dAs[p], a_shape, f32, f"dAs[{p}]")
        if dBs is not None and dBs[p] is not None and (dBs[p].shape != (r, dout) or dBs[p].dtype != f32):
            _expect(dBs[p], (r, dout), f32, f"dBs[{p}]")
    return L, din, r, douts


def _lora_arrays(dys, douts, As, Bs, dAs, dBs):
    """The C call's six per-projection arrays as one buffer: (the buffer, which
    must outlive the call, and the addresses of dy, dout, A, B, dA, dB)."""
    k = len(dys)
    vals = [_ptr(t) or 0 for t in dys]
    vals += douts
    for ts in (As, Bs, dAs, dBs):
        vals += [_ptr(t) or 0 for t in ts]
    buf = (ctypes.c_int64 * (6 * k))(*vals)
    base = ctypes.addressof(buf)
    return buf, [base + 8 * k * i for i in range(6)]


def attt_lora_grad(x: torch.Tensor, dys: Sequence[torch.Tensor], As: Sequence[torch.Tensor],
                   Bs: Sequence[torch.Tensor], scale: float, dAs: Optional[Sequence[torch.Tensor]] = None,
                   dBs: Optional[Sequence[torch.Tensor]] = None, workspace: Optional[torch.Tensor] = None,
                   stream=None):
    """Adapter gradients for projections sharing the input x.  Returns (dAs, dBs)."""
    L, din, r, douts = _lora_check(x, dys, As, Bs, dAs, dBs)
    k = len(dys)
    dev = x.device
    if dAs is None:
        dAs = [_empty(din, r, dtype=torch.float32, device=dev, stream=stream) for _ in range(k)]
    if dBs is None:
        dBs = [_empty(r, do, dtype=torch.float32, device=dev, stream=stream) for do in douts]
    if workspace is None:
        workspace = _empty(attt_lora_workspace_bytes(L, din, douts, r), dtype=torch.uint8, device=dev, stream=stream)
    buf, (p_dy, p_dout, p_A, p_B, p_dA, p_dB) = _lora_arrays(dys, douts, As, Bs, dAs, dBs)
    _check((_lib or load_library()).attt_lora_grad(
        _bf16(x), L, din, k, p_dy, p_dout, p_A, p_B, r, float(scale), p_dA, p_dB, _ptr(workspace), workspace.numel(),
        _stream(stream)), "attt_lora_grad")
    return dAs, dBs


LORA_NOALLOC_SCRATCH_BYTES = 16 << 20


def attt_lora_grad_noalloc(x: torch.Tensor, dys: Sequence[torch.Tensor], As: Sequence[torch.Tensor],
                           Bs: Sequence[torch.Tensor], scale: float, dAs: Sequence[torch.Tensor],
                           dBs: Sequence[torch.Tensor], stream=None):
    """attt_lora_grad without a workspace: the library uses its own static
    16 MiB device scratch and allocates nothing.  The caller passes the output
    tensors, which are checked like every other argument before the call.
    Returns (dAs, dBs)."""
    if dAs is None or dBs is None:
        raise ValueError("attt_lora_grad_noalloc: the caller passes the output tensors dAs and dBs")
    L, din, r, douts = _lora_check(x, dys, As, Bs, dAs, dBs)
    k = len(dys)
    buf, (p_dy, p_dout, p_A, p_B, p_dA, p_dB) = _lora_arrays(dys, douts, As, Bs, dAs, dBs)
    _check((_lib or load_library()).attt_lora_grad_noalloc(
        _bf16(x), L, din, k, p_dy, p_dout, p_A, p_B, r, float(scale), p_dA, p_dB, _stream(stream)),
        "attt_lora_grad_noalloc")
    return dAs, dBs


def attt_lora_step(A32: torch.Tensor, B32: torch.Tensor, dA: torch.Tensor, dB: torch.Tensor, lr: float,
                   A16: Optional[torch.Tensor] = None, B16: Optional[torch.Tensor] = None, stream=None) -> None:
    """In-place SGD step on the fp32 masters and bf16 refresh (Eq. 2)."""
    din, r = A32.shape
    dout = B32.shape[1]
    _expect(A32, (din, r), torch.float32, "A32")
    _expect(B32, (r, dout), torch.float32, "B32")
    _expect(dA, (din, r), torch.float32, "dA")
    _expect(dB, (r, dout), torch.float32, "dB")
    _expect(A16, (din, r), torch.bfloat16, "A16")
    _expect(B16, (r, dout), torch.bfloat16, "B16")
    _check((_lib or load_library()).attt_lora_step(
        _ptr(A32), _ptr(B32), _ptr(dA), _ptr(dB), din, dout, r, float(lr),
        _bf16(A16) if A16 is not None else None, _bf16(B16) if B16 is not None else None, _stream(stream)),
        "attt_lora_step")


# --------------------------------------------------------------------------
# the adapted projection of a chained update
# --------------------------------------------------------------------------

def attt_lora_forward_workspace_bytes(L: int, din: int, dout: int, r: int) -> int:
    return int(load_library().attt_lora_forward_workspace_bytes(int(L), int(din), int(dout), int(r)))


def attt_lora_input_grad_workspace_bytes(L: int, din: int, dout: int, r: int) -> int:
    return int(load_library().attt_lora_input_grad_workspace_bytes(int(L), int(din), int(dout), int(r)))


def attt_lora_forward(x: torch.Tensor, W0: torch.Tensor, A: torch.Tensor, B: torch.Tensor, scale: float,
                      h: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
                      stream=None) -> torch.Tensor:
    """h = x W0 + s (x A) B (bf16).  Returns h."""
    L, din = x.shape
    dout = W0.shape[1]
    r = A.shape[1]
    _expect(W0, (din, dout), torch.bfloat16, "W0")
    _expect(A, (din, r), torch.bfloat16, "A")
    _expect(B, (r, dout), torch.bfloat16, "B")
    _expect(h, (L, dout), torch.bfloat16, "h")
    if h is None:
        h = _empty(L, dout, dtype=torch.bfloat16, device=x.device, stream=stream)
    if workspace is None:
        workspace = _empty(attt_lora_forward_workspace_bytes(L, din, dout, r), dtype=torch.uint8,
                           device=x.device, stream=stream)
    _check((_lib or load_library()).attt_lora_forward(
        _bf16(x), _bf16(W0), _bf16(A), _bf16(B), L, din, dout, int(r), float(scale), _bf16(h), _ptr(workspace),
        workspace.numel(), _stream(stream)), "attt_lora_forward")
    return h


def attt_lora_input_grad(dy: torch.Tensor, W0: torch.Tensor, A: torch.Tensor, B: torch.Tensor, scale: float,
                         dx: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
                         stream=None) -> torch.Tensor:
    """dx = dy W0^T + s (dy B^T) A^T (fp32).  Returns dx."""
    L, dout = dy.shape
    din = W0.shape[0]
    r = A.shape[1]
    _expect(W0, (din, dout), torch.bfloat16, "W0")
    _expect(A, (din, r), torch.bfloat16, "A")
    _expect(B, (r, dout), torch.bfloat16, "B")
    _expect(dx, (L, din), torch.float32, "dx")
    if dx is None:
        dx = _empty(L, din, dtype=torch.float32, device=dy.device, stream=stream)
    if workspace is None:
        workspace = _empty(attt_lora_input_grad_workspace_bytes(L, din, dout, r), dtype=torch.uint8,
                           device=dy.device, stream=stream)
    _check((_lib or load_library()).attt_lora_input_grad(
        _bf16(dy), _bf16(W0), _bf16(A), _bf16(B), L, din, dout, int(r), float(scale), _ptr(dx), _ptr(workspace),
        workspace.numel(), _stream(stream)), "attt_lora_input_grad")
    return dx


def attt_cast_bf16(src: torch.Tensor, dst: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """dst = bf16(src) (round to nearest even).  Returns dst."""
    if src.dtype != torch.float32:
        raise ValueError(f"expected float32, got {src.dtype}")
    if dst is None:
        dst = _empty(src.shape, dtype=torch.bfloat16, device=src.device, stream=stream)
    if dst.numel() != src.numel():
        raise ValueError(f"dst: expected {src.numel()} elements, got {dst.numel()}")
    _check((_lib or load_library()).attt_cast_bf16(_ptr(src), _bf16(dst), src.numel(), _stream(stream)),
           "attt_cast_bf16")
    return dst


# --------------------------------------------------------------------------
# the episode (Algorithm 1 with the Sec. 4 / Appendix C schedule)
# --------------------------------------------------------------------------

class Episode:
    """Owning handle of an attt_episode.

    W0 (bf16 [din, d]) and Wlm (bf16 [V, d]) are borrowed by the library: this
    object keeps references to them so they outlive the episode.  A0 / B0
    (fp32) are the adapter's initial value, restored by reset().
    """

    def __init__(self, W0: torch.Tensor, Wlm: torch.Tensor, A0: torch.Tensor, B0: torch.Tensor, *, n: int,
                 max_history: int, max_update: int, scale: float, lr: float, w_min: float = 0.05,
                 grad_steps: int = 2, cadence: int = 5, optimizer: str = "sgd", betas=(0.9, 0.999),
                 eps: float = 1e-8, weight_decay: float = 0.01):
        self._lib = load_library()
        din, d = W0.shape
        V = Wlm.shape[0]
        r = A0.shape[1]
        if Wlm.shape[1] != d or A0.shape[0] != din or tuple(B0.shape) != (r, d):
            raise ValueError("shape mismatch between W0, Wlm, A0, B0")
        if A0.dtype != torch.float32 or B0.dtype != torch.float32:
            raise ValueError("A0 and B0 must be float32")
        self.cfg = EpisodeConfig(n=int(n), w_min=float(w_min), max_history=int(max_history),
                                 max_update=int(max_update), din=int(din), d=int(d), V=int(V), r=int(r),
                                 scale=float(scale), lr=float(lr), grad_steps=int(grad_steps),
                                 cadence=int(cadence), optimizer={"sgd": 0, "adamw": 1}[optimizer],
                                 beta1=float(betas[0]), beta2=float(betas[1]), eps=float(eps),
                                 weight_decay=float(weight_decay))
        e = ctypes.c_void_p()
        _check(self._lib.attt_episode_create(ctypes.byref(self.cfg), _bf16(W0), _bf16(Wlm), _ptr(A0), _ptr(B0),
                                             ctypes.byref(e)), "attt_episode_create")
        self.handle = e
        self._keep = (W0, Wlm)
        self.device = W0.device

    def close(self) -> None:
        if getattr(self, "handle", None):
            self._lib.attt_episode_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _out(self, losses, dx, L):
        c = self.cfg
        if losses is not None and (losses.dtype != torch.float32 or losses.numel() < c.grad_steps):
            raise ValueError("losses must be float32 with grad_steps entries")
        if dx is not None and (dx.dtype != torch.float32 or dx.numel() < c.grad_steps * L * c.din):
            raise ValueError("dx must be float32 [grad_steps, L, din]")
        return _ptr(losses), _ptr(dx)

    def update(self, tokens: torch.Tensor, x: torch.Tensor, losses: Optional[torch.Tensor] = None,
               dx: Optional[torch.Tensor] = None, stream=None) -> None:
        """One update on `tokens` (int32 [L]) with projection inputs `x` (bf16 [L, din])."""
        if tokens.dtype != torch.int32:
            raise ValueError("tokens must be int32")
        L = tokens.numel()
        if tuple(x.shape) != (L, self.cfg.din):
            raise ValueError("x must be [L, din]")
        pl, pd = self._out(losses, dx, L)
        _check(self._lib.attt_episode_update(self.handle, _ptr(tokens), _bf16(x), L, pl, pd, _stream(stream)),
               "attt_episode_update")

    def agent_step(self, tokens: torch.Tensor, x: torch.Tensor, losses: Optional[torch.Tensor] = None,
                   dx: Optional[torch.Tensor] = None, stream=None) -> bool:
        """Appends one agent step's text; returns True if it triggered an update."""
        if tokens.dtype != torch.int32:
            raise ValueError("tokens must be int32")
        n = tokens.numel()
        if tuple(x.shape) != (n, self.cfg.din):
            raise ValueError("x must be [len, din]")
        pending = self.pending_tokens()
        pl, pd = self._out(losses, dx, pending + n)
        up = ctypes.c_int(0)
        _check(self._lib.attt_episode_agent_step(self.handle, _ptr(tokens) if n else None,
                                                 _bf16(x) if n else None, n, pl, pd, ctypes.byref(up),
                                                 _stream(stream)), "attt_episode_agent_step")
        return bool(up.value)

    def reset(self, stream=None) -> None:
        _check(self._lib.attt_episode_reset(self.handle, _stream(stream)), "attt_episode_reset")

    def drift(self, x: torch.Tensor, kl: Optional[torch.Tensor] = None, kl_mean: Optional[torch.Tensor] = None,
              stream=None):
        """KL of the adapted from the base next-token distribution on the rows
        of x (bf16 [L, din]).  Returns (kl [L], kl_mean [1])."""
        L = x.shape[0]
        if tuple(x.shape) != (L, self.cfg.din):
            raise ValueError("x must be [L, din]")
        if kl is None:
            kl = _empty(L, dtype=torch.float32, device=x.device, stream=stream)
        if kl_mean is None:
            kl_mean = _empty(1, dtype=torch.float32, device=x.device, stream=stream)
        _check(self._lib.attt_episode_drift(self.handle, _bf16(x), L, _ptr(kl), _ptr(kl_mean), _stream(stream)),
               "attt_episode_drift")
        return kl, kl_mean

    def read_adapter(self, stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
        """(A [din, r], B [r, d]) fp32 copies of the current adapter."""
        c = self.cfg
        A = _empty((c.din, c.r), dtype=torch.float32, device=self.device, stream=stream)
        B = _empty((c.r, c.d), dtype=torch.float32, device=self.device, stream=stream)
        _check(self._lib.attt_episode_read_adapter(self.handle, _ptr(A), _ptr(B), _stream(stream)),
               "attt_episode_read_adapter")
        return A, B

    def history(self) -> History:
        h = self._lib.attt_episode_history(self.handle)
        return History._view(h, self.cfg.n, self.cfg.max_history, self)

    def pending_tokens(self) -> int:
        return int(self._lib.attt_episode_pending_tokens(self.handle))

    def save(self, stream=None) -> bytes:
        """A checkpoint of the episode (adapter, optimizer state, history, pending text)."""
        n = int(self._lib.attt_episode_checkpoint_bytes(self.handle))
        buf = ctypes.create_string_buffer(n)
        _check(self._lib.attt_episode_save(self.handle, buf, n, _stream(stream)), "attt_episode_save")
        return buf.raw

    def load(self, blob: bytes, stream=None) -> None:
        """Restores a checkpoint made by save() of an episode with the same configuration."""
        buf = ctypes.create_string_buffer(bytes(blob), len(blob))
        _check(self._lib.attt_episode_load(self.handle, buf, len(blob), _stream(stream)), "attt_episode_load")


# --------------------------------------------------------------------------
# adapter drift (Sec. 4, Fig. 6)
# --------------------------------------------------------------------------

def attt_kl_workspace_bytes(L: int, d: int, V: int) -> int:
    return int(load_library().attt_kl_workspace_bytes(L, d, V))


def attt_kl_drift(hp: torch.Tensor, hq: torch.Tensor, W: torch.Tensor, kl: Optional[torch.Tensor] = None,
                  kl_mean: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None, stream=None):
    """KL(softmax(h_p W^T) || softmax(h_q W^T)) per row (fp32 [L]) and its
    mean (fp32 [1]).  Returns (kl, kl_mean)."""
    L, d = hp.shape
    V = W.shape[0]
    if tuple(hq.shape) != (L, d) or W.shape[1] != d:
        raise ValueError("shape mismatch")
    _expect(kl, (L,), torch.float32, "kl")
    _expect(kl_mean, (1,), torch.float32, "kl_mean")
    dev = hp.device
    if kl is None:
        kl = _empty(L, dtype=torch.float32, device=dev, stream=stream)
    if kl_mean is None:
        kl_mean = _empty(1, dtype=torch.float32, device=dev, stream=stream)
    if workspace is None:
        workspace = _empty(attt_kl_workspace_bytes(L, d, V), dtype=torch.uint8, device=dev, stream=stream)
    _check((_lib or load_library()).attt_kl_drift(_bf16(hp), _bf16(hq), _bf16(W), L, d, V, _ptr(kl), _ptr(kl_mean),
                                        _ptr(workspace), workspace.numel(), _stream(stream)), "attt_kl_drift")
    return kl, kl_mean


# --------------------------------------------------------------------------
# layer norm
# --------------------------------------------------------------------------

_DTYPES = {torch.bfloat16: 0, torch.float32: 1}


def _norm_check(x: torch.Tensor):
    """(shape, type, the C ABI's name of it) of the rows of a layer norm."""
    shape, dtype = x.shape, x.dtype
    if len(shape) != 2:
        raise ValueError(f"x: expected a 2-D [L, d] tensor, got shape {tuple(shape)}")
    code = _DTYPES.get(dtype)
    if code is None:
        raise ValueError(f"x: expected bfloat16 or float32, got {dtype}")
    return shape, dtype, code


def attt_layer_norm_forward(x: torch.Tensor, gamma: torch.Tensor, beta: Optional[torch.Tensor] = None,
                            eps: float = 1e-5, y: Optional[torch.Tensor] = None,
                            mean: Optional[torch.Tensor] = None, rstd: Optional[torch.Tensor] = None, stream=None):
    """Layer norm of the rows of x (bf16 or fp32 [L, d], rows may lie inside wider
    ones), gamma and beta fp32 [d].  Returns (y, mean, rstd): y of x's type, fp32 [L]
    twice."""
    shape, dtype, code = _norm_check(x)
    L, d = shape
    if y is None:
        y = _empty(L, d, dtype=dtype, device=x.device, stream=stream)
    if mean is None:
        mean = _empty(L, dtype=_F32, device=x.device, stream=stream)
    if rstd is None:
        rstd = _empty(L, dtype=_F32, device=x.device, stream=stream)
    px, x_ld = _rows_ptr(x, "x")
    py, y_ld = _rows_of(y, shape, dtype, "y")
    _check((_lib or load_library()).attt_layer_norm_forward(
        px, x_ld, _f32_of(gamma, (d,), "gamma"), _f32_of(beta, (d,), "beta"), L, d, eps, code, py, y_ld,
        _f32_of(mean, (L,), "mean"), _f32_of(rstd, (L,), "rstd"), _stream(stream)), "attt_layer_norm_forward")
    return y, mean, rstd


def attt_layer_norm_workspace_bytes(L: int, d: int) -> int:
    return int(load_library().attt_layer_norm_workspace_bytes(int(L), int(d)))


def attt_layer_norm_backward(dy: torch.Tensor, x: torch.Tensor, gamma: torch.Tensor, mean: torch.Tensor,
                             rstd: torch.Tensor, dx: Optional[torch.Tensor] = None,
                             dgamma: Optional[torch.Tensor] = None, dbeta: Optional[torch.Tensor] = None,
                             workspace: Optional[torch.Tensor] = None, stream=None, weights: bool = True):
    """Gradients of the layer norm's x, gamma and beta from dy (bf16 or fp32 [L, d]),
    with the forward call's mean and rstd.  Returns (dx, dgamma, dbeta): dx of x's
    type, fp32 [d] twice.  Without `weights` (a frozen norm) gamma's and beta's are
    formed only where a tensor for them is given, else None."""
    shape, dtype, code = _norm_check(x)
    L, d = shape
    if dx is None:
        dx = _empty(L, d, dtype=dtype, device=x.device, stream=stream)
    if dgamma is None and weights:
        dgamma = _empty(d, dtype=_F32, device=x.device, stream=stream)
    if dbeta is None and weights:
        dbeta = _empty(d, dtype=_F32, device=x.device, stream=stream)
    if workspace is None:
        workspace = _empty(attt_layer_norm_workspace_bytes(L, d), dtype=torch.uint8, device=x.device, stream=stream)
    pg, g_ld = _rows_of(dy, shape, dtype, "dy")
    px, x_ld = _rows_ptr(x, "x")
    po, o_ld = _rows_of(dx, shape, dtype, "dx")
    vec, col = (d,), (L,)
    _check((_lib or load_library()).attt_layer_norm_backward(
        pg, g_ld, px, x_ld, _f32_of(gamma, vec, "gamma"), _f32_of(mean, col, "mean"), _f32_of(rstd, col, "rstd"), L, d,
        code, po, o_ld, _f32_of(dgamma, vec, "dgamma"), _f32_of(dbeta, vec, "dbeta"), _ptr(workspace),
        workspace.numel(), _stream(stream)), "attt_layer_norm_backward")
    return dx, dgamma, dbeta


# --------------------------------------------------------------------------
# log probabilities through the LM head
# --------------------------------------------------------------------------

LOGPROB_MAX_TOP = 20


def attt_logprob_workspace_bytes(L: int, d: int, V: int, topk: int = 0) -> int:
    return int(load_library().attt_logprob_workspace_bytes(int(L), int(d), int(V), int(topk)))


def attt_logprob_grad_workspace_bytes(L: int, d: int, V: int) -> int:
    return int(load_library().attt_logprob_grad_workspace_bytes(int(L), int(d), int(V)))


def _logprob_check(h: torch.Tensor, W: torch.Tensor, tgt: Optional[torch.Tensor]):
    if h.dim() != 2 or W.dim() != 2:
        raise ValueError("h and W: expected 2-D tensors")
    L, d = h.shape
    V = W.shape[0]
    _expect(h, (L, d), torch.bfloat16, "h")
    _expect(W, (V, d), torch.bfloat16, "W")
    _expect(tgt, (L,), torch.int32, "tgt")
    return L, d, V


def attt_logprob_forward(h: torch.Tensor, W: torch.Tensor, tgt: Optional[torch.Tensor] = None, topk: int = 0,
                         inv_temp: float = 1.0, logp: Optional[torch.Tensor] = None,
                         entropy: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None,
                         top_logp: Optional[torch.Tensor] = None, top_id: Optional[torch.Tensor] = None,
                         workspace: Optional[torch.Tensor] = None, stream=None):
    """Log probabilities of the tokens `tgt` (int32 [L], -1: none) under softmax(h
    W^T inv_temp), with every row's entropy, logsumexp and `topk` most probable
    tokens.  h (bf16 [L, d]) may be a slice of wider rows.  Returns (logp, entropy,
    lse, top_logp, top_id): fp32 [L] three times (logp None without tgt), fp32 and
    int32 [L, topk]."""
    L, d, V = _logprob_check(h, W, tgt)
    dev = h.device
    topk = int(topk)
    if tgt is None and logp is not None:
        raise ValueError("logp: there are no given tokens")
    if tgt is not None:
        logp = _out_f32(logp, (L,), "logp", dev, stream)
    entropy = _out_f32(entropy, (L,), "entropy", dev, stream)
    lse = _out_f32(lse, (L,), "lse", dev, stream)
    top_logp = _out_f32(top_logp, (L, topk), "top_logp", dev, stream)
    _expect(top_id, (L, topk), torch.int32, "top_id")
    if top_id is None:
        top_id = _empty(L, topk, dtype=torch.int32, device=dev, stream=stream)
    if workspace is None:
        workspace = _empty(attt_logprob_workspace_bytes(L, d, V, topk), dtype=torch.uint8, device=dev, stream=stream)
    ph, ld = _rows_ptr(h, "h")
    _check((_lib or load_library()).attt_logprob_forward(
        ph, ld, _ptr(W), _ptr(tgt), L, d, V, float(inv_temp), topk, _ptr(logp), _ptr(entropy), _ptr(lse),
        _ptr(top_logp) if topk else None, _ptr(top_id) if topk else None, _ptr(workspace), workspace.numel(),
        _stream(stream)), "attt_logprob_forward")
    return logp, entropy, lse, top_logp, top_id


def attt_logprob_input_grad(h: torch.Tensor, W: torch.Tensor, tgt: torch.Tensor, lse: torch.Tensor,
                            glogp: torch.Tensor, entropy: Optional[torch.Tensor] = None,
                            gent: Optional[torch.Tensor] = None, inv_temp: float = 1.0,
                            dh: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
                            stream=None) -> torch.Tensor:
    """The gradient (bf16 [L, d]) of sum_j glogp_j logp_j + gent_j entropy_j with
    respect to h, from the forward call's lse and (with gent) entropy.  Returns dh."""
    L, d, V = _logprob_check(h, W, tgt)
    for t, name in ((lse, "lse"), (glogp, "glogp"), (entropy, "entropy"), (gent, "gent")):
        _expect(t, (L,), torch.float32, name)
    _expect(dh, (L, d), torch.bfloat16, "dh")
    if dh is None:
        dh = _empty(L, d, dtype=torch.bfloat16, device=h.device, stream=stream)
    if workspace is None:
        workspace = _empty(attt_logprob_grad_workspace_bytes(L, d, V), dtype=torch.uint8, device=h.device,
                           stream=stream)
    ph, ld = _rows_ptr(h, "h")
    _check((_lib or load_library()).attt_logprob_input_grad(
        ph, ld, _ptr(W), _ptr(tgt), _ptr(lse), _ptr(entropy), _ptr(glogp), _ptr(gent), L, d, V, float(inv_temp),
        _ptr(dh), _ptr(workspace), workspace.numel(), _stream(stream)), "attt_logprob_input_grad")
    return dh


# --------------------------------------------------------------------------
# update-text repetition (Eq. 6), novelty (Eq. 7), the sequence filter
# --------------------------------------------------------------------------

class WordSets:
    """Owning handle of an attt_wordsets (the episode's update texts)."""

    def __init__(self, max_updates: int, max_bytes: int):
        self._lib = load_library()
        s = ctypes.c_void_p()
        _check(self._lib.attt_wordsets_create(int(max_updates), int(max_bytes), ctypes.byref(s)),
               "attt_wordsets_create")
        self.handle = s

    def close(self) -> None:
        if getattr(self, "handle", None):
            self._lib.attt_wordsets_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def __len__(self) -> int:
        return int(self._lib.attt_wordsets_updates(self.handle))


def attt_wordsets_create(max_updates: int, max_bytes: int) -> WordSets:
    return WordSets(max_updates, max_bytes)


def attt_wordsets_destroy(s: WordSets) -> None:
    s.close()


def attt_wordsets_reset(s: WordSets, stream=None) -> None:
    _check((_lib or load_library()).attt_wordsets_reset(s.handle, _stream(stream)), "attt_wordsets_reset")


def attt_wordsets_updates(s: WordSets) -> int:
    return int(load_library().attt_wordsets_updates(s.handle))


def attt_wordsets_status(s: WordSets, stream=None) -> int:
    return int(load_library().attt_wordsets_status(s.handle, _stream(stream)))


def attt_repetition(s: WordSets, text: torch.Tensor, tau: float = 0.5, out: Optional[torch.Tensor] = None,
                    keep: Optional[torch.Tensor] = None, stream=None):
    """Eq. 6 / Eq. 7 for the update text `text` (uint8 bytes on the device):
    returns (out, keep) with out = float32 [2] (rho, nu) and keep = int32 [1]."""
    if text.dtype != torch.uint8:
        raise ValueError("text must be uint8 bytes")
    _expect(out, (2,), torch.float32, "out")
    _expect(keep, (1,), torch.int32, "keep")
    dev = text.device
    if out is None:
        out = _empty(2, dtype=torch.float32, device=dev, stream=stream)
    if keep is None:
        keep = _empty(1, dtype=torch.int32, device=dev, stream=stream)
    n = text.numel()
    base = _ptr(out)
    _check((_lib or load_library()).attt_repetition(s.handle, _ptr(text) if n else None, n, float(tau), base, base + 4,
                                          _ptr(keep), _stream(stream)), "attt_repetition")
    return out, keep


# --------------------------------------------------------------------------
# a batch of concurrent episodes
# --------------------------------------------------------------------------

class Batch:
    """Owning handle of an attt_batch: E episodes sharing W0 and the LM head
    (borrowed: kept referenced here), each adapter starting at (A0, B0)."""

    def __init__(self, W0: torch.Tensor, Wlm: torch.Tensor, A0: torch.Tensor, B0: torch.Tensor, *, episodes: int,
                 n: int, max_history: int, max_update: int, scale: float, lr: float, w_min: float = 0.05,
                 grad_steps: int = 2):
        self._lib = load_library()
        din, d = W0.shape
        r = A0.shape[1]
        if Wlm.shape[1] != d or A0.shape[0] != din or tuple(B0.shape) != (r, d):
            raise ValueError("shape mismatch between W0, Wlm, A0, B0")
        self.cfg = BatchConfig(episodes=int(episodes), n=int(n), w_min=float(w_min), max_history=int(max_history),
                               max_update=int(max_update), din=int(din), d=int(d), V=int(Wlm.shape[0]), r=int(r),
                               scale=float(scale), lr=float(lr), grad_steps=int(grad_steps))
        b = ctypes.c_void_p()
        _check(self._lib.attt_batch_create(ctypes.byref(self.cfg), _bf16(W0), _bf16(Wlm), _ptr(A0), _ptr(B0),
                                           ctypes.byref(b)), "attt_batch_create")
        self.handle = b
        self._keep = (W0, Wlm)
        self.device = W0.device

    def close(self) -> None:
        if getattr(self, "handle", None):
            self._lib.attt_batch_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def update(self, tokens: torch.Tensor, x: torch.Tensor, lens: Sequence[int],
               losses: Optional[torch.Tensor] = None, dx: Optional[torch.Tensor] = None, stream=None) -> None:
        """One update of every episode with lens[e] > 0; tokens (int32) and x
        (bf16 [sum lens, din]) hold the episodes' rows one after another."""
        c = self.cfg
        if len(lens) != c.episodes:
            raise ValueError("one length per episode")
        R = int(sum(lens))
        if tokens.dtype != torch.int32 or tokens.numel() != R or tuple(x.shape) != (R, c.din):
            raise ValueError("tokens must be int32 [sum lens] and x [sum lens, din]")
        if losses is not None and (losses.dtype != torch.float32 or losses.numel() < c.episodes * c.grad_steps):
            raise ValueError("losses must be float32 [E, grad_steps]")
        if dx is not None and (dx.dtype != torch.float32 or dx.numel() < c.grad_steps * R * c.din):
            raise ValueError("dx must be float32 [grad_steps, sum lens, din]")
        arr = (ctypes.c_int64 * c.episodes)(*[int(v) for v in lens])
        _check(self._lib.attt_batch_update(self.handle, _ptr(tokens), _bf16(x), arr, _ptr(losses), _ptr(dx),
                                           _stream(stream)), "attt_batch_update")

    def reset(self, e: int = -1, stream=None) -> None:
        _check(self._lib.attt_batch_reset(self.handle, int(e), _stream(stream)), "attt_batch_reset")

    def read_adapter(self, e: int, stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
        c = self.cfg
        A = _empty((c.din, c.r), dtype=torch.float32, device=self.device, stream=stream)
        B = _empty((c.r, c.d), dtype=torch.float32, device=self.device, stream=stream)
        _check(self._lib.attt_batch_read_adapter(self.handle, int(e), _ptr(A), _ptr(B), _stream(stream)),
               "attt_batch_read_adapter")
        return A, B

    def history(self, e: int) -> History:
        h = self._lib.attt_batch_history(self.handle, int(e))
        return History._view(h, self.cfg.n, self.cfg.max_history, self)


def attt_lora_adamw_step(A32: torch.Tensor, B32: torch.Tensor, dA: torch.Tensor, dB: torch.Tensor,
                         mA: torch.Tensor, vA: torch.Tensor, mB: torch.Tensor, vB: torch.Tensor, lr: float, step: int,
                         betas=(0.9, 0.999), eps: float = 1e-8, weight_decay: float = 0.01,
                         A16: Optional[torch.Tensor] = None, B16: Optional[torch.Tensor] = None, stream=None) -> None:
    """In-place AdamW step on the fp32 masters (moments mA, vA, mB, vB), bf16 refresh."""
    din, r = A32.shape
    dout = B32.shape[1]
    _check((_lib or load_library()).attt_lora_adamw_step(
        _ptr(A32), _ptr(B32), _ptr(dA), _ptr(dB), _ptr(mA), _ptr(vA), _ptr(mB), _ptr(vB), din, dout, r, float(lr),
        float(betas[0]), float(betas[1]), float(eps), float(weight_decay), int(step),
        _bf16(A16) if A16 is not None else None, _bf16(B16) if B16 is not None else None, _stream(stream)),
        "attt_lora_adamw_step")


# --------------------------------------------------------------------------
# the step along orthogonalised momentum (Muon)
# --------------------------------------------------------------------------

def attt_lora_muon_workspace_bytes(dins: Sequence[int], douts: Sequence[int], r: int) -> int:
    k = len(dins)
    if len(douts) != k:
        raise ValueError("dins and douts must have one entry per projection")
    arr = (ctypes.c_int64 * (2 * k))(*[int(x) for x in dins], *[int(x) for x in douts])
    base = ctypes.addressof(arr)
    return int(load_library().attt_lora_muon_workspace_bytes(k, base, base + 8 * k, int(r)))


def attt_lora_muon_step(A32s: Sequence[torch.Tensor], B32s: Sequence[torch.Tensor], dAs: Sequence[torch.Tensor],
                        dBs: Sequence[torch.Tensor], mAs: Sequence[torch.Tensor], mBs: Sequence[torch.Tensor],
                        lr: float, momentum: float = 0.95, nesterov: bool = True, weight_decay: float = 0.0,
                        rms: float = 0.2, eps: float = 1e-7, ns_steps: int = 5,
                        A16s: Optional[Sequence[Optional[torch.Tensor]]] = None,
                        B16s: Optional[Sequence[Optional[torch.Tensor]]] = None,
                        workspace: Optional[torch.Tensor] = None, stream=None) -> None:
    """In-place Muon step of the adapters of some projections (A [din, r], B [r, dout],
    one rank): fp32 masters and momenta, bf16 refresh."""
    k = len(A32s)
    if k < 1 or any(len(ts) != k for ts in (B32s, dAs, dBs, mAs, mBs)) or (A16s is not None and len(A16s) != k) \
            or (B16s is not None and len(B16s) != k):
        raise ValueError("every list must have one entry per projection")
    f32, bf16 = torch.float32, torch.bfloat16
    if A32s[0].dim() != 2:
        raise ValueError(f"A32s[0]: expected a 2-D [din, r] tensor, got shape {tuple(A32s[0].shape)}")
    r = A32s[0].shape[1]
    dins, douts = [], []
    for i in range(k):
        A, B = A32s[i], B32s[i]
        if A.dim() != 2 or B.dim() != 2:
            raise ValueError(f"A32s[{i}], B32s[{i}]: expected 2-D tensors")
        sa, sb = (A.shape[0], r), (r, B.shape[1])
        dins.append(sa[0])
        douts.append(sb[1])
        for ts, shape, dtype, name in ((A32s, sa, f32, "A32s"), (dAs, sa, f32, "dAs"), (mAs, sa, f32, "mAs"),
                                       (B32s, sb, f32, "B32s"), (dBs, sb, f32, "dBs"), (mBs, sb, f32, "mBs"),
                                       (A16s, sa, bf16, "A16s"), (B16s, sb, bf16, "B16s")):
            t = ts[i] if ts is not None else None
            if t is not None and (t.shape != shape or t.dtype != dtype):
                _expect(t, shape, dtype, f"{name}[{i}]")
    if workspace is None:
        workspace = _empty(attt_lora_muon_workspace_bytes(dins, douts, r), dtype=torch.uint8,
                           device=A32s[0].device, stream=stream)
    vals = dins + douts
    for ts in (A32s, B32s, dAs, dBs, mAs, mBs, A16s or (), B16s or ()):
        vals += [_ptr(t) or 0 for t in ts]
    buf = (ctypes.c_int64 * len(vals))(*vals)
    base = ctypes.addressof(buf)
    at = [base + 8 * k * i for i in range(9)]
    p16a = at[8] if A16s is not None else None
    p16b = base + 8 * k * (9 if A16s is not None else 8) if B16s is not None else None
    _check((_lib or load_library()).attt_lora_muon_step(
        k, at[2], at[3], at[4], at[5], at[6], at[7], at[0], at[1], r, lr, momentum, 1 if nesterov else 0, weight_decay,
        rms, eps, ns_steps, p16a, p16b, _ptr(workspace), workspace.numel(), _stream(stream)), "attt_lora_muon_step")
