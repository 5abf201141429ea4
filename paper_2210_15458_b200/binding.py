"""ctypes binding of libarith_sampling.so: argument marshalling only.

Every function has the name and argument order of its C entry point
(include/arith_sampling.h); tensors are torch CUDA tensors whose data pointers are
passed through, `stream` defaults to torch's current stream.  bf16 logits may be
torch.bfloat16 tensors or int16/uint16 bit patterns.  There is no fallback: if the
library is missing or a call fails, an exception is raised.
"""
from __future__ import annotations

import contextlib
import ctypes
import os
from typing import Optional

import torch

from . import _build

F32 = 0
BF16 = 1
OK = 0
ERR_INVALID_ARG = -1
ERR_UNSUPPORTED = -2
ERR_CUDA = -3
ERR_TIMEOUT = -4
ERR_NUMERIC = -5
ERR_NO_PAGES = -6

PATH_COMPACT = 0
PATH_GENERAL = 1

TUNE_STEP_PATH = 1
TUNE_CLUSTER = 2
TUNE_CTAS_PER_SM = 3
TUNE_STAGES = 4
TUNE_MIN_CTAS = 5
TUNE_SERIAL_LAUNCH = 6
TUNE_WAIT_KCYCLES = 7
TUNE_DEBUG_NO_COPY = 8
TUNE_RADIX_NUCLEUS = 9

EXPORTS = ["as_lattice_codes", "as_lattice_codes_variant", "as_step", "as_step_typical", "as_step_lattice", "as_step_host", "as_step_host_work_bytes", "as_step_host_static",
           "as_decode_bigram",
           "as_decode_bigram_codes", "as_xp_lattice_state", "as_decode_bigram_xp", "as_encode_bigram", "as_ngram_diversity", "as_reward_mean", "as_logits_edit",
           "as_cache4_bytes", "as_cache4_append", "as_cache4_load", "as_cache4_attend_work_bytes", "as_cache4_attend",
           "as_pages_work_bytes", "as_pages_fork", "as_pages_grow", "as_pages_compact", "as_tune",
           "as_last_error", "as_version"]


class AsError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__("arith_sampling error %d: %s" % (code, msg))
        self.code = code


class as_step_diag(ctypes.Structure):
    _fields_ = [("d_p_tok", ctypes.c_void_p), ("d_cdf_lo", ctypes.c_void_p),
                ("d_n_kept", ctypes.c_void_p), ("d_lane_status", ctypes.c_void_p),
                ("d_path", ctypes.c_void_p)]


class as_logit_edits(ctypes.Structure):
    _fields_ = [("d_seq", ctypes.c_void_p), ("seq_ld", ctypes.c_longlong), ("d_len", ctypes.c_void_p),
                ("d_prompt_len", ctypes.c_void_p), ("repetition", ctypes.c_float), ("presence", ctypes.c_float),
                ("frequency", ctypes.c_float), ("d_bias", ctypes.c_void_p), ("bias_ld", ctypes.c_longlong),
                ("d_mask", ctypes.c_void_p), ("mask_ld", ctypes.c_longlong), ("mask_rows", ctypes.c_int),
                ("d_mask_row", ctypes.c_void_p)]


class as_cache4(ctypes.Structure):
    _fields_ = [("d_pages", ctypes.c_void_p), ("n_pages", ctypes.c_int), ("heads", ctypes.c_int),
                ("head_dim", ctypes.c_int), ("page_size", ctypes.c_int), ("d_k_scale", ctypes.c_void_p),
                ("d_v_scale", ctypes.c_void_p)]


_lib = None


def library_path() -> str:
    return _build.LIB


_path = None


def use_library(path: Optional[str]) -> None:
    """Switch to another build of the library (the bounds-checked one, in tests); None = the default."""
    global _lib, _path
    _lib, _path = None, path


def as_debug_bounds(reset: bool = True):
    """Checked builds only: (failures, first site, its index, its bound) since the last reset."""
    out = (ctypes.c_int * 4)()
    fn = lib().as_debug_bounds
    fn.argtypes = [ctypes.c_void_p, ctypes.c_int]
    fn.restype = ctypes.c_int
    _check(fn(ctypes.cast(out, ctypes.c_void_p), 1 if reset else 0))
    return tuple(out)


def lib():
    """Load the CUDA library (never builds or falls back silently)."""
    global _lib
    if _lib is None:
        path = _path or library_path()
        if not os.path.exists(path):
            raise RuntimeError("CUDA library %s not found: run `python -c 'import __graft_entry__ as g; "
                               "g.build()'` (nvcc, sm_100a) first" % path)
        L = ctypes.CDLL(path)
        P, I, D, LL = ctypes.c_void_p, ctypes.c_int, ctypes.c_double, ctypes.c_longlong
        L.as_lattice_codes.argtypes = [I, D, P, P]
        L.as_step.argtypes = [P, I, I, I, LL, P, D, I, D, P, P, ctypes.POINTER(as_step_diag), P]
        L.as_step_typical.argtypes = [P, I, I, I, LL, P, D, I, D, P, P, ctypes.POINTER(as_step_diag), P]
        L.as_step_typical.restype = I
        L.as_step_host.argtypes = [P, I, I, I, LL, P, D, I, D, P, P, P, P, ctypes.c_size_t, P]
        L.as_step_host_static.argtypes = [P, I, I, I, LL, P, D, I, D, P, P, P, P]
        L.as_step_host_static.restype = I
        L.as_step_host_work_bytes.argtypes = [I, I, LL]
        L.as_step_host_work_bytes.restype = ctypes.c_size_t
        L.as_decode_bigram.argtypes = [P, I, I, LL, P, I, I, D, I, I, D, I, D, P, P, P, P, P]
        L.as_decode_bigram_codes.argtypes = [P, I, I, LL, P, P, I, I, I, D, I, D, P, P, P, P, P]
        L.as_encode_bigram.argtypes = [P, I, I, LL, P, P, P, I, I, D, I, D, P, P, P, P]
        L.as_step_lattice.argtypes = [P, I, I, I, LL, I, D, I, D, I, D, P, P, P, P]
        L.as_step_lattice.restype = I
        L.as_lattice_codes_variant.argtypes = [I, D, I, P, P]
        L.as_lattice_codes_variant.restype = I
        L.as_ngram_diversity.argtypes = [P, P, I, I, I, P, P, P, P]
        L.as_reward_mean.argtypes = [P, P, I, I, I, P, I, P, P, P, P]
        L.as_xp_lattice_state.argtypes = [I, D, I, I, I, P, P]
        L.as_xp_lattice_state.restype = I
        L.as_decode_bigram_xp.argtypes = [P, I, I, LL, P, P, I, I, I, I, D, I, D, P, P, P, P]
        L.as_decode_bigram_xp.restype = I
        Z, PC = ctypes.c_size_t, ctypes.POINTER(as_cache4)
        L.as_logits_edit.argtypes = [P, I, I, I, LL, ctypes.POINTER(as_logit_edits), P, LL, P, P]
        L.as_cache4_bytes.argtypes = [I, I, I, I]
        L.as_cache4_append.argtypes = [PC, P, LL, P, LL, I, I, I, P, I, P, P, P]
        L.as_cache4_load.argtypes = [PC, P, P, I, I, I, P, I, P, P, P]
        L.as_cache4_attend_work_bytes.argtypes = [PC, I, I, I, I, I]
        L.as_cache4_attend.argtypes = [PC, P, LL, I, I, I, I, P, I, P, D, I, P, P, P, P, P, Z, P]
        L.as_pages_work_bytes.argtypes = [I, I, I]
        L.as_pages_fork.argtypes = [P, I, I, I, I, I, P, P, P, P, P, P, P, I, LL, LL, P, P, Z, P]
        L.as_pages_grow.argtypes = [P, I, I, I, I, P, P, P, P, P, Z, P]
        L.as_pages_compact.argtypes = [I, I, I, P, P, P, P, P, P, I, LL, LL, P, Z, P]
        for n in ("as_cache4_bytes", "as_cache4_attend_work_bytes", "as_pages_work_bytes"):
            getattr(L, n).restype = Z
        L.as_tune.argtypes = [I, I]
        L.as_last_error.restype = ctypes.c_char_p
        for n in ("as_lattice_codes", "as_step", "as_step_host", "as_decode_bigram",
                  "as_decode_bigram_codes", "as_xp_lattice_state", "as_decode_bigram_xp", "as_encode_bigram", "as_ngram_diversity", "as_reward_mean",
                  "as_logits_edit", "as_cache4_append", "as_cache4_load", "as_cache4_attend", "as_pages_fork", "as_pages_grow",
                  "as_pages_compact", "as_tune", "as_version"):
            getattr(L, n).restype = I
        _lib = L
    return _lib


def _check(rc: int) -> None:
    if rc != OK:
        raise AsError(rc, lib().as_last_error().decode())


# The current device's current stream, without building a Stream object around it (0.3 us instead of 4.8): look-ups that torch has
# but does not list, so that the public one stands in where they are missing.
_raw_stream, _device = (getattr(torch._C, name, None) for name in ("_cuda_getCurrentRawStream", "_cuda_getDevice"))


def _current_stream() -> int:
    if _raw_stream is None or _device is None:
        return torch.cuda.current_stream().cuda_stream
    return _raw_stream(_device())


def _stream(stream) -> int:
    if stream is None:
        return _current_stream()
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


_NO_SWITCH = contextlib.nullcontext()


def _owner(stream, device):
    """A context in which tensors are allocated from the memory of the stream that the call launches on.  Scratch is dropped on
    return: its block may only go to later work of the stream whose kernels still use it, and may only come from earlier work
    of that stream.  (`stream` as the calls take it: None, an object with a cuda_stream, or a raw handle.)"""
    if stream is None:
        return _NO_SWITCH
    raw = _stream(stream)
    if raw == _current_stream():
        return _NO_SWITCH
    if isinstance(stream, torch.cuda.Stream):
        return torch.cuda.stream(stream)
    # (0 and 1 are both the default stream)
    return torch.cuda.stream(torch.cuda.default_stream(device) if raw in (0, 1) else torch.cuda.ExternalStream(raw, device))


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else t.data_ptr()


_DTYPE_CODE = {torch.float32: F32, torch.bfloat16: BF16, torch.int16: BF16, torch.uint16: BF16}
_I32 = torch.int32


def _logits_dtype(t: torch.Tensor) -> int:
    d = _DTYPE_CODE.get(t.dtype)
    if d is not None:
        return d
    raise TypeError("logits must be float32 or bfloat16 (or 16-bit integer bit patterns)")


def _logits_layout(t: torch.Tensor):
    shape, stride = t.shape, t.stride()
    if len(shape) != 2 or stride[1] != 1:
        raise ValueError("logits / table must be 2-D with unit stride along the vocabulary")
    lanes, width = shape
    return lanes, width, (stride[0] if lanes > 1 else max(stride[0], width))


def as_version() -> int:
    return lib().as_version()


def as_tune(key: int, value: int) -> None:
    _check(lib().as_tune(key, value))


def as_lattice_codes(N: int, u: float, out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    if out is None:
        out = torch.empty(max(N, 0), dtype=torch.float64, device="cuda")
    _check(lib().as_lattice_codes(N, u, _ptr(out), _stream(stream)))
    return out


LATTICE_SHIFTED, LATTICE_PAPER_DEFINITION, LATTICE_NAIVE = 0, 1, 2
NGRAM_MAX_ITEMS = 16384     # AS_NGRAM_MAX_ITEMS


def as_lattice_codes_variant(N: int, b: float, variant: int, out: Optional[torch.Tensor] = None,
                             stream=None) -> torch.Tensor:
    if out is None:
        out = torch.empty(max(N, 0), dtype=torch.float64, device="cuda")
    _check(lib().as_lattice_codes_variant(N, b, variant, _ptr(out), _stream(stream)))
    return out


def as_step(logits: torch.Tensor, codes: torch.Tensor, temp: float = 1.0, top_k: int = 0,
            top_p: float = 1.0, tokens: Optional[torch.Tensor] = None,
            codes_out: Optional[torch.Tensor] = None, diag: Optional[dict] = None, V: Optional[int] = None,
            stream=None, typical_p: Optional[float] = None):
    """tokens, codes' = one decode step.  `diag`, if a dict, receives the tensors p_tok,
    cdf_lo, n_kept, lane_status, path (allocated here unless already present).  With typical_p
    the call goes to as_step_typical (the typical cut in place of the nucleus)."""
    lanes, width, ld = _logits_layout(logits)
    V = width if V is None else V
    dev = logits.device
    if tokens is None:
        tokens = torch.empty(lanes, dtype=torch.int32, device=dev)
    if codes_out is None:
        codes_out = torch.empty(lanes, dtype=torch.float64, device=dev)
    if codes.dtype != torch.float64 or codes.numel() != lanes:
        raise ValueError("codes must be float64 with one entry per lane")
    dg = None
    if diag is not None:
        diag.setdefault("p_tok", torch.empty(lanes, dtype=torch.float64, device=dev))
        diag.setdefault("cdf_lo", torch.empty(lanes, dtype=torch.float64, device=dev))
        diag.setdefault("n_kept", torch.empty(lanes, dtype=torch.int32, device=dev))
        diag.setdefault("lane_status", torch.empty(lanes, dtype=torch.int32, device=dev))
        diag.setdefault("path", torch.empty(lanes, dtype=torch.int32, device=dev))
        dg = as_step_diag(_ptr(diag["p_tok"]), _ptr(diag["cdf_lo"]), _ptr(diag["n_kept"]),
                          _ptr(diag["lane_status"]), _ptr(diag["path"]))
    if typical_p is not None:
        if 0.0 < top_p < 1.0:
            raise ValueError("a step takes top_p or typical_p, not both")
        _check(lib().as_step_typical(_ptr(logits), _logits_dtype(logits), lanes, V, ld, _ptr(codes), temp, top_k,
                                     typical_p, _ptr(tokens), _ptr(codes_out),
                                     ctypes.byref(dg) if dg is not None else None, _stream(stream)))
        return tokens, codes_out
    _check(lib().as_step(_ptr(logits), _logits_dtype(logits), lanes, V, ld, _ptr(codes), temp, top_k, top_p,
                         _ptr(tokens), _ptr(codes_out), ctypes.byref(dg) if dg is not None else None,
                         _stream(stream)))
    return tokens, codes_out


def as_step_lattice(logits: torch.Tensor, N: int, u: float, j0: int = 0, temp: float = 1.0, top_k: int = 0,
                    top_p: float = 1.0, tokens: Optional[torch.Tensor] = None,
                    codes_out: Optional[torch.Tensor] = None, V: Optional[int] = None, stream=None):
    """First decode step with the lattice codes (j0 + i + u)/N formed in the kernel."""
    lanes, width, ld = _logits_layout(logits)
    V = width if V is None else V
    dev = logits.device
    if tokens is None:
        tokens = torch.empty(lanes, dtype=torch.int32, device=dev)
    if codes_out is None:
        codes_out = torch.empty(lanes, dtype=torch.float64, device=dev)
    _check(lib().as_step_lattice(_ptr(logits), _logits_dtype(logits), lanes, V, ld, N, u, j0, temp, top_k, top_p,
                                 _ptr(tokens), _ptr(codes_out), None, _stream(stream)))
    return tokens, codes_out


def as_step_host_work_bytes(dtype: int, lanes: int, ld: int) -> int:
    return lib().as_step_host_work_bytes(dtype, lanes, ld)


def as_step_host(h_logits: torch.Tensor, h_codes: torch.Tensor, temp: float, top_k: int, top_p: float,
                 h_tokens: torch.Tensor, h_codes_out: torch.Tensor, h_lane_status: Optional[torch.Tensor],
                 d_work: torch.Tensor, V: Optional[int] = None, stream=None) -> None:
    """Host-buffer step: all h_* are CPU tensors (pinned for speed), d_work a CUDA byte buffer."""
    lanes, width, ld = _logits_layout(h_logits)
    V = width if V is None else V
    _check(lib().as_step_host(_ptr(h_logits), _logits_dtype(h_logits), lanes, V, ld, _ptr(h_codes), temp,
                              top_k, top_p, _ptr(h_tokens), _ptr(h_codes_out), _ptr(h_lane_status),
                              _ptr(d_work), d_work.numel() * d_work.element_size(), _stream(stream)))


STATIC_WORK_BYTES = 24 << 20


def as_step_host_static(h_logits: torch.Tensor, h_codes: torch.Tensor, temp: float, top_k: int, top_p: float,
                        h_tokens: torch.Tensor, h_codes_out: torch.Tensor, h_lane_status: Optional[torch.Tensor],
                        V: Optional[int] = None, stream=None) -> None:
    """as_step_host for callers that own no device memory: the device work space is a buffer
    built into the library (STATIC_WORK_BYTES).  Every tensor here is a CPU tensor; nothing is
    allocated on the device, neither by the library nor by this wrapper.  Steps that need more
    work space than the buffer holds raise AsError(ERR_UNSUPPORTED).  Calls share the buffer, so
    do not let two of them overlap on the GPU."""
    lanes, width, ld = _logits_layout(h_logits)
    V = width if V is None else V
    _check(lib().as_step_host_static(_ptr(h_logits), _logits_dtype(h_logits), lanes, V, ld, _ptr(h_codes), temp,
                                     top_k, top_p, _ptr(h_tokens), _ptr(h_codes_out), _ptr(h_lane_status),
                                     _stream(stream)))


def as_decode_bigram(table: torch.Tensor, start_tokens: torch.Tensor, N: int, u: float, T: int, eos: int,
                     temp: float = 1.0, top_k: int = 0, top_p: float = 1.0, V: Optional[int] = None,
                     codes_final: Optional[torch.Tensor] = None, lane_status: Optional[torch.Tensor] = None,
                     seq: Optional[torch.Tensor] = None, length: Optional[torch.Tensor] = None, stream=None,
                     per_step: bool = True):
    rows, width, ld = _logits_layout(table)
    V = width if V is None else V
    if rows < V:
        raise ValueError("bigram table needs at least V rows")
    S = start_tokens.numel()
    lanes = S * max(N, 0)
    dev = table.device
    if codes_final is None and per_step:    # also the loop's state for the per-step kernels
        codes_final = torch.empty(lanes, dtype=torch.float64, device=dev)
    if seq is None:
        seq = torch.empty((lanes, T), dtype=torch.int32, device=dev)
    if length is None:
        length = torch.empty(lanes, dtype=torch.int32, device=dev)
    _check(lib().as_decode_bigram(_ptr(table), _logits_dtype(table), V, ld, _ptr(start_tokens), S, N, u, T, eos,
                                  temp, top_k, top_p, _ptr(seq), _ptr(length), _ptr(codes_final),
                                  _ptr(lane_status), _stream(stream)))
    return seq, length


def as_decode_bigram_codes(table: torch.Tensor, prev: torch.Tensor, codes_in: torch.Tensor, T: int, eos: int,
                           temp: float = 1.0, top_k: int = 0, top_p: float = 1.0, V: Optional[int] = None,
                           codes_final: Optional[torch.Tensor] = None,
                           lane_status: Optional[torch.Tensor] = None, seq: Optional[torch.Tensor] = None,
                           length: Optional[torch.Tensor] = None, stream=None, per_step: bool = True):
    rows, width, ld = _logits_layout(table)
    V = width if V is None else V
    if rows < V:
        raise ValueError("bigram table needs at least V rows")
    lanes = prev.numel()
    dev = table.device
    if codes_final is None and per_step:    # also the loop's state for the per-step kernels
        codes_final = torch.empty(lanes, dtype=torch.float64, device=dev)
    if seq is None:
        seq = torch.empty((lanes, T), dtype=torch.int32, device=dev)
    if length is None:
        length = torch.empty(lanes, dtype=torch.int32, device=dev)
    _check(lib().as_decode_bigram_codes(_ptr(table), _logits_dtype(table), V, ld, _ptr(prev), _ptr(codes_in),
                                        lanes, T, eos, temp, top_k, top_p, _ptr(seq), _ptr(length),
                                        _ptr(codes_final), _ptr(lane_status), _stream(stream)))
    return seq, length


def as_xp_lattice_state(N: int, u: float, j0: int = 0, count: Optional[int] = None, S: int = 1,
                        out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """int64 [S*count, 4] (the bits of four unsigned 64-bit words per lane): decoder state of the
    lattice codes (j + u)/N, j = j0 .. j0+count-1, one copy per start token."""
    count = N - j0 if count is None else count
    if out is None:
        out = torch.empty((max(S, 0) * max(count, 0), 4), dtype=torch.int64, device="cuda")
    _check(lib().as_xp_lattice_state(N, u, j0, count, S, _ptr(out), _stream(stream)))
    return out


def as_decode_bigram_xp(table: torch.Tensor, prev: torch.Tensor, state: torch.Tensor, N: int, T: int, eos: int,
                        temp: float = 1.0, top_k: int = 0, top_p: float = 1.0, V: Optional[int] = None,
                        lane_status: Optional[torch.Tensor] = None, seq: Optional[torch.Tensor] = None,
                        length: Optional[torch.Tensor] = None, stream=None):
    """Algorithm 1's loop with extended-precision codes; `state` [lanes, 4] int64 is updated in place."""
    rows, width, ld = _logits_layout(table)
    V = width if V is None else V
    if rows < V:
        raise ValueError("bigram table needs at least V rows")
    lanes = prev.numel()
    if state.dtype != torch.int64 or state.numel() != 4 * lanes or not state.is_contiguous():
        raise ValueError("state must be a contiguous [lanes, 4] int64 tensor")
    dev = table.device
    if seq is None:
        seq = torch.empty((lanes, T), dtype=torch.int32, device=dev)
    if length is None:
        length = torch.empty(lanes, dtype=torch.int32, device=dev)
    _check(lib().as_decode_bigram_xp(_ptr(table), _logits_dtype(table), V, ld, _ptr(prev), _ptr(state), lanes, N, T,
                                     eos, temp, top_k, top_p, _ptr(seq), _ptr(length), _ptr(lane_status),
                                     _stream(stream)))
    return seq, length


def as_encode_bigram(table: torch.Tensor, prev: torch.Tensor, seq: torch.Tensor, length: torch.Tensor,
                     temp: float = 1.0, top_k: int = 0, top_p: float = 1.0, V: Optional[int] = None,
                     lane_status: Optional[torch.Tensor] = None, stream=None):
    """Interval [lo, lo + width) of each lane's sequence in dictionary order (Sec. 4.1)."""
    rows, width_, ld = _logits_layout(table)
    V = width_ if V is None else V
    if rows < V:
        raise ValueError("bigram table needs at least V rows")
    if seq.dim() != 2 or not seq.is_contiguous() or seq.dtype != torch.int32:
        raise ValueError("seq must be a contiguous [lanes, T] int32 tensor")
    lanes, T = seq.shape
    if prev.numel() != lanes or length.numel() != lanes:
        raise ValueError("prev and length need one entry per lane")
    dev = table.device
    lo = torch.empty(lanes, dtype=torch.float64, device=dev)
    width = torch.empty(lanes, dtype=torch.float64, device=dev)
    _check(lib().as_encode_bigram(_ptr(table), _logits_dtype(table), V, ld, _ptr(prev), _ptr(seq), _ptr(length),
                                  lanes, T, temp, top_k, top_p, _ptr(lo), _ptr(width), _ptr(lane_status),
                                  _stream(stream)))
    return lo, width


def _groups(seq: torch.Tensor, length: torch.Tensor, N: int):
    if seq.dim() != 2 or not seq.is_contiguous() or seq.dtype != torch.int32:
        raise ValueError("seq must be a contiguous [lanes, T] int32 tensor")
    lanes, T = seq.shape
    if N < 1 or lanes % N or length.numel() != lanes:
        raise ValueError("lanes must be a multiple of N, with one length per lane")
    return lanes // N, T


def as_ngram_diversity(seq: torch.Tensor, length: torch.Tensor, N: int, stream=None):
    """(unique[S,4], total[S,4], d[S]): n-gram diversity of each group of N lanes (Sec. 5.1)."""
    S, T = _groups(seq, length, N)
    dev = seq.device
    unique = torch.empty((S, 4), dtype=torch.int64, device=dev)
    total = torch.empty((S, 4), dtype=torch.int64, device=dev)
    d = torch.empty(S, dtype=torch.float64, device=dev)
    _check(lib().as_ngram_diversity(_ptr(seq), _ptr(length), S, N, T, _ptr(unique), _ptr(total), _ptr(d),
                                    _stream(stream)))
    return unique, total, d


def as_reward_mean(seq: torch.Tensor, length: torch.Tensor, N: int, r: torch.Tensor,
                   group_status: Optional[torch.Tensor] = None, stream=None):
    """(lane_reward[lanes], mean[S]) for the additive reward r[token] (Sec. 4.2 estimator)."""
    S, T = _groups(seq, length, N)
    if r.dtype != torch.float64 or not r.is_contiguous():
        raise ValueError("r must be a contiguous float64 tensor")
    dev = seq.device
    lane_reward = torch.empty(S * N, dtype=torch.float64, device=dev)
    mean = torch.empty(S, dtype=torch.float64, device=dev)
    _check(lib().as_reward_mean(_ptr(seq), _ptr(length), S, N, T, _ptr(r), r.numel(), _ptr(lane_reward),
                                _ptr(mean), _ptr(group_status), _stream(stream)))
    return lane_reward, mean


# The calls below allocate what is not passed (outputs, scratch) from the memory of the stream they launch on, as if they stood
# under torch.cuda.stream(stream): an output that other streams use as well is the caller's to record there.


def _int32(t: Optional[torch.Tensor], name: str, numel: Optional[int] = None):
    """Device pointer of a contiguous int32 tensor (None stays None)."""
    if t is None:
        return None
    if t.dtype is not _I32 or not t.is_contiguous() or (numel is not None and t.numel() != numel):
        raise ValueError("%s must be a contiguous int32 tensor%s" % (name, "" if numel is None else " of %d entries" % numel))
    return t.data_ptr()


def as_logits_edit(logits: torch.Tensor, seq: Optional[torch.Tensor] = None, length: Optional[torch.Tensor] = None,
                   prompt_length: Optional[torch.Tensor] = None, repetition: float = 1.0, presence: float = 0.0,
                   frequency: float = 0.0, bias: Optional[torch.Tensor] = None, mask: Optional[torch.Tensor] = None,
                   mask_row: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None,
                   lane_status: Optional[torch.Tensor] = None, V: Optional[int] = None, stream=None) -> torch.Tensor:
    """Penalties, bias and grammar mask on logits [lanes, V].  seq [lanes, T] int32 with length [lanes]
    is the history (as_decode_bigram's layout), bias float32 [V] or [lanes, V], mask int32 [rows, ceil(V/32)]
    (bit set = allowed) with mask_row [lanes] (-1 = none).  out=logits edits in place."""
    lanes, width, ld = _logits_layout(logits)
    V = width if V is None else V
    out_ld = V
    if out is None:
        with _owner(stream, logits.device):
            out = logits.new_empty((lanes, V))
    elif out.dtype != logits.dtype or out.dim() != 2 or out.shape[0] != lanes or out.shape[1] < V:
        raise ValueError("out must have the logits' dtype and a row of at least V for each lane")
    else:
        out_ld = _logits_layout(out)[2]
    e = as_logit_edits(None, 0, None, None, repetition, presence, frequency)
    if seq is not None:
        if seq.dim() != 2 or seq.shape[0] != lanes or length is None:
            raise ValueError("seq must be [lanes, T] and comes with a length for each lane")
        e.d_seq, e.seq_ld = _int32(seq, "seq"), seq.shape[1]
        e.d_len, e.d_prompt_len = _int32(length, "length", lanes), _int32(prompt_length, "prompt_length", lanes)
    if bias is not None:
        shape, stride = bias.shape, bias.stride()
        rows = shape[0] if len(shape) == 2 else 1
        if bias.dtype is not torch.float32 or stride[-1] != 1 or shape[-1] < V or len(shape) > 2 or rows not in (1, lanes):
            raise ValueError("bias must be float32, [V] or [lanes, V], with unit stride along the vocabulary")
        e.d_bias, e.bias_ld = bias.data_ptr(), (stride[0] if rows > 1 else 0)
    if mask is not None:
        shape, stride = mask.shape, mask.stride()
        if mask.dtype is not _I32 or len(shape) != 2 or stride[1] != 1 or shape[1] < (V + 31) // 32:
            raise ValueError("mask must be int32 [rows, ceil(V / 32)] with unit stride along a row")
        e.d_mask, e.mask_rows, e.mask_ld = mask.data_ptr(), shape[0], (stride[0] if shape[0] > 1 else shape[1])
        e.d_mask_row = _int32(mask_row, "mask_row", lanes)
    _check(lib().as_logits_edit(logits.data_ptr(), _logits_dtype(logits), lanes, V, ld, ctypes.byref(e), out.data_ptr(),
                                out_ld, _int32(lane_status, "lane_status", lanes), _stream(stream)))
    return out


def as_cache4_bytes(n_pages: int, heads: int, head_dim: int, page_size: int) -> int:
    return lib().as_cache4_bytes(n_pages, heads, head_dim, page_size)


def cache4_pages(n_pages: int, heads: int, head_dim: int, page_size: int, planes: Optional[int] = None,
                 device="cuda") -> torch.Tensor:
    """Zeroed pages of a 4-bit cache, uint8 [n_pages, heads, page_size / 16, 18 * head_dim], the shape that tells the
    calls below heads, head_dim and page_size; with `planes`, one such tensor for each layer ([planes, ...])."""
    shape = (n_pages, heads, page_size // 16, 18 * head_dim)
    return torch.zeros(shape if planes is None else (planes,) + shape, dtype=torch.uint8, device=device)


def _cache4(pages: torch.Tensor, k_scale, v_scale) -> as_cache4:
    shape = pages.shape
    if pages.dtype is not torch.uint8 or len(shape) != 4 or not pages.is_contiguous() or shape[3] % 18:
        raise ValueError("pages must be a contiguous uint8 tensor [n_pages, heads, page_size / 16, 18 * head_dim]")
    n, heads, tiles, width = shape
    for s in (k_scale, v_scale):
        if s is not None and (s.dtype is not torch.float32 or s.numel() != heads or not s.is_contiguous()):
            raise ValueError("k_scale and v_scale must be contiguous float32 with an entry for each head")
    return as_cache4(pages.data_ptr(), n, heads, width // 18, tiles * 16, _ptr(k_scale), _ptr(v_scale))


def _tokens(t: torch.Tensor, D: int, name: str):
    """(lanes, T, heads, elements from token to token) of a [lanes, T, heads, D] tensor whose heads lie side by side."""
    shape = t.shape
    if len(shape) != 4 or shape[3] != D:
        raise ValueError("%s must be [lanes, T, heads, %d]" % (name, D))
    lanes, T, heads, _ = shape
    sl, st, sh, sd = t.stride()
    ld = st if T > 1 else sl if lanes > 1 else heads * D
    if sd != 1 or (heads > 1 and sh != D) or (lanes > 1 and T > 1 and sl != T * st):
        raise ValueError("%s: heads must lie side by side and tokens at one distance" % name)
    return lanes, T, heads, ld


def _table(table: torch.Tensor, length: torch.Tensor, lanes: int):
    shape = table.shape
    if len(shape) != 2 or shape[0] != lanes:
        raise ValueError("table must be [lanes, max_pages]")
    return _int32(table, "table"), shape[1], _int32(length, "length", lanes)


def as_cache4_append(pages: torch.Tensor, k: torch.Tensor, v: torch.Tensor, table: torch.Tensor, length: torch.Tensor,
                     k_scale: Optional[torch.Tensor] = None, v_scale: Optional[torch.Tensor] = None,
                     lane_status: Optional[torch.Tensor] = None, stream=None) -> None:
    """Store k, v [lanes, T, heads, D] as the last T of each lane's length[lane] tokens."""
    c = _cache4(pages, k_scale, v_scale)
    lanes, T, heads, k_ld = _tokens(k, c.head_dim, "k")
    if v.shape != k.shape or v.dtype != k.dtype or heads != c.heads:
        raise ValueError("k and v must have the same shape and dtype, and the cache's heads")
    tp, max_pages, lp = _table(table, length, lanes)
    _check(lib().as_cache4_append(ctypes.byref(c), k.data_ptr(), k_ld, v.data_ptr(), _tokens(v, c.head_dim, "v")[3],
                                  _logits_dtype(k), lanes, T, tp, max_pages, lp,
                                  _int32(lane_status, "lane_status", lanes), _stream(stream)))


def as_cache4_load(pages: torch.Tensor, table: torch.Tensor, length: torch.Tensor, T: int,
                   k_scale: Optional[torch.Tensor] = None, v_scale: Optional[torch.Tensor] = None, dtype=torch.bfloat16,
                   lane_status: Optional[torch.Tensor] = None, stream=None):
    """(k, v) [lanes, T, heads, D]: what is stored for the last T tokens of each lane (zeros where there is none)."""
    c = _cache4(pages, k_scale, v_scale)
    lanes = length.numel()
    with _owner(stream, pages.device):
        k = pages.new_empty((lanes, T, c.heads, c.head_dim), dtype=dtype)
        v = torch.empty_like(k)
    tp, max_pages, lp = _table(table, length, lanes)
    _check(lib().as_cache4_load(ctypes.byref(c), k.data_ptr(), v.data_ptr(), _logits_dtype(k), lanes, T, tp, max_pages, lp,
                                _int32(lane_status, "lane_status", lanes), _stream(stream)))
    return k, v


def as_cache4_attend_work_bytes(pages: torch.Tensor, dtype: int, lanes: int, T: int, q_heads: int, N: int = 1) -> int:
    return lib().as_cache4_attend_work_bytes(ctypes.byref(_cache4(pages, None, None)), dtype, lanes, T, q_heads, N)


def as_cache4_attend(pages: torch.Tensor, q: torch.Tensor, table: torch.Tensor, length: torch.Tensor, scale: float,
                     k_scale: Optional[torch.Tensor] = None, v_scale: Optional[torch.Tensor] = None, N: int = 1,
                     shared: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None,
                     lse: Optional[torch.Tensor] = None, lane_status: Optional[torch.Tensor] = None,
                     work: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """Attention of q [lanes, T, q_heads, D], the last T tokens of each lane, over the lane's cached tokens (causal).
    shared [lanes / N] int32: how many leading tokens the N lanes of a group have in the same pages.  Bad lengths and pages
    and waits that ran out are reported in lane_status alone."""
    c = _cache4(pages, k_scale, v_scale)
    lanes, T, heads, q_ld = _tokens(q, c.head_dim, "q")
    if out is not None and (out.shape != q.shape or out.dtype != q.dtype or not out.is_contiguous()):
        raise ValueError("out must be contiguous, with the shape and dtype of q")
    if lse is not None and (lse.dtype != torch.float32 or lse.numel() != lanes * T * heads or not lse.is_contiguous()):
        raise ValueError("lse must be contiguous float32 [lanes, T, q_heads]")
    L = lib()
    dt = _logits_dtype(q)
    need = L.as_cache4_attend_work_bytes(ctypes.byref(c), dt, lanes, T, heads, N)
    tp, max_pages, lp = _table(table, length, lanes)
    if out is None or work is None:
        with _owner(stream, q.device):
            out = q.new_empty((lanes, T, heads, c.head_dim)) if out is None else out
            work = length.new_empty((need + 3) // 4) if work is None else work
    _check(L.as_cache4_attend(ctypes.byref(c), q.data_ptr(), q_ld, dt, lanes, T, heads, tp, max_pages, lp, scale, N,
                              _int32(shared, "shared", lanes // N if N > 0 else None), out.data_ptr(), _ptr(lse),
                              _int32(lane_status, "lane_status", lanes), work.data_ptr(),
                              work.numel() * work.element_size(), _stream(stream)))
    return out


def as_pages_work_bytes(lanes_in: int, lanes_out: int, n_pages: int) -> int:
    return lib().as_pages_work_bytes(lanes_in, lanes_out, n_pages)


def _pool(pool: Optional[torch.Tensor], n_pages: int):
    """(pointer, planes, bytes from plane to plane, bytes of a page) of a pool [planes, n_pages, ...]."""
    if pool is None:
        return None, 0, 0, 16
    if pool.dim() < 2 or pool.shape[1] != n_pages or not pool[0].is_contiguous():
        raise ValueError("pool must be [planes, n_pages, ...] with contiguous planes")
    e = pool.element_size()
    return pool.data_ptr(), pool.shape[0], pool.stride(0) * e, pool.stride(1) * e


def _pages_work(work: Optional[torch.Tensor], lanes_in: int, lanes_out: int, n_pages: int, like: torch.Tensor):
    """(scratch, its bytes); allocated under _owner."""
    if work is None:
        work = like.new_empty((lib().as_pages_work_bytes(lanes_in, lanes_out, n_pages) + 3) // 4)
    return work, work.numel() * work.element_size()


def as_pages_fork(parent: torch.Tensor, table: torch.Tensor, length: torch.Tensor, ref: torch.Tensor, page_size: int,
                  pool: Optional[torch.Tensor] = None, table_out: Optional[torch.Tensor] = None,
                  length_out: Optional[torch.Tensor] = None, ref_out: Optional[torch.Tensor] = None,
                  lane_status: Optional[torch.Tensor] = None, work: Optional[torch.Tensor] = None, stream=None):
    """(table, length, ref) in which lane i continues lane parent[i] (-1: nothing); pool [planes, n_pages, ...] is the
    cache whose partly filled last pages are copied.  ref_out may be ref; the other outputs are new tensors."""
    lanes, max_pages = table.shape
    n = parent.numel()
    data, planes, stride, page_bytes = _pool(pool, ref.numel())
    with _owner(stream, ref.device):
        if table_out is None:
            table_out = table.new_empty((n, max_pages))
        if length_out is None:
            length_out = table.new_empty(n)
        if ref_out is None:
            ref_out = torch.empty_like(ref)
        work, nbytes = _pages_work(work, lanes, n, ref.numel(), ref)
    _check(lib().as_pages_fork(_int32(parent, "parent"), lanes, n, max_pages, page_size, ref.numel(), _int32(table, "table"),
                               _int32(length, "length", lanes), _int32(ref, "ref"),
                               _int32(table_out, "table_out", n * max_pages), _int32(length_out, "length_out", n),
                               _int32(ref_out, "ref_out", ref.numel()), data, planes, stride, page_bytes,
                               _int32(lane_status, "lane_status", n), work.data_ptr(), nbytes, _stream(stream)))
    return table_out, length_out, ref_out


def as_pages_grow(add: torch.Tensor, table: torch.Tensor, length: torch.Tensor, ref: torch.Tensor, page_size: int,
                  lane_status: Optional[torch.Tensor] = None, work: Optional[torch.Tensor] = None, stream=None) -> None:
    """Give every lane the pages for add[lane] more tokens; table, length and ref are updated in place."""
    lanes, max_pages = table.shape
    with _owner(stream, ref.device):
        work, nbytes = _pages_work(work, lanes, lanes, ref.numel(), ref)
    _check(lib().as_pages_grow(_int32(add, "add", lanes), lanes, max_pages, page_size, ref.numel(), _int32(table, "table"),
                               _int32(length, "length", lanes), _int32(ref, "ref"),
                               _int32(lane_status, "lane_status", lanes), work.data_ptr(), nbytes, _stream(stream)))


def as_pages_compact(table: torch.Tensor, ref: torch.Tensor, pool: Optional[torch.Tensor] = None,
                     table_out: Optional[torch.Tensor] = None, ref_out: Optional[torch.Tensor] = None,
                     used: Optional[torch.Tensor] = None, work: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """Move the pages in use to the front of the pool; returns their number (int32 [] on the device).  Without
    table_out / ref_out the table and the reference counts are updated in place."""
    lanes, max_pages = table.shape
    table_out = table if table_out is None else table_out
    ref_out = ref if ref_out is None else ref_out
    data, planes, stride, page_bytes = _pool(pool, ref.numel())
    with _owner(stream, ref.device):
        if used is None:
            used = table.new_empty(())
        work, nbytes = _pages_work(work, lanes, lanes, ref.numel(), ref)
    _check(lib().as_pages_compact(lanes, max_pages, ref.numel(), _int32(table, "table"), _int32(ref, "ref"),
                                  _int32(table_out, "table_out", table.numel()), _int32(ref_out, "ref_out", ref.numel()),
                                  _int32(used, "used", 1), data, planes, stride, page_bytes, work.data_ptr(), nbytes,
                                  _stream(stream)))
    return used
