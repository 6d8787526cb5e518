"""Chunkwise preconditioned delta rule (PDN / PGDN / PKDA) on MI355X.

Thin ctypes binding of libpdn.so, the C ABI declared in include/pdn.h.  The
binding only marshals arguments: it maps torch tensors to device pointers,
allocates outputs and the workspace when the caller does not pass them, and
turns status codes into exceptions.  Every step of the computation runs in
the library's HIP kernels; there is no fallback.  Importing this package
fails loudly if the library has not been built.
"""
from __future__ import annotations

import ctypes
import os

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libpdn.so")

if not os.path.exists(LIB_PATH):
    raise ImportError(
        f"{LIB_PATH} is missing: build the HIP library first "
        "(python -c 'import __graft_entry__ as g; g.build()' or "
        "python paper_2604_21100_amd/_build.py)")

# The library and torch must share one HIP runtime.  torch ships its own
# libamdhip64 / libhsa-runtime64 under the same sonames as the system ROCm
# that libpdn.so is linked against: if libpdn.so were loaded first, torch
# would later map a second pair, and two HSA runtimes in one process make
# every HIP call undefined.  Loading torch first makes libpdn.so bind to the
# runtime already in the process.
try:
    import torch  # noqa: F401
except ImportError:   # no torch: the C ABI alone, nothing else maps HIP
    torch = None
_lib = ctypes.CDLL(LIB_PATH)


class _NotBuilt:
    """In the compiled binding's place: the calls that need it (those on a pool of
    states) say what is wrong, everything else goes without it."""

    def __init__(self, why):
        self._why = why

    def __getattr__(self, name):
        raise ImportError(f"_pdn_torch is missing or was built for another "
                          f"torch ({self._why}): build it with the library")


try:
    if torch is None:
        raise ImportError("no torch")
    from . import _pdn_torch
except ImportError as _e:
    _pdn_torch = _NotBuilt(_e)


def loaded_hip_runtimes():
    """Paths of the HIP runtime libraries mapped into this process."""
    try:
        with open("/proc/self/maps") as f:
            maps = f.read()
    except OSError:
        return []
    return sorted({ln.split()[-1] for ln in maps.splitlines()
                   if "libamdhip64" in ln and "/" in ln})


if len(loaded_hip_runtimes()) > 1:
    raise ImportError(
        "two HIP runtimes are mapped into this process "
        f"({loaded_hip_runtimes()}); import torch before anything that "
        "loads the system ROCm runtime")

# ---------------------------------------------------------------- enums
PDN_OK, PDN_ERR_NULL, PDN_ERR_SHAPE, PDN_ERR_DTYPE, PDN_ERR_UNSUPPORTED, \
    PDN_ERR_ALIGN, PDN_ERR_ALIAS, PDN_ERR_WORKSPACE, PDN_ERR_VALUE, \
    PDN_ERR_HIP, PDN_ERR_SCRATCH = range(11)
PDN_F32, PDN_BF16 = 0, 1
PDN_GATE_NONE, PDN_GATE_SCALAR, PDN_GATE_CHANNEL = 0, 1, 2
PDN_PRECOND_SQUASH, PDN_PRECOND_IDENTITY, PDN_PRECOND_EXTERNAL, \
    PDN_PRECOND_DIAG_SM, PDN_PRECOND_ATQ = 0, 1, 2, 3, 4

GATES = {"none": PDN_GATE_NONE, "scalar": PDN_GATE_SCALAR,
         "channel": PDN_GATE_CHANNEL}
PRECONDS = {"squash": PDN_PRECOND_SQUASH, "identity": PDN_PRECOND_IDENTITY,
            "external": PDN_PRECOND_EXTERNAL, "diag_sm": PDN_PRECOND_DIAG_SM,
            "atq": PDN_PRECOND_ATQ}
# modes driven by the diagonal key-Gram recurrence (they take beta_p, g_p,
# A0 and return A_T)
GRAM_PRECONDS = ("squash", "diag_sm", "atq")
# write-key normalisation of the squash mode (pdn_knorm)
KNORMS = {"none": 0, "m": 1, "1pm": 2, "beta": 3}

# what a head norm divides by, and the activation of its gate (pdn_norm, pdn_act)
NORMS = {"rms": 0, "l2": 1}
ACTS = {"none": 0, "silu": 1, "sigmoid": 2}

_vp = ctypes.c_void_p


class Problem(ctypes.Structure):
    _fields_ = [("B", ctypes.c_int64), ("T", ctypes.c_int64),
                ("H", ctypes.c_int64), ("dk", ctypes.c_int32),
                ("dv", ctypes.c_int32), ("chunk", ctypes.c_int32),
                ("io", ctypes.c_int), ("gate", ctypes.c_int),
                ("precond", ctypes.c_int), ("x", ctypes.c_float),
                ("scale", ctypes.c_float), ("ridge", ctypes.c_float),
                ("knorm", ctypes.c_int)]


class Inputs(ctypes.Structure):
    _fields_ = [(n, _vp) for n in ("q", "k", "v", "beta", "g", "beta_p",
                                   "g_p", "log_a_scale", "A0", "S0",
                                   "ktilde")]


class FwdOut(ctypes.Structure):
    _fields_ = [("o", _vp), ("S_T", _vp), ("A_T", _vp)]


class BwdOut(ctypes.Structure):
    _fields_ = [(n, _vp) for n in ("dq", "dk", "dv", "dbeta", "dg", "dS0",
                                   "dbeta_p", "dg_p", "dlog_a_scale", "dA0",
                                   "dktilde")]


class Slots(ctypes.Structure):
    _fields_ = ([(n, ctypes.c_int64) for n in ("tokens", "slots", "Hk", "q_stride",
                                               "k_stride", "v_stride")]
                + [(n, _vp) for n in ("starts", "slot", "slot_out", "fresh",
                                      "S", "A", "tape")]
                + [("tape_tokens", ctypes.c_int64), ("pending", _vp),
                   ("accepted", _vp)])


class Rnorm(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int64), ("D", ctypes.c_int64),
                ("io", ctypes.c_int), ("stream", ctypes.c_int),
                ("post_norm", ctypes.c_int32), ("alpha", ctypes.c_float),
                ("eps", ctypes.c_float)]


class Hnorm(ctypes.Structure):
    _fields_ = ([("tokens", ctypes.c_int64), ("H", ctypes.c_int64),
                 ("d", ctypes.c_int32), ("io", ctypes.c_int),
                 ("norm", ctypes.c_int), ("act", ctypes.c_int),
                 ("head_weight", ctypes.c_int32), ("eps", ctypes.c_float)]
                + [(n, ctypes.c_int64) for n in (
                    "x_stride", "z_stride", "y_stride", "dy_stride",
                    "dx_stride", "dz_stride")])


class LogitsArgs(ctypes.Structure):
    _fields_ = ([(n, ctypes.c_int64) for n in ("rows", "V", "N")]
                + [("dtype", ctypes.c_int), ("out_dtype", ctypes.c_int),
                   ("probs", ctypes.c_int32), ("stride", ctypes.c_int64)]
                + [(n, _vp) for n in ("logits", "starts", "temperature",
                                      "repetition", "presence", "frequency",
                                      "counts")]
                + [("slots", ctypes.c_int64)]
                + [(n, _vp) for n in ("slot", "ids", "bias_starts",
                                      "bias_ids", "bias_values")]
                + [("biases", ctypes.c_int64), ("mask", _vp),
                   ("masks", ctypes.c_int64), ("mask_rows", _vp)])


_lib.pdn_workspace_size.argtypes = [ctypes.POINTER(Problem), ctypes.c_int,
                                    ctypes.POINTER(ctypes.c_size_t)]
_lib.pdn_workspace_size.restype = ctypes.c_int
_lib.pdn_chunk_fwd.argtypes = [ctypes.POINTER(Problem), ctypes.POINTER(Inputs),
                               ctypes.POINTER(FwdOut), _vp, ctypes.c_size_t,
                               _vp]
_lib.pdn_chunk_fwd.restype = ctypes.c_int
_lib.pdn_chunk_fwd_events.argtypes = [
    ctypes.POINTER(Problem), ctypes.POINTER(Inputs), ctypes.POINTER(FwdOut),
    _vp, ctypes.c_size_t, _vp, ctypes.POINTER(_vp), ctypes.c_int]
_lib.pdn_chunk_fwd_events.restype = ctypes.c_int
_lib.pdn_chunk_bwd.argtypes = [ctypes.POINTER(Problem), ctypes.POINTER(Inputs),
                               _vp, _vp, ctypes.POINTER(BwdOut), _vp,
                               ctypes.c_size_t, _vp]
_lib.pdn_chunk_bwd.restype = ctypes.c_int
_lib.pdn_chunk_bwd_events.argtypes = [
    ctypes.POINTER(Problem), ctypes.POINTER(Inputs), _vp, _vp,
    ctypes.POINTER(BwdOut), _vp, ctypes.c_size_t, _vp, ctypes.POINTER(_vp),
    ctypes.c_int]
_lib.pdn_chunk_bwd_events.restype = ctypes.c_int
_lib.pdn_chunk_fwd_train.argtypes = [
    ctypes.POINTER(Problem), ctypes.POINTER(Inputs), ctypes.POINTER(FwdOut),
    _vp, ctypes.c_size_t, _vp, ctypes.POINTER(_vp), ctypes.c_int]
_lib.pdn_chunk_fwd_train.restype = ctypes.c_int
_lib.pdn_chunk_bwd_train.argtypes = [
    ctypes.POINTER(Problem), ctypes.POINTER(Inputs), _vp, _vp,
    ctypes.POINTER(BwdOut), _vp, ctypes.c_size_t, _vp, ctypes.POINTER(_vp),
    ctypes.c_int]
_lib.pdn_chunk_bwd_train.restype = ctypes.c_int
_lib.pdn_chunk_fwd_noalloc.argtypes = [
    ctypes.POINTER(Problem), ctypes.POINTER(Inputs), ctypes.POINTER(FwdOut),
    _vp]
_lib.pdn_chunk_fwd_noalloc.restype = ctypes.c_int
for _f in (_lib.pdn_slot_fwd, _lib.pdn_slot_draft):
    _f.argtypes = [_vp] * 5   # (the structures by reference, or their bytes)
    _f.restype = ctypes.c_int
_lib.pdn_draft_verify.argtypes = [ctypes.c_int64, ctypes.c_int64,
                                  ctypes.c_int64, ctypes.c_int, *[_vp] * 9,
                                  ctypes.c_size_t, _vp]
_lib.pdn_draft_verify.restype = ctypes.c_int
_lib.pdn_draft_verify_workspace_size.argtypes = [
    ctypes.c_int64, ctypes.c_int64, ctypes.POINTER(ctypes.c_size_t)]
_lib.pdn_draft_verify_workspace_size.restype = ctypes.c_int
_size_p = ctypes.POINTER(ctypes.c_size_t)
_lib.pdn_residual_norm.argtypes = [ctypes.POINTER(Rnorm), *[_vp] * 8]
_lib.pdn_residual_norm_bwd.argtypes = [ctypes.POINTER(Rnorm), *[_vp] * 13,
                                       ctypes.c_size_t, _vp]
_lib.pdn_residual_norm_bwd_workspace_size.argtypes = [ctypes.POINTER(Rnorm),
                                                      _size_p]
_lib.pdn_head_norm.argtypes = [ctypes.POINTER(Hnorm), *[_vp] * 5]
_lib.pdn_head_norm_bwd.argtypes = [ctypes.POINTER(Hnorm), *[_vp] * 8,
                                   ctypes.c_size_t, _vp]
_lib.pdn_head_norm_bwd_workspace_size.argtypes = [ctypes.POINTER(Hnorm),
                                                  _size_p]
_lib.pdn_logits.argtypes = [ctypes.POINTER(LogitsArgs), _vp, _vp,
                            ctypes.c_size_t, _vp]
_lib.pdn_logits_workspace_size.argtypes = [ctypes.c_int64, ctypes.c_int64,
                                           _size_p]
_lib.pdn_token_counts.argtypes = [*[ctypes.c_int64] * 4, ctypes.c_int32,
                                  *[_vp] * 8]
for _f in (_lib.pdn_residual_norm, _lib.pdn_residual_norm_bwd,
           _lib.pdn_residual_norm_bwd_workspace_size, _lib.pdn_head_norm,
           _lib.pdn_head_norm_bwd, _lib.pdn_head_norm_bwd_workspace_size,
           _lib.pdn_logits, _lib.pdn_logits_workspace_size,
           _lib.pdn_token_counts):
    _f.restype = ctypes.c_int
_lib.pdn_noalloc_scratch_bytes.argtypes = []
_lib.pdn_noalloc_scratch_bytes.restype = ctypes.c_size_t
_lib.pdn_status_string.argtypes = [ctypes.c_int]
_lib.pdn_status_string.restype = ctypes.c_char_p
_lib.pdn_abi_version.argtypes = []
_lib.pdn_abi_version.restype = ctypes.c_int
_lib.pdn_scan_segments.argtypes = [ctypes.POINTER(Problem),
                                   ctypes.POINTER(ctypes.c_int)]
_lib.pdn_scan_segments.restype = ctypes.c_int

ABI_VERSION = 7   # PDN_ABI_VERSION: the struct layouts mirrored above
if _lib.pdn_abi_version() != ABI_VERSION:
    raise ImportError(f"{LIB_PATH} implements ABI version "
                      f"{_lib.pdn_abi_version()}, this binding mirrors "
                      f"version {ABI_VERSION}: rebuild the library")

EXPORTED = ("pdn_workspace_size", "pdn_chunk_fwd", "pdn_chunk_fwd_events",
            "pdn_chunk_bwd", "pdn_chunk_bwd_events", "pdn_chunk_fwd_train",
            "pdn_chunk_bwd_train", "pdn_chunk_fwd_noalloc",
            "pdn_noalloc_scratch_bytes", "pdn_status_string",
            "pdn_abi_version", "pdn_scan_segments", "pdn_slot_fwd",
            "pdn_slot_draft", "pdn_draft_verify",
            "pdn_draft_verify_workspace_size", "pdn_residual_norm",
            "pdn_residual_norm_bwd", "pdn_residual_norm_bwd_workspace_size",
            "pdn_head_norm", "pdn_head_norm_bwd",
            "pdn_head_norm_bwd_workspace_size", "pdn_logits",
            "pdn_logits_workspace_size", "pdn_token_counts")
FWD_STAGE_EVENTS = 4   # PDN_FWD_STAGE_EVENTS
BWD_STAGE_EVENTS = 7   # PDN_BWD_STAGE_EVENTS
FWD_STAGES = ("precond", "chunk_prep", "chunk_scan")
BWD_STAGES = ("bwd_precond_recompute", "bwd_chunk_prep", "bwd_state_save_scan",
              "bwd_state_adjoint_scan", "bwd_chunk_grads", "bwd_precond_reverse")


class PdnError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {pdn_status_string(status)} "
                         f"(status {status})")


def pdn_status_string(status: int) -> str:
    return _lib.pdn_status_string(int(status)).decode()


def pdn_abi_version() -> int:
    return _lib.pdn_abi_version()


def make_problem(B, T, H, dk, dv, *, io="bf16", gate="none",
                 precond="squash", x=1.5, scale=1.0, chunk=64,
                 ridge=1.0, knorm="none") -> Problem:
    return Problem(B, T, H, dk, dv, chunk,
                   PDN_BF16 if io == "bf16" else PDN_F32,
                   GATES[gate] if isinstance(gate, str) else int(gate),
                   PRECONDS[precond] if isinstance(precond, str)
                   else int(precond), x, scale, ridge,
                   KNORMS[knorm] if isinstance(knorm, str) else int(knorm))


def pdn_workspace_size(problem: Problem, with_bwd: bool = False) -> int:
    n = ctypes.c_size_t(0)
    st = _lib.pdn_workspace_size(ctypes.byref(problem), int(with_bwd),
                                 ctypes.byref(n))
    if st != PDN_OK:
        raise PdnError(st, "pdn_workspace_size")
    return n.value


def pdn_scan_segments(problem: Problem) -> int:
    n = ctypes.c_int(0)
    st = _lib.pdn_scan_segments(ctypes.byref(problem), ctypes.byref(n))
    if st != PDN_OK:
        raise PdnError(st, "pdn_scan_segments")
    return n.value


# ------------------------------------------------------- raw pointer calls
def pdn_chunk_fwd_raw(problem: Problem, inputs: Inputs, out: FwdOut, ws: int,
                      ws_bytes: int, stream: int) -> int:
    """Direct call with raw pointers; returns the status code."""
    return _lib.pdn_chunk_fwd(ctypes.byref(problem), ctypes.byref(inputs),
                              ctypes.byref(out), ws, ws_bytes, stream)


def pdn_chunk_fwd_events_raw(problem: Problem, inputs: Inputs, out: FwdOut,
                             ws: int, ws_bytes: int, stream: int,
                             events) -> int:
    """pdn_chunk_fwd_events with raw hipEvent_t handles (ints)."""
    arr = (_vp * len(events))(*events)
    return _lib.pdn_chunk_fwd_events(ctypes.byref(problem),
                                     ctypes.byref(inputs), ctypes.byref(out),
                                     ws, ws_bytes, stream, arr, len(events))


def pdn_chunk_fwd_noalloc_raw(problem: Problem, inputs: Inputs, out: FwdOut,
                              stream: int) -> int:
    """pdn_chunk_fwd_noalloc with raw pointers; returns the status code."""
    return _lib.pdn_chunk_fwd_noalloc(ctypes.byref(problem),
                                      ctypes.byref(inputs), ctypes.byref(out),
                                      stream)


def pdn_noalloc_scratch_bytes() -> int:
    return _lib.pdn_noalloc_scratch_bytes()


def pdn_chunk_bwd_raw(problem: Problem, inputs: Inputs, dO: int, dS_T: int,
                      out: BwdOut, ws: int, ws_bytes: int,
                      stream: int) -> int:
    return _lib.pdn_chunk_bwd(ctypes.byref(problem), ctypes.byref(inputs), dO,
                              dS_T, ctypes.byref(out), ws, ws_bytes, stream)


# ------------------------------------------------------- torch marshalling
def _ptr(t):
    if t is None:
        return None
    if not t.is_contiguous():
        raise ValueError("tensors passed to libpdn must be contiguous")
    return t.data_ptr()


def _io_of(t):
    import torch
    if t.dtype == torch.bfloat16:
        return "bf16"
    if t.dtype == torch.float32:
        return "f32"
    raise TypeError(f"q/k/v must be float32 or bfloat16, got {t.dtype}")


def _stream(stream, device):
    import torch
    s = stream if stream is not None else torch.cuda.current_stream(device)
    return s.cuda_stream


def _inputs(q, k, v, beta, g, beta_p, g_p, log_a_scale, A0, S0, ktilde):
    return Inputs(*[_ptr(t) for t in (q, k, v, beta, g, beta_p, g_p,
                                      log_a_scale, A0, S0, ktilde)])


def pdn_chunk_fwd(q, k, v, beta, *, g=None, gate="none", precond="squash",
                  beta_p=None, g_p=None, log_a_scale=None, A0=None, S0=None,
                  ktilde=None, x=1.5, scale=1.0, chunk=64, ridge=1.0,
                  knorm="none", o=None, S_T=None, A_T=None, want_state=True,
                  workspace=None, stream=None, stage_events=None,
                  train=False):
    """Forward pass on torch device tensors in the ABI layouts of pdn.h.

    Returns (o, S_T, A_T); S_T / A_T are None when not requested.  Outputs and
    the workspace are allocated with torch when not given.  stage_events: 4
    recorded-at-stage-boundary torch.cuda.Event objects (see
    pdn_chunk_fwd_events), or None.  train=True runs pdn_chunk_fwd_train:
    the workspace (then of the backward's size, and required) keeps the
    intermediates pdn_chunk_bwd(..., saved=True) reads."""
    import torch
    B, T, H, dk = q.shape
    dv = v.shape[-1]
    io = _io_of(q)
    prob = make_problem(B, T, H, dk, dv, io=io, gate=gate, precond=precond,
                        x=x, scale=scale, chunk=chunk, ridge=ridge,
                        knorm=knorm)
    dev = q.device
    if o is None:
        o = torch.empty((B, T, H, dv), dtype=q.dtype, device=dev)
    if S_T is None and want_state:
        S_T = torch.empty((B, H, dk, dv), dtype=torch.float32, device=dev)
    if A_T is None and want_state and precond in GRAM_PRECONDS:
        A_T = torch.empty((B, H, dk), dtype=torch.float32, device=dev)
    nbytes = pdn_workspace_size(prob, train)
    if workspace is None:
        if train:
            raise ValueError("train=True needs the caller's workspace (it "
                             "carries the intermediates to the backward)")
        workspace = torch.empty(max(nbytes, 1), dtype=torch.uint8, device=dev)
    inp = _inputs(q, k, v, beta, g, beta_p, g_p, log_a_scale, A0, S0, ktilde)
    out = FwdOut(_ptr(o), _ptr(S_T), _ptr(A_T))
    if train:
        evs = [_event_handle(e) if e is not None else None
               for e in (stage_events or [])]
        arr = (_vp * len(evs))(*evs) if evs else None
        st = _lib.pdn_chunk_fwd_train(
            ctypes.byref(prob), ctypes.byref(inp), ctypes.byref(out),
            _ptr(workspace), workspace.numel(), _stream(stream, dev), arr,
            len(evs))
    elif stage_events is None:
        st = pdn_chunk_fwd_raw(prob, inp, out, _ptr(workspace),
                               workspace.numel(), _stream(stream, dev))
    else:
        st = pdn_chunk_fwd_events_raw(
            prob, inp, out, _ptr(workspace), workspace.numel(),
            _stream(stream, dev),
            [_event_handle(e) if e is not None else None for e in stage_events])
    if st != PDN_OK:
        raise PdnError(st, "pdn_chunk_fwd")
    return o, S_T, A_T


def pdn_chunk_fwd_noalloc(q, k, v, beta, *, o, g=None, gate="none",
                          precond="squash", beta_p=None, g_p=None,
                          log_a_scale=None, A0=None, S0=None, ktilde=None,
                          x=1.5, scale=1.0, chunk=64, ridge=1.0,
                          knorm="none", S_T=None, A_T=None, stream=None):
    """pdn_chunk_fwd through the no-allocation entry point: the caller passes
    every output (o required, S_T / A_T optional) and no workspace; the
    library uses its fixed per-device scratch.  Returns (o, S_T, A_T)."""
    B, T, H, dk = q.shape
    dv = v.shape[-1]
    prob = make_problem(B, T, H, dk, dv, io=_io_of(q), gate=gate,
                        precond=precond, x=x, scale=scale, chunk=chunk,
                        ridge=ridge, knorm=knorm)
    inp = _inputs(q, k, v, beta, g, beta_p, g_p, log_a_scale, A0, S0, ktilde)
    out = FwdOut(_ptr(o), _ptr(S_T), _ptr(A_T))
    st = pdn_chunk_fwd_noalloc_raw(prob, inp, out, _stream(stream, q.device))
    if st != PDN_OK:
        raise PdnError(st, "pdn_chunk_fwd_noalloc")
    return o, S_T, A_T


def _event_handle(ev):
    """Raw hipEvent_t of a torch.cuda.Event (created on first use)."""
    if ev.cuda_event == 0:
        import torch
        ev.record(torch.cuda.current_stream())   # forces creation
    return ev.cuda_event


def pdn_chunk_bwd(q, k, v, beta, dO, *, g=None, gate="none", precond="squash",
                  beta_p=None, g_p=None, log_a_scale=None, A0=None, S0=None,
                  ktilde=None, dS_T=None, x=1.5, scale=1.0, chunk=64,
                  outputs=None, want_optional=True, workspace=None,
                  stream=None, stage_events=None, saved=False):
    """Backward pass on torch device tensors (layouts of pdn.h).

    Returns a dict with dq, dk, dv, dbeta and, when present, dg, dS0 and the
    preconditioner gradients dbeta_p, dg_p, dlog_a_scale, dA0 (squash) or
    dktilde (external).  Outputs and the workspace are allocated with torch
    when not given (``outputs``: dict of preallocated tensors).  saved=True
    runs pdn_chunk_bwd_train on the intermediates a preceding
    pdn_chunk_fwd(..., train=True) left in ``workspace``."""
    import torch
    B, T, H, dk = q.shape
    dv = v.shape[-1]
    io = _io_of(q)
    prob = make_problem(B, T, H, dk, dv, io=io, gate=gate, precond=precond,
                        x=x, scale=scale, chunk=chunk)
    dev = q.device
    f32 = torch.float32
    out = dict(outputs or {})

    def need(name, shape, dtype):
        if name not in out:
            out[name] = torch.empty(shape, dtype=dtype, device=dev)

    need("dq", (B, T, H, dk), q.dtype)
    need("dk", (B, T, H, dk), q.dtype)
    need("dv", (B, T, H, dv), q.dtype)
    need("dbeta", (B, T, H), f32)
    if gate != "none":
        need("dg", tuple(g.shape), f32)
    if want_optional:
        need("dS0", (B, H, dk, dv), f32)
        if precond == "squash":
            need("dbeta_p", (B, T, H), f32)
            need("dg_p", (B, T, H), f32)
            need("dlog_a_scale", (H,), f32)
            need("dA0", (B, H, dk), f32)
        if precond == "external":
            need("dktilde", (B, T, H, dk), q.dtype)
    nbytes = pdn_workspace_size(prob, True)
    if workspace is None:
        if saved:
            raise ValueError("saved=True needs the training forward's workspace")
        workspace = torch.empty(max(nbytes, 1), dtype=torch.uint8, device=dev)
    inp = _inputs(q, k, v, beta, g, beta_p, g_p, log_a_scale, A0, S0, ktilde)
    bo = BwdOut(*[_ptr(out.get(n)) for n, _ in BwdOut._fields_])
    if saved:
        evs = [_event_handle(e) if e is not None else None
               for e in (stage_events or [])]
        arr = (_vp * len(evs))(*evs) if evs else None
        st = _lib.pdn_chunk_bwd_train(
            ctypes.byref(prob), ctypes.byref(inp), _ptr(dO), _ptr(dS_T),
            ctypes.byref(bo), _ptr(workspace), workspace.numel(),
            _stream(stream, dev), arr, len(evs))
    elif stage_events is None:
        st = pdn_chunk_bwd_raw(prob, inp, _ptr(dO), _ptr(dS_T), bo,
                               _ptr(workspace), workspace.numel(),
                               _stream(stream, dev))
    else:
        evs = [_event_handle(e) if e is not None else None
               for e in stage_events]
        arr = (_vp * len(evs))(*evs)
        st = _lib.pdn_chunk_bwd_events(
            ctypes.byref(prob), ctypes.byref(inp), _ptr(dO), _ptr(dS_T),
            ctypes.byref(bo), _ptr(workspace), workspace.numel(),
            _stream(stream, dev), arr, len(evs))
    if st != PDN_OK:
        raise PdnError(st, "pdn_chunk_bwd")
    return out


# ------------------------------------------------------- states in a pool
# These calls run once a token, so checks and marshalling are compiled
# (csrc/pdn_torch.cpp): a decode call takes the host 7 us, the launch included.
def _address(fn):
    return ctypes.cast(fn, _vp).value


_SLOT_FWD, _SLOT_DRAFT, _VERIFY, _VERIFY_SIZE = map(_address, (
    _lib.pdn_slot_fwd, _lib.pdn_slot_draft, _lib.pdn_draft_verify,
    _lib.pdn_draft_verify_workspace_size))


def _call_on(where, device, stream, fn, *args):
    """fn(*args, stream) with `device` current, and `stream` too where one is
    named: what the call allocates is then that stream's memory, and what is
    freed while it runs goes to that stream's next tensors, not to another's."""
    if stream is not None:
        if stream.device != device:
            raise ValueError(f"the stream is on {stream.device}, not on {device}")
        with torch.cuda.stream(stream):
            out = fn(*args, stream.cuda_stream)
    elif device.type != "cuda" or torch._C._cuda_getDevice() == device.index:
        out = fn(*args, torch._C._cuda_getCurrentRawStream(device.index or 0)
                 if device.type == "cuda" else 0)
    else:
        with torch.cuda.device(device):
            out = fn(*args, torch._C._cuda_getCurrentRawStream(device.index))
    if type(out) is int:
        raise PdnError(out, where)
    return out


def pdn_tape_record(dk, dv, gate="none", precond="squash") -> int:
    """Elements of a pending token's record for one head (see pdn_slots)."""
    return (dk + dv + (dk if gate == "channel" else 4)
            + (dk if precond in GRAM_PRECONDS else 0))


def pdn_slot_fwd(q, k, v, beta, S, *, starts=None, slots=None, slots_out=None,
                 fresh=None, max_tokens=None, g=None, gate="none",
                 precond="squash", beta_p=None, g_p=None, log_a_scale=None,
                 A=None, ktilde=None, x=1.5, scale=1.0, ridge=1.0,
                 knorm="none", o=None, stream=None):
    """Advance states of a pool over packed sequences (pdn_slot_fwd of pdn.h).

    q, k [tokens, Hk, dk] and v [tokens, H, dv], rows of any token stride
    that keeps them apart (slices of one projection); S [slots, H, dk, dv] and A [slots, H, dk] are
    read and written in place.  starts [N + 1], slots, slots_out, fresh [N]:
    int32 on the device.  Without starts the rows are shared evenly
    by the sequences (one row each without slots too).  max_tokens: the most
    rows a sequence has (default: unknown, at most all; worth giving, as one
    row or a few take leaner kernels).  Returns o."""
    return _call_on(
        "pdn_slot_fwd", S.device, stream, _pdn_torch.slot, _SLOT_FWD, q, k, v,
        beta, S, None, None, None, 0, starts, slots, slots_out, fresh,
        max_tokens, g, GATES[gate], PRECONDS[precond], beta_p, g_p,
        log_a_scale, A, ktilde, x, scale, ridge, KNORMS[knorm], o)


def pdn_slot_draft(q, k, v, beta, S, tape, pending, *, accepted=None,
                   starts=None, slots=None, slots_out=None, fresh=None,
                   max_tokens=None, g=None, gate="none", precond="squash",
                   beta_p=None, g_p=None, log_a_scale=None, A=None,
                   ktilde=None, x=1.5, scale=1.0, ridge=1.0, knorm="none",
                   o=None, stream=None):
    """Score drafted tokens on states of a pool (pdn_slot_draft of pdn.h).

    The tokens the last call left pending are applied as far as `accepted`
    ([N] int32, e.g. of pdn_draft_verify) says, then the new ones are scored
    and left pending.  tape: [slots, most tokens, H, pdn_tape_record(...)]
    fp32; pending: [slots, H] int32, zero at first.  max_tokens defaults to what
    the tape holds.  The rest as in pdn_slot_fwd.  Returns o."""
    if tape.dim() != 4:
        raise ValueError("tape must be [slots, tokens, H, record]")
    if max_tokens is None and starts is not None:
        max_tokens = tape.shape[1]
    return _call_on(
        "pdn_slot_draft", S.device, stream, _pdn_torch.slot, _SLOT_DRAFT, q, k,
        v, beta, S, tape, pending, accepted,
        pdn_tape_record(*S.shape[-2:], gate, precond), starts, slots,
        slots_out, fresh, max_tokens, g, GATES[gate], PRECONDS[precond],
        beta_p, g_p, log_a_scale, A, ktilde, x, scale, ridge, KNORMS[knorm], o)


def pdn_draft_verify_workspace_size(N: int, V: int) -> int:
    n = ctypes.c_size_t(0)
    st = _lib.pdn_draft_verify_workspace_size(N, V, ctypes.byref(n))
    if st != PDN_OK:
        raise PdnError(st, "pdn_draft_verify_workspace_size")
    return n.value


def pdn_draft_verify(p, ids, u, r, *, q=None, starts=None, accepted=None,
                     token=None, workspace=None, stream=None):
    """Verify drafted tokens against the target's probabilities
    (pdn_draft_verify of pdn.h).

    p, q: [rows, V], fp32 or bf16; ids [rows] int32, the tokens fed; u [rows],
    r [N] fp32 in [0, 1).  Returns (accepted, token), int32 [N]: the rows that hold
    (what pdn_slot_draft applies) and the token after them."""
    return _call_on(
        "pdn_draft_verify", p.device, stream, _pdn_torch.verify, _VERIFY,
        _VERIFY_SIZE, p, q, ids, u, r, starts, accepted, token, workspace)


# ------------------------------------------------- around the rule in a block
(_RNORM, _RNORM_BWD, _RNORM_SIZE, _HNORM, _HNORM_BWD, _HNORM_SIZE, _LOGITS,
 _LOGITS_SIZE, _COUNTS) = map(_address, (
     _lib.pdn_residual_norm, _lib.pdn_residual_norm_bwd,
     _lib.pdn_residual_norm_bwd_workspace_size, _lib.pdn_head_norm,
     _lib.pdn_head_norm_bwd, _lib.pdn_head_norm_bwd_workspace_size,
     _lib.pdn_logits, _lib.pdn_logits_workspace_size, _lib.pdn_token_counts))


def _dtype_number(dtype):
    if dtype is None:
        return -1
    if dtype == torch.float32:
        return PDN_F32
    if dtype == torch.bfloat16:
        return PDN_BF16
    raise TypeError(f"tensors must be float32 or bfloat16, got {dtype}")


def _act(act, z):
    return ACTS[act if act is not None else "none" if z is None else "silu"]


def pdn_residual_norm(y, residual=None, *, weight=None, post_norm=False,
                      post_weight=None, scale=None, alpha=1.0, eps=1e-6,
                      h_dtype=None, want_h=True, u=None, h=None, stream=None):
    """A block's output y joins the residual stream, and the next block's input
    is the norm of the sum (pdn_residual_norm of pdn.h):

      h = residual + alpha * scale * (y, or RMSNorm(y) * post_weight)
      u = RMSNorm(h) * weight

    y, u: [..., D]; residual, h of their own dtype (an fp32 stream, say);
    weight, post_weight, scale: [D] fp32 or None (= 1).  Without a residual
    h_dtype (default: y's) names h's.  h may be residual itself.  Returns
    (u, h); h is None with want_h=False."""
    return _call_on(
        "pdn_residual_norm", y.device, stream, _pdn_torch.residual_norm,
        _RNORM, y, residual, weight, post_weight, scale, post_norm, alpha, eps,
        _dtype_number(h_dtype), want_h, u, h)


def pdn_residual_norm_bwd_workspace_size(rows: int, D: int) -> int:
    """Bytes for gradients of vectors (none are needed without)."""
    n = ctypes.c_size_t(0)
    p = Rnorm(rows=rows, D=D, alpha=1.0, eps=1.0)
    st = _lib.pdn_residual_norm_bwd_workspace_size(ctypes.byref(p),
                                                   ctypes.byref(n))
    if st != PDN_OK:
        raise PdnError(st, "pdn_residual_norm_bwd_workspace_size")
    return n.value


def pdn_residual_norm_bwd(du, h, y=None, *, dh=None, weight=None,
                          post_norm=False, post_weight=None, scale=None,
                          alpha=1.0, eps=1e-6, outputs=None,
                          want_residual=True, want_vectors=True,
                          workspace=None, stream=None):
    """Gradients of <du, u> + <dh, h> of pdn_residual_norm, from the h that
    it returned; y where it was normed or scaled.  Returns a dict of dy,
    dresidual and, of the vectors given, dweight, dpost_weight, dscale.
    ``outputs``: dict of preallocated tensors (dresidual may be dh)."""
    out = outputs or {}
    return _call_on(
        "pdn_residual_norm_bwd", du.device, stream,
        _pdn_torch.residual_norm_bwd, _RNORM_BWD, _RNORM_SIZE, du, h, y, dh,
        weight, post_weight, scale, post_norm, alpha, eps, want_residual,
        want_vectors, out.get("dy"), out.get("dresidual"), out.get("dweight"),
        out.get("dpost_weight"), out.get("dscale"), workspace)


def pdn_head_norm(x, *, norm="rms", weight=None, z=None, act=None, eps=1e-6,
                  y=None, stream=None):
    """Norm over each head's channels, with a weight and an output gate
    (pdn_head_norm of pdn.h): norm(x) * weight * act(z).

    x, z, y: [..., H, d], tokens' rows of any even spacing (slices of one
    projection); norm "rms", or "l2" for unit queries and keys; weight [d] or
    [H, d] fp32; act "silu" (default where z is given) or "sigmoid".  y may be
    x itself.  Returns y."""
    return _call_on(
        "pdn_head_norm", x.device, stream, _pdn_torch.head_norm, _HNORM, x,
        NORMS[norm], weight, z, _act(act, z), eps, y)


def pdn_head_norm_bwd_workspace_size(tokens: int, H: int, d: int,
                                     head_weight: bool = False) -> int:
    """Bytes for a weight's gradient (none are needed without); head_weight: of
    a weight [H, d]."""
    n = ctypes.c_size_t(0)
    p = Hnorm(tokens=tokens, H=H, d=d, head_weight=head_weight, eps=1.0)
    st = _lib.pdn_head_norm_bwd_workspace_size(ctypes.byref(p),
                                               ctypes.byref(n))
    if st != PDN_OK:
        raise PdnError(st, "pdn_head_norm_bwd_workspace_size")
    return n.value


def pdn_head_norm_bwd(dy, x, *, norm="rms", weight=None, z=None, act=None,
                      eps=1e-6, outputs=None, want_vectors=True,
                      workspace=None, stream=None):
    """Gradients of <dy, y> of pdn_head_norm.  Returns a dict of dx and, where
    there is a gate and a weight, dz and dweight.  ``outputs``: dict of
    preallocated tensors, rows spaced like x's may be (dx may be dy)."""
    out = outputs or {}
    return _call_on(
        "pdn_head_norm_bwd", x.device, stream, _pdn_torch.head_norm_bwd,
        _HNORM_BWD, _HNORM_SIZE, dy, x, NORMS[norm], weight, z, _act(act, z),
        eps, want_vectors, out.get("dx"), out.get("dz"), out.get("dweight"),
        workspace)


def pdn_logits_workspace_size(rows: int, V: int) -> int:
    n = ctypes.c_size_t(0)
    st = _lib.pdn_logits_workspace_size(rows, V, ctypes.byref(n))
    if st != PDN_OK:
        raise PdnError(st, "pdn_logits_workspace_size")
    return n.value


def pdn_logits(logits, *, probs=True, temperature=None, repetition=None,
               presence=None, frequency=None, counts=None, slots=None,
               ids=None, starts=None, bias=None, mask=None, mask_rows=None,
               dtype=None, out=None, workspace=None, stream=None):
    """Logits to the probabilities that pdn_draft_verify reads (pdn_logits of
    pdn.h): penalties for repeated tokens, biases, grammar masks, softmax.

    logits: [rows, V], rows of any spacing; starts [N + 1], slots [N]: the
    packed sequences and their rows of counts [slots, V] (int32, see
    pdn_token_counts); ids [rows]: the tokens fed, not counted yet;
    temperature (0: the largest logit), repetition, presence, frequency: [N]
    fp32; bias: (starts [N + 1], ids, values), lists of tokens and what is added
    to their logits; mask: [masks, (V + 31) // 32] int32, a bit a token that is
    allowed, mask_rows [rows] the mask of each row (-1: none).  Without starts
    the rows are shared evenly by the sequences.  probs=False: the changed logits
    themselves.  dtype: of the result (default fp32, of logits theirs); out may be
    the logits.  Returns [rows, V]."""
    bias = bias if bias is not None else (None, None, None)
    if len(bias) != 3:
        raise ValueError("bias must be (starts, ids, values)")
    return _call_on(
        "pdn_logits", logits.device, stream, _pdn_torch.logits, _LOGITS,
        _LOGITS_SIZE, logits, probs, temperature, repetition, presence,
        frequency, counts, slots, ids, starts, *bias, mask, mask_rows, out,
        _dtype_number(dtype), workspace)


def pdn_token_counts(ids, counts, *, starts=None, slots=None, slots_out=None,
                     fresh=None, accepted=None, prompt=False, stream=None):
    """Add tokens to the table of counts that pdn_logits reads
    (pdn_token_counts of pdn.h): counts [slots, V] int32, zero at first.

    ids: packed tokens; of each sequence the first accepted[n] (None: all) are
    added to its row slots[n], as generated, or with prompt=True as the
    prompt's.  fresh[n] non-zero: the row is cleared first; slots_out: the rows are
    written there (a fork).  Returns counts."""
    return _call_on(
        "pdn_token_counts", counts.device, stream, _pdn_torch.token_counts,
        _COUNTS, ids, counts, starts, slots, slots_out, fresh, accepted, prompt)
