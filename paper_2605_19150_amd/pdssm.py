"""Thin ctypes binding of libpdssm.so (the C ABI declared in include/pdssm.h).

Only argument marshalling happens here: shape/dtype/device checks, output and
workspace allocation with torch, and passing raw device pointers plus the
current HIP stream to the library.  Every step of the scan runs in the HIP
kernels.  If the library is missing the binding raises; there is no fallback.

Tensor layouts (all contiguous, on one GPU):
  idx [B,L,H] int32, pi [H,K,N] int32, D/b/c [B,L,H,N] complex64,
  h0/h_final/dh_final/dh0 [B,H,N] complex64, y/dy [B,L,H] float32,
  saved [B,H,C,N] complex64 (C = num_chunks).
With bf16 I/O (FLAG_BF16_IO), D, b, c and dD, db, dc are bfloat16 tensors
  [B,L,H,N,2] holding (re, im) (torch.view_as_real(x).to(torch.bfloat16)).
The real-valued model (FLAG_REAL_IO): D, b, c, dD, db, dc and saved are
  float32 ([B,L,H,N], saved [B,H,C,N]: the states are real); h0, dh_final,
  h_final and dh0 stay complex64 (scan_fwd and scan_bwd also take a real
  float32 h0 / dh_final and widen it).
Straight-through surrogate gradients (Sec. 3.1 Prop. 2): q [B,L,H,K] float32,
  z [B,L,H,N] complex64, G [H,K,N,N] float32, routing logits [B,L,H,K] and
  dense dictionary M [H,K,N,N] float32.
Gated recurrent layers (gated_fwd and the functions after it) take rows:
  x, ga, gi, dy [B,L,C] for B sequences of one length, or [T,C] with the
  sequences' bounds cu [S+1] int32; float32 or bfloat16, rows at one pitch
  (parts of wider rows, not the first rows of each of several longer sequences)
  of at most 2^24 entries, entries of a row next to each other.  rate [C] and
  the states [S,C] are float32.  What is returned for rows behind the last sequence
  (cu[S] < T) is zero.  Activations in the 8-bit form are pairs (q, e): int8
  [T,C] and [ceil(T/32),C].
Linear attention (decay_attn_fwd and the functions after it) takes heads' rows
  q [B,L,Hq,Dk], k [B,L,Hk,Dk], v [B,L,Hv,Dv], or [T,heads,D] with cu; float32 or
  bfloat16, parts of wider rows too (any steps from row to row and head to head,
  the rows of a batch evenly spaced).  rate [H] and the states [S,H,Dk,Dv] are
  float32; Hq, Hk and Hv divide H.  Group norm takes rows as the gated layers do.
The functions of both kinds of layers run on the current stream of the
  tensors' device, or on the one given as stream, behind what the current stream
  has to do; who reads the results on another stream has to wait for that one.
"""
import ctypes
import functools
import inspect
import math
import os
import struct

import torch

_LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libpdssm.so")
_lib = None

OK, ERR_INVALID_ARG, ERR_UNSUPPORTED, ERR_WORKSPACE, ERR_HIP, ERR_INDEX = 0, -1, -2, -3, -4, -5
OP_FWD, OP_BWD, OP_COMPOSE, OP_STE_GRADS = 1, 2, 3, 4
FLAG_PREPARED = 1
FLAG_BF16_IO = 2
FLAG_REAL_IO = 4
FLAG_ZERO_REST = 8  # gated_fwd, gated_bwd: rows behind the last sequence are written, as zeros


class PdssmError(RuntimeError):
    def __init__(self, status, what):
        super().__init__("%s: %s" % (what, status_string(status)))
        self.status = status


class Desc(ctypes.Structure):
    _fields_ = [("B", ctypes.c_int32), ("L", ctypes.c_int32), ("H", ctypes.c_int32),
                ("N", ctypes.c_int32), ("K", ctypes.c_int32), ("chunk", ctypes.c_int32),
                ("flags", ctypes.c_uint32)]


class Rows(ctypes.Structure):
    _fields_ = [("p", ctypes.c_void_p), ("ld", ctypes.c_int64), ("e", ctypes.c_void_p)]


class Heads(ctypes.Structure):
    _fields_ = [("p", ctypes.c_void_p), ("ld", ctypes.c_int64), ("hs", ctypes.c_int64)]


class AttnDesc(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("T", "S", "H", "Hq", "Hk", "Hv", "Dk", "Dv")] + [
        ("scale", ctypes.c_float), ("flags", ctypes.c_uint32)]


class NormDesc(ctypes.Structure):
    _fields_ = [("T", ctypes.c_int32), ("C", ctypes.c_int32), ("G", ctypes.c_int32), ("act", ctypes.c_int32),
                ("eps", ctypes.c_float), ("flags", ctypes.c_uint32)]


class GatedDesc(ctypes.Structure):
    _fields_ = [("T", ctypes.c_int32), ("C", ctypes.c_int32), ("S", ctypes.c_int32), ("flags", ctypes.c_uint32)]


EXPORTS = ("pdssm_abi_version", "pdssm_chunk_len", "pdssm_num_chunks", "pdssm_workspace_size",
           "pdssm_uses_fused", "pdssm_scan_segments", "pdssm_status_string", "pdssm_prepare", "pdssm_scan_fwd", "pdssm_scan_fwd_noalloc",
           "pdssm_scan_bwd", "pdssm_compose_chunks", "pdssm_scan_bwd_ste", "pdssm_ste_grads",
           "pdssm_softmax_vjp", "pdssm_decode_step", "pdssm_dict_argmax", "pdssm_route", "pdssm_project",
           "pdssm_gated_workspace_size", "pdssm_gated_fwd", "pdssm_gated_bwd", "pdssm_gated_step", "pdssm_pack8",
           "pdssm_unpack8", "pdssm_project_wgrad_workspace_size", "pdssm_project_wgrad",
           "pdssm_decay_attn_workspace_size", "pdssm_decay_attn_fwd", "pdssm_decay_attn_bwd", "pdssm_decay_attn_step",
           "pdssm_group_norm", "pdssm_group_norm_workspace_size", "pdssm_group_norm_bwd")


def lib_path():
    return _LIB_PATH


def load():
    """Load libpdssm.so once (raises if it has not been built)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(_LIB_PATH):
        raise ImportError("libpdssm.so is not built (%s); run __graft_entry__.build()" % _LIB_PATH)
    L = ctypes.CDLL(_LIB_PATH)
    P, I, Z = ctypes.c_void_p, ctypes.c_int, ctypes.c_size_t
    D = ctypes.POINTER(Desc)
    L.pdssm_abi_version.argtypes, L.pdssm_abi_version.restype = [], I
    L.pdssm_chunk_len.argtypes, L.pdssm_chunk_len.restype = [D], I
    L.pdssm_num_chunks.argtypes, L.pdssm_num_chunks.restype = [D], I
    L.pdssm_workspace_size.argtypes, L.pdssm_workspace_size.restype = [D, I], Z
    L.pdssm_status_string.argtypes, L.pdssm_status_string.restype = [I], ctypes.c_char_p
    L.pdssm_uses_fused.argtypes, L.pdssm_uses_fused.restype = [D], I
    L.pdssm_scan_segments.argtypes, L.pdssm_scan_segments.restype = [D], I
    L.pdssm_prepare.argtypes, L.pdssm_prepare.restype = [D, P, P, Z, P, P], I
    L.pdssm_scan_fwd.argtypes = [D] + [P] * 10 + [Z, P, P]
    L.pdssm_scan_fwd.restype = I
    L.pdssm_scan_fwd_noalloc.argtypes = [D] + [P] * 11
    L.pdssm_scan_fwd_noalloc.restype = I
    L.pdssm_scan_bwd.argtypes = [D] + [P] * 13 + [Z, P, P]
    L.pdssm_scan_bwd.restype = I
    L.pdssm_compose_chunks.argtypes = [D] + [P] * 7
    L.pdssm_compose_chunks.restype = I
    L.pdssm_scan_bwd_ste.argtypes = [D] + [P] * 14 + [Z, P, P]
    L.pdssm_scan_bwd_ste.restype = I
    L.pdssm_ste_grads.argtypes = [D] + [P] * 7 + [Z, P, P]
    L.pdssm_ste_grads.restype = I
    L.pdssm_softmax_vjp.argtypes = [P, P, P, ctypes.c_int64, ctypes.c_int32, ctypes.c_int64,
                                    ctypes.c_float, P]
    L.pdssm_softmax_vjp.restype = I
    L.pdssm_decode_step.argtypes = [D] + [P] * 10
    L.pdssm_decode_step.restype = I
    I32 = ctypes.c_int32
    L.pdssm_dict_argmax.argtypes = [I32, I32, I32, P, P, P]
    L.pdssm_dict_argmax.restype = I
    L.pdssm_route.argtypes = [I32, I32, I32, I32, P, P, P, P, P]
    L.pdssm_route.restype = I
    L.pdssm_project.argtypes = [I32] * 5 + [P] * 10 + [P]
    L.pdssm_project.restype = I
    U32, I64, V3 = ctypes.c_uint32, ctypes.c_int64, ctypes.POINTER(ctypes.c_void_p)
    G, R = P, P  # GatedDesc and Rows, by address
    L.pdssm_gated_workspace_size.argtypes, L.pdssm_gated_workspace_size.restype = [G, I], Z
    L.pdssm_gated_fwd.argtypes = [G, R, R, R] + [P] * 6 + [V3, V3, P, Z, P, P]
    L.pdssm_gated_fwd.restype = I
    L.pdssm_gated_bwd.argtypes = [G, R, R, R] + [P] * 4 + [R, P, V3, I64] + [P] * 3 + [Z, P, P]
    L.pdssm_gated_bwd.restype = I
    L.pdssm_gated_step.argtypes = [G, R, R, R] + [P] * 7
    L.pdssm_gated_step.restype = I
    L.pdssm_pack8.argtypes, L.pdssm_pack8.restype = [I32, I32, U32, R, P, P, P], I
    L.pdssm_unpack8.argtypes, L.pdssm_unpack8.restype = [I32, I32, U32, P, P, P, P], I
    L.pdssm_project_wgrad_workspace_size.argtypes, L.pdssm_project_wgrad_workspace_size.restype = [I32] * 3, Z
    L.pdssm_project_wgrad.argtypes, L.pdssm_project_wgrad.restype = [I32] * 3 + [P] * 5 + [Z, P], I
    L.pdssm_decay_attn_workspace_size.argtypes, L.pdssm_decay_attn_workspace_size.restype = [P, I, I], Z
    L.pdssm_decay_attn_fwd.argtypes, L.pdssm_decay_attn_fwd.restype = [P] * 10 + [Z, P, P], I
    L.pdssm_decay_attn_bwd.argtypes, L.pdssm_decay_attn_bwd.restype = [P] * 14 + [Z, P, P], I
    L.pdssm_decay_attn_step.argtypes, L.pdssm_decay_attn_step.restype = [P] * 11, I
    L.pdssm_group_norm.argtypes, L.pdssm_group_norm.restype = [P] * 7, I
    L.pdssm_group_norm_workspace_size.argtypes, L.pdssm_group_norm_workspace_size.restype = [P], Z
    L.pdssm_group_norm_bwd.argtypes, L.pdssm_group_norm_bwd.restype = [P] * 11 + [Z, P], I
    if L.pdssm_abi_version() != 1:
        raise ImportError("libpdssm.so ABI version mismatch")
    _lib = L
    return L


def status_string(st):
    return load().pdssm_status_string(int(st)).decode()


def desc(B, L, H, N, K, chunk=0):
    return Desc(int(B), int(L), int(H), int(N), int(K), int(chunk), 0)


def scan_segments(d):
    return load().pdssm_scan_segments(ctypes.byref(d))


def uses_fused(d):
    """1 when the single-read kernels run this descriptor, 0 when the
    multi-pass kernels do (dictionary tables beyond LDS), < 0 on error."""
    return load().pdssm_uses_fused(ctypes.byref(d))


def chunk_len(d):
    return load().pdssm_chunk_len(ctypes.byref(d))


def num_chunks(d):
    return load().pdssm_num_chunks(ctypes.byref(d))


def workspace_size(d, op):
    n = load().pdssm_workspace_size(ctypes.byref(d), int(op))
    if n == ctypes.c_size_t(-1).value:
        raise PdssmError(ERR_INVALID_ARG, "workspace_size")
    return n


def _p(t):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


def _stream(stream):
    s = stream if stream is not None else torch.cuda.current_stream()
    return ctypes.c_void_p(s.cuda_stream)


def _need(t, name, dtype, shape, device):
    if not isinstance(t, torch.Tensor):
        raise TypeError("%s must be a torch.Tensor" % name)
    if t.dtype != dtype:
        raise TypeError("%s must be %s, got %s" % (name, dtype, t.dtype))
    if tuple(t.shape) != tuple(shape):
        raise ValueError("%s must have shape %s, got %s" % (name, tuple(shape), tuple(t.shape)))
    if t.device != device or t.device.type != "cuda":
        raise ValueError("%s must be on %s" % (name, device))
    if not t.is_contiguous():
        raise ValueError("%s must be contiguous" % name)


def dims_of(idx, pi):
    B, L, H = idx.shape
    H2, K, N = pi.shape
    if H2 != H:
        raise ValueError("idx and pi disagree on H")
    return B, L, H, N, K


def is_bf16_io(D):
    """D given as bf16 (re, im) pairs [..., N, 2] rather than complex64."""
    return isinstance(D, torch.Tensor) and D.dtype == torch.bfloat16


def is_real_io(D):
    """D given as real float32 rows (the real-valued model)."""
    return isinstance(D, torch.Tensor) and D.dtype == torch.float32


def _check_inputs(idx, pi, D, b, c):
    B, L, H, N, K = dims_of(idx, pi)
    dev = idx.device
    _need(idx, "idx", torch.int32, (B, L, H), dev)
    _need(pi, "pi", torch.int32, (H, K, N), dev)
    for t, n in ((D, "D"), (b, "b"), (c, "c")):
        if is_bf16_io(D):
            _need(t, n, torch.bfloat16, (B, L, H, N, 2), dev)
        elif is_real_io(D):
            _need(t, n, torch.float32, (B, L, H, N), dev)
        else:
            _need(t, n, torch.complex64, (B, L, H, N), dev)
    return B, L, H, N, K, dev


class Scan:
    """Pre-allocated outputs and one workspace for one problem size; prepare(),
    fwd() and bwd() allocate nothing, so they can be timed in a loop.

    Without prepare() every scan builds the dictionary tables itself.  After
    prepare(pi) the scans reuse the tables in the workspace; call prepare()
    again whenever the contents of pi change."""

    def __init__(self, B, L, H, N, K, chunk=0, device="cuda", ste=False, bf16=False, real=False):
        self.d = desc(B, L, H, N, K, chunk)
        self.dp = desc(B, L, H, N, K, chunk)
        self.bf16 = bf16
        self.real = real
        self.d.flags = (FLAG_BF16_IO if bf16 else 0) | (FLAG_REAL_IO if real else 0)
        self.dp.flags = FLAG_PREPARED | self.d.flags
        self.prepared = False
        self.dims = (B, L, H, N, K)
        self.device = torch.device(device)
        self.C = num_chunks(self.d)
        if self.C < 0:
            raise PdssmError(self.C, "num_chunks")
        self.chunk = chunk_len(self.d)
        self.fused = uses_fused(self.d) == 1
        self.segments = load().pdssm_scan_segments(ctypes.byref(self.d))
        dev = self.device
        nws = max(workspace_size(self.d, OP_FWD), workspace_size(self.d, OP_BWD), 1)
        self.ws = torch.empty(nws, dtype=torch.uint8, device=dev)
        self.y = torch.empty((B, L, H), dtype=torch.float32, device=dev)
        self.h_final = torch.empty((B, H, N), dtype=torch.complex64, device=dev)
        self.saved = torch.empty((B, H, self.C, N), dtype=torch.float32 if real else torch.complex64, device=dev)
        if bf16:
            self.dD = torch.empty((B, L, H, N, 2), dtype=torch.bfloat16, device=dev)
        elif real:
            self.dD = torch.empty((B, L, H, N), dtype=torch.float32, device=dev)
        else:
            self.dD = torch.empty((B, L, H, N), dtype=torch.complex64, device=dev)
        self.db = torch.empty_like(self.dD)
        self.dc = torch.empty_like(self.dD)
        self.dh0 = torch.empty((B, H, N), dtype=torch.complex64, device=dev)
        self.status = torch.zeros(1, dtype=torch.int32, device=dev)
        self.ste = ste
        if ste:
            self.q = torch.empty((B, L, H, K), dtype=torch.float32, device=dev)
            self.z = torch.empty((B, L, H, N), dtype=torch.float32 if real else torch.complex64, device=dev)
            self.G = torch.empty((H, K, N, N), dtype=torch.float32, device=dev)
            self.ws_ste = torch.empty(max(workspace_size(self.d, OP_STE_GRADS), 1), dtype=torch.uint8,
                                      device=dev)

    def _desc(self):
        return ctypes.byref(self.dp if self.prepared else self.d)

    def _check(self, idx, pi, D, b, c, h0=None, dy=None, dh_final=None):
        """Every tensor argument has the type, shape, device and layout this
        Scan was built for (the library reads them through raw pointers)."""
        B, L, H, N, K = self.dims
        dev = self.device if self.device.index is not None else idx.device
        _need(idx, "idx", torch.int32, (B, L, H), dev)
        _need(pi, "pi", torch.int32, (H, K, N), dev)
        for t, n in ((D, "D"), (b, "b"), (c, "c")):
            if self.bf16:
                _need(t, n, torch.bfloat16, (B, L, H, N, 2), dev)
            elif self.real:
                _need(t, n, torch.float32, (B, L, H, N), dev)
            else:
                _need(t, n, torch.complex64, (B, L, H, N), dev)
        for t, n in ((h0, "h0"), (dh_final, "dh_final")):
            if t is not None:
                _need(t, n, torch.complex64, (B, H, N), dev)
        if dy is not None:
            _need(dy, "dy", torch.float32, (B, L, H), dev)

    def prepare(self, pi, stream=None):
        B, L, H, N, K = self.dims
        _need(pi, "pi", torch.int32, (H, K, N), pi.device)
        st = load().pdssm_prepare(ctypes.byref(self.d), _p(pi), _p(self.ws), self.ws.numel(),
                                  _p(self.status), _stream(stream))
        if st != OK:
            raise PdssmError(st, "pdssm_prepare")
        self.prepared = True

    def fwd(self, idx, pi, D, b, c, h0=None, stream=None):
        self._check(idx, pi, D, b, c, h0=h0)
        st = load().pdssm_scan_fwd(self._desc(), _p(idx), _p(pi), _p(D), _p(b), _p(c),
                                   _p(h0), _p(self.y), _p(self.h_final), _p(self.saved),
                                   _p(self.ws), self.ws.numel(), _p(self.status), _stream(stream))
        if st != OK:
            raise PdssmError(st, "pdssm_scan_fwd")
        return self.y, self.h_final, self.saved

    def bwd(self, idx, pi, D, b, c, dy, dh_final=None, stream=None):
        self._check(idx, pi, D, b, c, dy=dy, dh_final=dh_final)
        st = load().pdssm_scan_bwd(self._desc(), _p(idx), _p(pi), _p(D), _p(b), _p(c),
                                   _p(self.saved), _p(dy), _p(dh_final), _p(self.dD), _p(self.db),
                                   _p(self.dc), _p(self.dh0), _p(self.ws), self.ws.numel(),
                                   _p(self.status), _stream(stream))
        if st != OK:
            raise PdssmError(st, "pdssm_scan_bwd")
        return self.dD, self.db, self.dc, self.dh0

    def bwd_ste(self, idx, pi, D, b, c, dy, dh_final=None, stream=None):
        """bwd() plus the scaled states z (Scan(..., ste=True))."""
        self._check(idx, pi, D, b, c, dy=dy, dh_final=dh_final)
        st = load().pdssm_scan_bwd_ste(self._desc(), _p(idx), _p(pi), _p(D), _p(b), _p(c),
                                       _p(self.saved), _p(dy), _p(dh_final), _p(self.dD), _p(self.db),
                                       _p(self.dc), _p(self.dh0), _p(self.z), _p(self.ws),
                                       self.ws.numel(), _p(self.status), _stream(stream))
        if st != OK:
            raise PdssmError(st, "pdssm_scan_bwd_ste")
        return self.dD, self.db, self.dc, self.dh0, self.z

    def ste_grads(self, idx, pi, q=True, G=True, stream=None):
        """Scores q [B,L,H,K] and dictionary gradient G [H,K,N,N] from the db
        and z of the last bwd_ste() (each None when not asked for)."""
        qq, GG = (self.q if q else None), (self.G if G else None)
        B, L, H, N, K = self.dims
        _need(idx, "idx", torch.int32, (B, L, H), self.db.device)
        _need(pi, "pi", torch.int32, (H, K, N), self.db.device)
        st = load().pdssm_ste_grads(ctypes.byref(self.d), _p(idx), _p(pi), _p(self.db), _p(self.z), _p(qq),
                                    _p(GG), _p(self.ws_ste), self.ws_ste.numel(), _p(self.status),
                                    _stream(stream))
        if st != OK:
            raise PdssmError(st, "pdssm_ste_grads")
        return qq, GG

    def check_status(self):
        """Synchronise and raise if a kernel flagged an out-of-range index."""
        torch.cuda.synchronize(self.device)
        st = int(self.status.item())
        if st != OK:
            raise PdssmError(st, "kernel index check")


def _state_arg(x, name, real, dims, dev):
    """A [B,H,N] state argument: complex64, or for the real model also float32
    (widened to complex64, imaginary part 0)."""
    if x is None:
        return None
    if real and isinstance(x, torch.Tensor) and x.dtype == torch.float32:
        _need(x, name, torch.float32, dims, dev)
        return x.to(torch.complex64)
    _need(x, name, torch.complex64, dims, dev)
    return x


def scan_fwd(idx, pi, D, b, c, h0=None, chunk=0, stream=None):
    """Returns (y [B,L,H] f32, h_final [B,H,N] c64, saved [B,H,C,N] c64, or
    f32 for real inputs)."""
    B, L, H, N, K, dev = _check_inputs(idx, pi, D, b, c)
    h0 = _state_arg(h0, "h0", is_real_io(D), (B, H, N), dev)
    s = Scan(B, L, H, N, K, chunk, dev, bf16=is_bf16_io(D), real=is_real_io(D))
    s.fwd(idx, pi, D, b, c, h0, stream)
    s.check_status()
    return s.y, s.h_final, s.saved


def scan_fwd_noalloc(idx, pi, D, b, c, h0=None, chunk=0, y=None, h_final=None, saved=None, stream=None):
    """pdssm_scan_fwd_noalloc: the forward with the library's own device
    workspace (no workspace argument).  Outputs may be passed in (y, h_final,
    saved); the call then allocates nothing.  Returns (y, h_final, saved)."""
    B, L, H, N, K, dev = _check_inputs(idx, pi, D, b, c)
    h0 = _state_arg(h0, "h0", is_real_io(D), (B, H, N), dev)
    d = desc(B, L, H, N, K, chunk)
    d.flags = (FLAG_BF16_IO if is_bf16_io(D) else 0) | (FLAG_REAL_IO if is_real_io(D) else 0)
    C = num_chunks(d)
    if C < 0:
        raise PdssmError(C, "num_chunks")
    y = torch.empty((B, L, H), dtype=torch.float32, device=dev) if y is None else y
    h_final = torch.empty((B, H, N), dtype=torch.complex64, device=dev) if h_final is None else h_final
    sdt = saved_dtype(D)
    saved = torch.empty((B, H, C, N), dtype=sdt, device=dev) if saved is None else saved
    _need(y, "y", torch.float32, (B, L, H), dev)
    _need(h_final, "h_final", torch.complex64, (B, H, N), dev)
    _need(saved, "saved", sdt, (B, H, C, N), dev)
    st = load().pdssm_scan_fwd_noalloc(ctypes.byref(d), _p(idx), _p(pi), _p(D), _p(b), _p(c), _p(h0), _p(y),
                                       _p(h_final), _p(saved), None, _stream(stream))
    if st != OK:
        raise PdssmError(st, "pdssm_scan_fwd_noalloc")
    return y, h_final, saved


def saved_dtype(D):
    """dtype of the saved chunk states for inputs D: float32 for the real
    model (its states are real), else complex64."""
    return torch.float32 if is_real_io(D) else torch.complex64


def scan_bwd(idx, pi, D, b, c, saved, dy, dh_final=None, chunk=0, stream=None):
    """Returns (dD, db, dc [B,L,H,N] c64, or [B,L,H,N,2] bf16 for bf16 inputs,
    or [B,L,H,N] f32 for real inputs; dh0 [B,H,N] c64)."""
    B, L, H, N, K, dev = _check_inputs(idx, pi, D, b, c)
    s = Scan(B, L, H, N, K, chunk, dev, bf16=is_bf16_io(D), real=is_real_io(D))
    _need(saved, "saved", saved_dtype(D), (B, H, s.C, N), dev)
    _need(dy, "dy", torch.float32, (B, L, H), dev)
    dh_final = _state_arg(dh_final, "dh_final", is_real_io(D), (B, H, N), dev)
    s.saved = saved
    s.bwd(idx, pi, D, b, c, dy, dh_final, stream)
    s.check_status()
    return s.dD, s.db, s.dc, s.dh0


def compose_chunks(idx, pi, D, chunk, stream=None):
    """Returns (pi_out [B,H,C,N] int32, d_out [B,H,C,N] c64)."""
    B, L, H, N, K = dims_of(idx, pi)
    dev = idx.device
    _need(idx, "idx", torch.int32, (B, L, H), dev)
    _need(pi, "pi", torch.int32, (H, K, N), dev)
    _need(D, "D", torch.complex64, (B, L, H, N), dev)
    if chunk < 1:
        raise ValueError("chunk must be >= 1")
    tau = min(int(chunk), L)
    C = -(-L // tau)
    pi_out = torch.empty((B, H, C, N), dtype=torch.int32, device=dev)
    d_out = torch.empty((B, H, C, N), dtype=torch.complex64, device=dev)
    status = torch.zeros(1, dtype=torch.int32, device=dev)
    d = desc(B, L, H, N, K, tau)
    st = load().pdssm_compose_chunks(ctypes.byref(d), _p(idx), _p(pi), _p(D), _p(pi_out),
                                     _p(d_out), _p(status), _stream(stream))
    if st != OK:
        raise PdssmError(st, "pdssm_compose_chunks")
    torch.cuda.synchronize(dev)
    if int(status.item()) != OK:
        raise PdssmError(int(status.item()), "kernel index check")
    return pi_out, d_out


def scan_bwd_ste(idx, pi, D, b, c, saved, dy, dh_final=None, chunk=0, stream=None):
    """Returns (dD, db, dc, dh0, z [B,L,H,N] c64, or f32 for real inputs;
    with bf16 inputs dD, db, dc are bf16 pairs and z stays c64)."""
    B, L, H, N, K, dev = _check_inputs(idx, pi, D, b, c)
    s = Scan(B, L, H, N, K, chunk, dev, ste=True, bf16=is_bf16_io(D), real=is_real_io(D))
    _need(saved, "saved", saved_dtype(D), (B, H, s.C, N), dev)
    _need(dy, "dy", torch.float32, (B, L, H), dev)
    dh_final = _state_arg(dh_final, "dh_final", is_real_io(D), (B, H, N), dev)
    s.saved = saved
    out = s.bwd_ste(idx, pi, D, b, c, dy, dh_final, stream)
    s.check_status()
    return out


def ste_grads(idx, pi, g, z, q=True, G=True, stream=None):
    """(q [B,L,H,K] f32 or None, G [H,K,N,N] f32 or None) from g = db and z
    of scan_bwd_ste: the scores of every map at every step and, per head and
    map, the sum of Re(g_t z_t^H) over the steps that chose the map.  g, z
    complex64; or float32 for the real-valued model; or g as bf16 (re, im)
    pairs [B,L,H,N,2] (the bf16 setting's db) with z complex64."""
    B, L, H = idx.shape
    N = g.shape[3]
    K = pi.shape[1]
    dev = idx.device
    real, bf16 = is_real_io(g), is_bf16_io(g)
    _need(idx, "idx", torch.int32, (B, L, H), dev)
    _need(pi, "pi", torch.int32, (H, K, N), dev)
    if bf16:
        _need(g, "g", torch.bfloat16, (B, L, H, N, 2), dev)
    else:
        _need(g, "g", torch.float32 if real else torch.complex64, (B, L, H, N), dev)
    _need(z, "z", torch.float32 if real else torch.complex64, (B, L, H, N), dev)
    d = desc(B, L, H, N, K)
    d.flags = FLAG_REAL_IO if real else (FLAG_BF16_IO if bf16 else 0)
    ws = torch.empty(max(workspace_size(d, OP_STE_GRADS), 1), dtype=torch.uint8, device=dev)
    qq = torch.empty((B, L, H, K), dtype=torch.float32, device=dev) if q else None
    GG = torch.empty((H, K, N, N), dtype=torch.float32, device=dev) if G else None
    status = torch.zeros(1, dtype=torch.int32, device=dev)
    st = load().pdssm_ste_grads(ctypes.byref(d), _p(idx), _p(pi), _p(g), _p(z), _p(qq), _p(GG), _p(ws),
                                ws.numel(), _p(status), _stream(stream))
    if st != OK:
        raise PdssmError(st, "pdssm_ste_grads")
    torch.cuda.synchronize(dev)
    if int(status.item()) != OK:
        raise PdssmError(int(status.item()), "kernel index check")
    return qq, GG


def softmax_vjp(x, gy, dim, temp, out=None, stream=None):
    """gx = s * (gy - sum(s * gy, dim)) / temp with s = softmax(x / temp, dim)."""
    if x.dtype != torch.float32 or gy.dtype != torch.float32 or x.shape != gy.shape:
        raise TypeError("x and gy must be float32 tensors of one shape")
    if not (x.is_contiguous() and gy.is_contiguous()) or x.device.type != "cuda" or gy.device != x.device:
        raise ValueError("x and gy must be contiguous and on one GPU")
    dim = dim % x.dim()
    outer = 1
    for n in x.shape[:dim]:
        outer *= int(n)
    inner = 1
    for n in x.shape[dim + 1:]:
        inner *= int(n)
    gx = torch.empty_like(x) if out is None else out
    _need(gx, "out", torch.float32, tuple(x.shape), x.device)
    st = load().pdssm_softmax_vjp(_p(x), _p(gy), _p(gx), outer, int(x.shape[dim]), inner, float(temp),
                                  _stream(stream))
    if st != OK:
        raise PdssmError(st, "pdssm_softmax_vjp")
    return gx


def surrogate_grads(q, G, logits, M, temp, stream=None):
    """The two surrogate gradients of Prop. 2: (d logits [B,L,H,K], dM [H,K,N,N])."""
    return softmax_vjp(logits, q, 3, temp, stream=stream), softmax_vjp(M, G, 2, temp, stream=stream)


def decode_step(idx, pi, D, b, c, h=None, out=None, y=None, stream=None, check=True):
    """One recurrence step per sequence: returns (h_new [B,H,N] c64, y [B,H] f32).
    idx [B,H] int32; D, b, c [B,H,N] c64 (or [B,H,N,2] bf16 pairs, or [B,H,N]
    float32 for the real-valued model); h [B,H,N] c64 or None (zero state).
    out may be h itself (in-place update)."""
    B, H = idx.shape
    H2, K, N = pi.shape
    if H2 != H:
        raise ValueError("idx and pi disagree on H")
    dev = idx.device
    _need(idx, "idx", torch.int32, (B, H), dev)
    _need(pi, "pi", torch.int32, (H, K, N), dev)
    for t, n in ((D, "D"), (b, "b"), (c, "c")):
        if is_bf16_io(D):
            _need(t, n, torch.bfloat16, (B, H, N, 2), dev)
        elif is_real_io(D):
            _need(t, n, torch.float32, (B, H, N), dev)
        else:
            _need(t, n, torch.complex64, (B, H, N), dev)
    if h is not None:
        _need(h, "h", torch.complex64, (B, H, N), dev)
    out = torch.empty((B, H, N), dtype=torch.complex64, device=dev) if out is None else out
    y = torch.empty((B, H), dtype=torch.float32, device=dev) if y is None else y
    status = torch.zeros(1, dtype=torch.int32, device=dev) if check else None
    d = desc(B, 1, H, N, K)
    d.flags = (FLAG_BF16_IO if is_bf16_io(D) else 0) | (FLAG_REAL_IO if is_real_io(D) else 0)
    st = load().pdssm_decode_step(ctypes.byref(d), _p(idx), _p(pi), _p(D), _p(b), _p(c), _p(h), _p(out), _p(y),
                                  _p(status), _stream(stream))
    if st != OK:
        raise PdssmError(st, "pdssm_decode_step")
    if check:
        torch.cuda.synchronize(dev)
        if int(status.item()) != OK:
            raise PdssmError(int(status.item()), "kernel index check")
    return out, y


def dict_argmax(M, stream=None):
    """pi [H,K,N] int32 = first argmax over the rows i of every column j of
    the dense dictionary M [H,K,N,N] float32."""
    H, K, N, N2 = M.shape
    if N2 != N:
        raise ValueError("M must be [H,K,N,N]")
    _need(M, "M", torch.float32, (H, K, N, N), M.device)
    pi = torch.empty((H, K, N), dtype=torch.int32, device=M.device)
    st = load().pdssm_dict_argmax(H, K, N, _p(M), _p(pi), _stream(stream))
    if st != OK:
        raise PdssmError(st, "pdssm_dict_argmax")
    return pi


def route(u, S, logits=True, stream=None):
    """Routing scores and choices: u [B,L,Dm] bf16, S [H,K,Dm] bf16 ->
    (logits [B,L,H,K] f32 or None, idx [B,L,H] int32)."""
    B, L, Dm = u.shape
    H, K, Dm2 = S.shape
    if Dm2 != Dm:
        raise ValueError("u and S disagree on the contraction length")
    _need(u, "u", torch.bfloat16, (B, L, Dm), u.device)
    _need(S, "S", torch.bfloat16, (H, K, Dm), u.device)
    lg = torch.empty((B, L, H, K), dtype=torch.float32, device=u.device) if logits else None
    idx = torch.empty((B, L, H), dtype=torch.int32, device=u.device)
    st = load().pdssm_route(B * L, Dm, H, K, _p(u), _p(S), _p(lg), _p(idx), _stream(stream))
    if st != OK:
        raise PdssmError(st, "pdssm_route")
    return lg, idx


def project(u, S=None, Wb=None, Wc=None, Wd=None, logits=True, N=None, stream=None):
    """pdssm_project: the token projections of a layer in one product.
    u [B,L,Dm] bf16; S [H,K,Dm] bf16 (routing); Wb, Wc, Wd [H,2N,Dm] bf16
    (b, c and the diagonal generator).  Returns a dict with logits [B,L,H,K]
    f32 and idx [B,L,H] int32 (with S), and b, c, D [B,L,H,N] complex64 (each
    with its weights)."""
    B, L, Dm = u.shape
    dev = u.device
    _need(u, "u", torch.bfloat16, (B, L, Dm), dev)
    Ws = [w for w in (Wb, Wc, Wd) if w is not None]
    if S is None and not Ws:
        raise ValueError("project: nothing to compute")
    H = S.shape[0] if S is not None else Ws[0].shape[0]
    K = S.shape[1] if S is not None else 1
    if Ws:
        N = Ws[0].shape[1] // 2
    N = N or 8
    if S is not None:
        _need(S, "S", torch.bfloat16, (H, K, Dm), dev)
    for w, n in ((Wb, "Wb"), (Wc, "Wc"), (Wd, "Wd")):
        if w is not None:
            _need(w, n, torch.bfloat16, (H, 2 * N, Dm), dev)
    out = {}
    if S is not None:
        out["logits"] = torch.empty((B, L, H, K), dtype=torch.float32, device=dev) if logits else None
        out["idx"] = torch.empty((B, L, H), dtype=torch.int32, device=dev)
    for w, n in ((Wb, "b"), (Wc, "c"), (Wd, "D")):
        if w is not None:
            out[n] = torch.empty((B, L, H, N), dtype=torch.complex64, device=dev)
    st = load().pdssm_project(B * L, Dm, H, K, N, _p(u), _p(S), _p(Wb), _p(Wc), _p(Wd), _p(out.get("logits")),
                              _p(out.get("idx")), _p(out.get("b")), _p(out.get("c")), _p(out.get("D")),
                              _stream(stream))
    if st != OK:
        raise PdssmError(st, "pdssm_project")
    return out


# ---- gated recurrent layers ------------------------------------------------

GATED_CHUNK = 128  # rows between two saved states
KEPT_ROWS = 32     # rows that share an exponent in the 8-bit form
GATE_HOLD = -64.0  # a gate logit at or under this one holds the state
OP_SIZE_ERROR = ctypes.c_size_t(-1).value


def _ceil(n, k):
    return -(-n // k)


def _on_its_device(f):
    """f with the device of its first argument, by place or by name, as the
    current one, which is where its kernels are launched."""
    name = next(iter(inspect.signature(f).parameters))

    @functools.wraps(f)
    def on(*args, **kw):
        t = args[0] if args else kw.get(name)
        if isinstance(t, (tuple, list)) and t:
            t = t[0]
        if isinstance(t, torch.Tensor) and t.is_cuda and t.device.index != torch.cuda.current_device():
            with torch.cuda.device(t.device):
                return f(*args, **kw)
        return f(*args, **kw)
    return on


# the current stream of a device as a number; torch.cuda.current_stream builds
# an object for it, a fifth of a short call's time
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda i: torch.cuda.current_stream(i).cuda_stream)


def _on(stream, dev, tensors):
    """The stream to launch on, as a number.  One of the caller's own that is not
    the current one waits for it (the memory of the outputs may still be in use
    there, by work of whoever had it before), and learns of every tensor of the
    call, so that none is given to other work before it has run.  A stream of
    another device is refused."""
    current = _raw_stream(dev.index)
    if stream is None:
        return current
    if stream.device != dev:
        raise ValueError("stream must be one of %s" % dev)
    if stream.cuda_stream == current:
        return current
    stream.wait_stream(torch.cuda.current_stream(dev))
    for t in tensors:
        if t is not None:
            t.record_stream(stream)
    return stream.cuda_stream


def _tensor(t, name, dtype, shape, dev):
    """_need, quick where nothing is wrong; the address."""
    if not (isinstance(t, torch.Tensor) and t.dtype is dtype and t.shape == shape and t.is_cuda and t.device == dev and
            t.is_contiguous()):
        _need(t, name, dtype, shape, dev)
    return t.data_ptr()


def _rows(t, name, dtype, shape, dev):
    """pdssm_rows of rows [T,C] or [B,L,C] that may be a part of wider rows."""
    if not isinstance(t, torch.Tensor):
        raise TypeError("%s must be a torch.Tensor" % name)
    if t.dtype is not dtype:
        raise TypeError("%s must be %s, got %s" % (name, dtype, t.dtype))
    if t.shape != shape:
        raise ValueError("%s must have shape %s, got %s" % (name, tuple(shape), tuple(t.shape)))
    if not t.is_cuda or t.device != dev:
        raise ValueError("%s must be on %s" % (name, dev))
    C, step = shape[-1], t.stride()
    if step[-1] != 1 and C > 1:
        raise ValueError("%s: the entries of a row must be next to each other" % name)
    ld = C
    if len(shape) == 3:
        B, L = shape[0], shape[1]
        if L > 1:
            ld = step[1]
            if B > 1 and step[0] != L * ld:
                raise ValueError("%s: rows must be evenly spaced over the batch" % name)
        elif B > 1:
            ld = step[0]
    elif shape[0] > 1:
        ld = step[0]
    if ld < C:
        raise ValueError("%s: rows must not overlap" % name)
    return _ROW.pack(t.data_ptr(), ld, 0)


def _kept(pair, name, T, C, dev):
    """(address of the codes, address of the exponents) of a pair (q, e) in the 8-bit form."""
    q, e = pair
    _int32(T, C)
    return (_tensor(q, name + " codes", torch.int8, (T, C), dev),
            _tensor(e, name + " exponents", torch.int8, (_ceil(T, KEPT_ROWS), C), dev))


def _kept_rows(pair, name, T, C, dev):
    """pdssm_rows of a pair."""
    q_at, e_at = _kept(pair, name, T, C, dev)
    return _ROW.pack(q_at, C, e_at)


def _int32(*sizes):
    """Sizes that the library takes as 32-bit numbers."""
    if max(sizes) > 0x7fffffff:
        raise PdssmError(ERR_UNSUPPORTED, "sizes %s" % (sizes,))


# pdssm_gated_desc and pdssm_rows as bytes, which the library reads during the
# call; ctypes structures take seven times as long to make
_DESC, _ROW = struct.Struct("iiiI"), struct.Struct("PqP")


def _desc(T, C, S, flags):
    _int32(T, C, S)
    return _DESC.pack(T, C, S, flags)


def _row_type(t):
    if not isinstance(t, torch.Tensor):
        raise TypeError("rows must be a torch.Tensor")
    if t.dtype is torch.bfloat16:
        return FLAG_BF16_IO
    if t.dtype is torch.float32:
        return 0
    raise TypeError("rows must be float32 or bfloat16, got %s" % t.dtype)


def _sequences(t, cu):
    """(T, C, S) of rows t [B,L,C], or [T,C] with the bounds cu [S+1]."""
    if cu is None:
        if t.dim() != 3:
            raise ValueError("rows must be [B,L,C], or [T,C] with cu")
        B, L, C = t.shape
        T, S = B * L, B
    else:
        if t.dim() != 2:
            raise ValueError("rows must be [T,C] when cu is given")
        T, C = t.shape
        if not isinstance(cu, torch.Tensor) or cu.dim() != 1 or cu.shape[0] < 2:
            raise ValueError("cu must be [S+1] with S >= 1")
        S = cu.shape[0] - 1
        _tensor(cu, "cu", torch.int32, (S + 1,), t.device)
    if C < 1 or S < 1:
        raise ValueError("rows need at least one channel and one sequence")
    return T, C, S


def _gated_ws(desc, op, dev):
    n = load().pdssm_gated_workspace_size(desc, op)
    if n == OP_SIZE_ERROR:
        raise PdssmError(ERR_UNSUPPORTED, "gated_workspace_size")
    return torch.empty(n, dtype=torch.uint8, device=dev) if n else None


def _state(t, name, S, C, dev):
    return None if t is None else _tensor(t, name, torch.float32, (S, C), dev)


def _at(t):
    return None if t is None else t.data_ptr()


def _done(st, status, what):
    """Raise on a refusal; with a status tensor, synchronise and raise if a kernel reported a bad index."""
    if st != OK:
        raise PdssmError(st, what)
    if status is not None:
        torch.cuda.synchronize()
        st = int(status.item())
        if st != OK:
            raise PdssmError(st, what)


def _three(tensors):
    return (ctypes.c_void_p * 3)(*[t.data_ptr() for t in tensors])


def _status(check, dev):
    return torch.zeros(1, dtype=torch.int32, device=dev) if check else None


@_on_its_device
def gated_fwd(x, ga, gi, rate, cu=None, h0=None, hold8=False, check=True, stream=None):
    """The gated recurrence h_t = a_t h_{t-1} + sqrt(1 - a_t^2) sigmoid(gi_t) x_t
    with a_t = exp(-rate * sigmoid(ga_t)), over every sequence from its state
    in h0 [S,C] (default 0).  Returns (y, h_final [S,C], saved
    [ceil(T/128),C]), y = h in the rows' type and shape; with hold8=True also
    ((q, e) of x, of ga, of gi): the inputs in the 8-bit form, which gated_bwd
    takes in their place.  Rows behind the last sequence are zero, in the 8-bit
    form too.  check=False neither synchronises nor reports a bad cu."""
    flags = _row_type(x)
    T, C, S = _sequences(x, cu)
    if cu is not None:
        flags |= FLAG_ZERO_REST
    dev, shape = x.device, x.shape
    d = _desc(T, C, S, flags)
    rows = [_rows(t, n, x.dtype, shape, dev) for t, n in ((x, "x"), (ga, "ga"), (gi, "gi"))]
    rate_at = _tensor(rate, "rate", torch.float32, (C,), dev)
    h0_at = _state(h0, "h0", S, C, dev)
    y = torch.empty_like(x, memory_format=torch.contiguous_format)
    h_final = rate.new_empty((S, C))
    saved = rate.new_empty((_ceil(T, GATED_CHUNK), C))
    kept = q = e = None
    if hold8:
        kept = tuple((torch.empty((T, C), dtype=torch.int8, device=dev),
                      torch.empty((_ceil(T, KEPT_ROWS), C), dtype=torch.int8, device=dev)) for _ in range(3))
        q, e = _three([k[0] for k in kept]), _three([k[1] for k in kept])
    ws = _gated_ws(d, OP_FWD, dev)
    status = _status(check, dev)
    s = _on(stream, dev, (x, ga, gi, rate, cu, h0, y, h_final, saved, ws, status,
                          *([t for k in kept for t in k] if hold8 else ())))
    st = load().pdssm_gated_fwd(d, *rows, rate_at, _at(cu), h0_at, y.data_ptr(), h_final.data_ptr(), saved.data_ptr(), q, e,
                                _at(ws), ws.numel() if ws is not None else 0, _at(status), s)
    _done(st, status, "pdssm_gated_fwd")
    return (y, h_final, saved, kept) if hold8 else (y, h_final, saved)


@_on_its_device
def gated_bwd(x, ga, gi, rate, saved, dy, cu=None, h0=None, dh_final=None, check=True, stream=None):
    """Gradients of gated_fwd: (dx, dga, dgi, drate [C], dh0 [S,C]) from dy (rows
    as y) and dh_final [S,C] (default 0); saved, cu and h0 as in the forward.  x, ga, gi are the
    forward's rows, or all three the pairs (q, e) that it returned with
    hold8=True.  dx, dga and dgi, in dy's type and shape, are the three parts of one
    tensor [..., 3C], the gradient of a projection that makes the three; rows
    behind the last sequence are zero in them, so project_wgrad may sum over all."""
    flags = _row_type(dy)
    T, C, S = _sequences(dy, cu)
    if cu is not None:
        flags |= FLAG_ZERO_REST
    dev, shape = dy.device, dy.shape
    ins = ((x, "x"), (ga, "ga"), (gi, "gi"))
    eight = isinstance(x, (tuple, list))
    if any(isinstance(t, (tuple, list)) != eight for t, _ in ins):
        raise TypeError("x, ga and gi must be all rows or all pairs (q, e)")
    d = _desc(T, C, S, flags)
    r = [_kept_rows(t, n, T, C, dev) if eight else _rows(t, n, dy.dtype, shape, dev) for t, n in ins]
    dy_rows = _rows(dy, "dy", dy.dtype, shape, dev)
    rate_at = _tensor(rate, "rate", torch.float32, (C,), dev)
    saved_at = _tensor(saved, "saved", torch.float32, (_ceil(T, GATED_CHUNK), C), dev)
    h0_at, dhf_at = _state(h0, "h0", S, C, dev), _state(dh_final, "dh_final", S, C, dev)
    rows = dy.new_empty((*shape[:-1], 3 * C))
    grads = rows.split(C, -1)
    drate = torch.empty_like(rate)
    dh0 = rate.new_empty((S, C))
    ws = _gated_ws(d, OP_BWD, dev)
    status = _status(check, dev)
    s = _on(stream, dev, (*([t for k in (x, ga, gi) for t in k] if eight else (x, ga, gi)), rate, saved, dy, cu, h0,
                          dh_final, rows, drate, dh0, ws, status))
    st = load().pdssm_gated_bwd(d, *r, rate_at, _at(cu), h0_at, saved_at, dy_rows, dhf_at, _three(grads), 3 * C,
                                drate.data_ptr(), dh0.data_ptr(), _at(ws), ws.numel() if ws is not None else 0, _at(status), s)
    _done(st, status, "pdssm_gated_bwd")
    return (*grads, drate, dh0)


@_on_its_device
def gated_step(x, ga, gi, rate, h, slots=None, out=None, y=None, check=True, stream=None):
    """One token of the gated recurrence for each row of x, ga, gi [B,C]: returns
    (h_new [S,C], y [B,C]).  h [S,C] holds the states; row b advances state
    slots[b] (int32; default b).  A negative slot skips its row; a slot past the
    pool or named by an earlier row is an error and skips it too.  Skipped rows of
    y, and states that no row advances, are not written.  out [S,C] takes the new
    states; default: in place."""
    flags = _row_type(x)
    shape = x.shape
    if len(shape) != 2:
        raise ValueError("x must be [B,C]")
    B, C = shape
    dev = x.device
    if not isinstance(h, torch.Tensor) or h.dim() != 2:
        raise ValueError("h must be [S,C]")
    S = h.shape[0]
    d = _desc(B, C, S, flags)
    rows = [_rows(t, n, x.dtype, shape, dev) for t, n in ((x, "x"), (ga, "ga"), (gi, "gi"))]
    rate_at = _tensor(rate, "rate", torch.float32, (C,), dev)
    h_at = _tensor(h, "h", torch.float32, (S, C), dev)
    out_at = h_at if out is None else _tensor(out, "out", torch.float32, (S, C), dev)
    slots_at = None if slots is None else _tensor(slots, "slots", torch.int32, (B,), dev)
    y_at = None if y is None else _tensor(y, "y", x.dtype, shape, dev)
    if y is None:
        y = torch.empty_like(x, memory_format=torch.contiguous_format)
        y_at = y.data_ptr()
    status = _status(check, dev)
    s = _on(stream, dev, (x, ga, gi, rate, h, out, slots, y, status))
    st = load().pdssm_gated_step(d, *rows, rate_at, slots_at, h_at, out_at, y_at, _at(status), s)
    _done(st, status, "pdssm_gated_step")
    return h if out is None else out, y


@_on_its_device
def pack8(u, stream=None):
    """(q, e): rows u [T,C] or [B,L,C] in the 8-bit form, q [T,C] and
    e [ceil(T/32),C] int8 with T = B*L; the value of q[t,c] is q[t,c] * 2^e[t//32,c]."""
    flags = _row_type(u)
    if u.dim() not in (2, 3):
        raise ValueError("u must be [T,C] or [B,L,C]")
    C, dev = u.shape[-1], u.device
    T = u.shape[0] if u.dim() == 2 else u.shape[0] * u.shape[1]
    _int32(T, C)
    rows = _rows(u, "u", u.dtype, u.shape, dev)
    q = torch.empty((T, C), dtype=torch.int8, device=dev)
    e = torch.empty((_ceil(T, KEPT_ROWS), C), dtype=torch.int8, device=dev)
    s = _on(stream, dev, (u, q, e))
    _done(load().pdssm_pack8(T, C, flags, rows, q.data_ptr(), e.data_ptr(), s), None, "pdssm_pack8")
    return q, e


@_on_its_device
def unpack8(pair, dtype=torch.float32, stream=None):
    """The values [T,C] that a pair (q, e) of the 8-bit form stands for, exact in float32 and bfloat16."""
    q, e = pair
    if dtype not in (torch.float32, torch.bfloat16):
        raise TypeError("dtype must be float32 or bfloat16")
    if not isinstance(q, torch.Tensor) or q.dim() != 2:
        raise ValueError("q must be [T,C]")
    T, C = q.shape
    dev = q.device
    q_at, e_at = _kept(pair, "u", T, C, dev)
    out = torch.empty_like(q, dtype=dtype)
    s = _on(stream, dev, (q, e, out))
    _done(load().pdssm_unpack8(T, C, FLAG_BF16_IO if dtype is torch.bfloat16 else 0, q_at, e_at, out.data_ptr(), s), None,
          "pdssm_unpack8")
    return out


@_on_its_device
def project_wgrad(dP, u8, stream=None):
    """dW [M,Dm] float32 = dP^T u, the weight gradient of a projection P = u W^T:
    dP bfloat16 with B*L rows of M entries in all (the bf16 pairs that
    scan_bwd returns, [B,L,H,N,2], are rows of 2*H*N), u8 the activations u in
    the 8-bit form (pack8).  All rows count: where sequences are packed, those
    behind the last one have to be zero in one of the two and finite in the other
    (gated_fwd and gated_bwd return zeros there)."""
    q, e = u8
    if not isinstance(q, torch.Tensor) or q.dim() != 2:
        raise ValueError("u8 must be a pair (q, e) with q [T,Dm]")
    T, Dm = q.shape
    dev = q.device
    q_at, e_at = _kept(u8, "u", T, Dm, dev)
    if not isinstance(dP, torch.Tensor) or dP.dim() < 2:
        raise ValueError("dP must be rows [T,M] or [B,L,...]")
    shape = dP.shape
    dP_at = _tensor(dP, "dP", torch.bfloat16, shape, dev)
    lead = 1 if len(shape) == 2 else 2  # axes that count rows
    if math.prod(shape[:lead]) != T:
        raise ValueError("dP and u8 disagree on the number of rows")
    M = math.prod(shape[lead:])
    _int32(M)
    n = load().pdssm_project_wgrad_workspace_size(T, M, Dm)
    if n == OP_SIZE_ERROR:
        raise PdssmError(ERR_UNSUPPORTED, "project_wgrad_workspace_size")
    dW = torch.empty((M, Dm), dtype=torch.float32, device=dev)
    ws = torch.empty(n, dtype=torch.uint8, device=dev) if n else None
    s = _on(stream, dev, (dP, q, e, dW, ws))
    _done(load().pdssm_project_wgrad(T, M, Dm, dP_at, q_at, e_at, dW.data_ptr(), _at(ws), n, s), None, "pdssm_project_wgrad")
    return dW


# ---- linear attention with a decay for each head ----------------------------

_ATTN_DESC, _HEADS = struct.Struct("8ifI"), struct.Struct("Pqq")


def _heads(t, name, dtype, lead, D, dev):
    """(address, entries from row to row, from head to head, heads) of heads' rows [*lead, heads, D] that may be
    parts of wider rows."""
    if not isinstance(t, torch.Tensor):
        raise TypeError("%s must be a torch.Tensor" % name)
    if t.dtype is not dtype:
        raise TypeError("%s must be %s, got %s" % (name, dtype, t.dtype))
    n, shape = len(lead), t.shape
    if len(shape) != n + 2 or shape[0] != lead[0] or (n == 2 and shape[1] != lead[1]) or shape[-1] != D:
        raise ValueError("%s must have shape (%s, heads, %s), got %s" % (name, ", ".join(map(str, lead)), D, tuple(shape)))
    if not t.is_cuda or t.device != dev:
        raise ValueError("%s must be on %s" % (name, dev))
    heads = shape[n]
    if t.is_contiguous():
        return t.data_ptr(), heads * D, D, heads
    step = t.stride()
    if step[-1] != 1 and D > 1:
        raise ValueError("%s: the entries of a row must be next to each other" % name)
    ld = 0
    if n == 2:
        B, L = lead
        if L > 1:
            ld = step[1]
            if B > 1 and step[0] != L * ld:
                raise ValueError("%s: rows must be evenly spaced over the batch" % name)
        elif B > 1:
            ld = step[0]
    elif lead[0] > 1:
        ld = step[0]
    return t.data_ptr(), ld, step[n] if heads > 1 else 0, heads


def _attn(q, k, v, rate, scale, S, lead, T):
    """(desc, pdssm_heads of q, k and v, address of rate, (H, Dk, Dv), device)."""
    flags = _row_type(q)
    dev, dtype = q.device, q.dtype
    if not isinstance(rate, torch.Tensor) or rate.dim() != 1:
        raise ValueError("rate must be [H]")
    H = rate.shape[0]
    rate_at = _tensor(rate, "rate", torch.float32, (H,), dev)
    if not isinstance(v, torch.Tensor) or v.dim() != len(lead) + 2:
        raise ValueError("v must be rows [%s,heads,D]" % ",".join("BL" if len(lead) == 2 else "T"))
    Dk, Dv = q.shape[-1], v.shape[-1]
    qp, ql, qs, hq = _heads(q, "q", dtype, lead, Dk, dev)
    kp, kl, ks, hk = _heads(k, "k", dtype, lead, Dk, dev)
    vp, vl, vs, hv = _heads(v, "v", dtype, lead, Dv, dev)
    if hq < 1 or hk < 1 or hv < 1 or H % hq or H % hk or H % hv:
        raise ValueError("q, k and v have %d, %d and %d heads, which have to divide the %d of rate" % (hq, hk, hv, H))
    if not 1 <= Dk <= 256 or not 1 <= Dv <= 256:
        raise ValueError("heads must have 1 to 256 entries, got %d and %d" % (Dk, Dv))
    scale = Dk ** -0.5 if scale is None else float(scale)
    if not abs(scale) < math.inf:
        raise ValueError("scale must be finite")
    if T > 0x7fffffff or S > 0x7fffffff:
        _int32(T, S)
    return (_ATTN_DESC.pack(T, S, H, hq, hk, hv, Dk, Dv, scale, flags),
            (_HEADS.pack(qp, ql, qs), _HEADS.pack(kp, kl, ks), _HEADS.pack(vp, vl, vs)), rate_at, (H, Dk, Dv), dev)


def _head_sequences(t, cu):
    """(lead, T, S) of heads' rows t [B,L,heads,D], or [T,heads,D] with the bounds cu [S+1]."""
    if not isinstance(t, torch.Tensor) or t.dim() != (4 if cu is None else 3):
        raise ValueError("rows must be [B,L,heads,D], or [T,heads,D] with cu")
    lead = t.shape[:-2]
    if cu is None:
        S, T = lead[0], lead[0] * lead[1]
    else:
        if not isinstance(cu, torch.Tensor) or cu.dim() != 1 or cu.shape[0] < 2:
            raise ValueError("cu must be [S+1] with S >= 1")
        S, T = cu.shape[0] - 1, lead[0]
        _tensor(cu, "cu", torch.int32, (S + 1,), t.device)
    if S < 1:
        raise ValueError("rows need at least one sequence")
    return lead, T, S


def _attn_ws(desc, cu, op, dev):
    n = load().pdssm_decay_attn_workspace_size(desc, 0 if cu is None else 1, op)
    if n == OP_SIZE_ERROR:
        raise PdssmError(ERR_UNSUPPORTED, "decay_attn_workspace_size")
    return torch.empty(n, dtype=torch.uint8, device=dev) if n else None


def _matrix_state(t, name, shape, dev):
    return None if t is None else _tensor(t, name, torch.float32, shape, dev)


@_on_its_device
def decay_attn_fwd(q, k, v, rate, scale=None, cu=None, h0=None, check=True, stream=None):
    """Linear attention with a decay for each head, over every sequence from its
    state in h0 [S,H,Dk,Dv] (default 0): with a = exp(-rate[h]),
    S_t = a S_{t-1} + k_t v_t^T and o_t = scale * S_t^T q_t (default scale
    Dk**-0.5).  q, k and v may have fewer heads than the H of rate: head h reads
    head h // (H / heads).  Returns (o [..,H,Dv] in the rows' type, h_final
    [S,H,Dk,Dv]).  Rows behind the last sequence are zero.  check=False neither
    synchronises nor reports a bad cu."""
    lead, T, S = _head_sequences(q, cu)
    d, rows, rate_at, (H, Dk, Dv), dev = _attn(q, k, v, rate, scale, S, lead, T)
    h0_at = _matrix_state(h0, "h0", (S, H, Dk, Dv), dev)
    o = q.new_empty((*lead, H, Dv))
    h_final = rate.new_empty((S, H, Dk, Dv))
    ws = _attn_ws(d, cu, OP_FWD, dev)
    status = _status(check, dev)
    s = _on(stream, dev, (q, k, v, rate, cu, h0, o, h_final, ws, status))
    st = load().pdssm_decay_attn_fwd(d, *rows, rate_at, _at(cu), h0_at, o.data_ptr(), h_final.data_ptr(), _at(ws),
                                     ws.numel() if ws is not None else 0, _at(status), s)
    _done(st, status, "pdssm_decay_attn_fwd")
    return o, h_final


@_on_its_device
def decay_attn_bwd(q, k, v, rate, do, scale=None, cu=None, h0=None, dh_final=None, check=True, stream=None):
    """Gradients of decay_attn_fwd: (dq, dk, dv, dh0 [S,H,Dk,Dv]) from do (rows as
    o) and dh_final [S,H,Dk,Dv] (default 0); the rest as in the forward.  dq, dk
    and dv are dense, in the shapes of q, k and v; a head that several share has
    the sum of theirs.  The rates are constants, there is no gradient of them."""
    lead, T, S = _head_sequences(q, cu)
    d, rows, rate_at, (H, Dk, Dv), dev = _attn(q, k, v, rate, scale, S, lead, T)
    *do_at, heads = _heads(do, "do", q.dtype, lead, Dv, dev)
    do_at = _HEADS.pack(*do_at)
    if heads != H:
        raise ValueError("do must have the %d heads of rate, got %d" % (H, heads))
    h0_at, dhf_at = (_matrix_state(t, n, (S, H, Dk, Dv), dev) for t, n in ((h0, "h0"), (dh_final, "dh_final")))
    dq, dk, dv = (torch.empty(t.shape, dtype=t.dtype, device=dev) for t in (q, k, v))
    dh0 = rate.new_empty((S, H, Dk, Dv))
    ws = _attn_ws(d, cu, OP_BWD, dev)
    status = _status(check, dev)
    s = _on(stream, dev, (q, k, v, rate, do, cu, h0, dh_final, dq, dk, dv, dh0, ws, status))
    st = load().pdssm_decay_attn_bwd(d, *rows, do_at, rate_at, _at(cu), h0_at, dhf_at, dq.data_ptr(), dk.data_ptr(),
                                     dv.data_ptr(), dh0.data_ptr(), _at(ws), ws.numel() if ws is not None else 0,
                                     _at(status), s)
    _done(st, status, "pdssm_decay_attn_bwd")
    return dq, dk, dv, dh0


@_on_its_device
def decay_attn_step(q, k, v, rate, h, scale=None, slots=None, out=None, o=None, check=True, stream=None):
    """One token of decay_attn_fwd for each row of q [B,Hq,Dk], k [B,Hk,Dk] and
    v [B,Hv,Dv]: returns (h_new [S,H,Dk,Dv], o [B,H,Dv]).  h [S,H,Dk,Dv] holds the
    states; slots, out and skipped rows as in gated_step."""
    if not isinstance(q, torch.Tensor) or q.dim() != 3:
        raise ValueError("q must be [B,heads,D]")
    if not isinstance(h, torch.Tensor) or h.dim() != 4:
        raise ValueError("h must be [S,H,Dk,Dv]")
    B, S = q.shape[0], h.shape[0]
    d, rows, rate_at, (H, Dk, Dv), dev = _attn(q, k, v, rate, scale, S, q.shape[:1], B)
    h_at = _tensor(h, "h", torch.float32, (S, H, Dk, Dv), dev)
    out_at = h_at if out is None else _tensor(out, "out", torch.float32, (S, H, Dk, Dv), dev)
    slots_at = None if slots is None else _tensor(slots, "slots", torch.int32, (B,), dev)
    if o is None:
        o = q.new_empty((B, H, Dv))
        o_at = o.data_ptr()
    else:
        o_at = _tensor(o, "o", q.dtype, (B, H, Dv), dev)
    status = _status(check, dev)
    s = _on(stream, dev, (q, k, v, rate, h, out, slots, o, status))
    st = load().pdssm_decay_attn_step(d, *rows, rate_at, slots_at, h_at, out_at, o_at, _at(status), s)
    _done(st, status, "pdssm_decay_attn_step")
    return h if out is None else out, o


# ---- group norm --------------------------------------------------------------

_NORM_DESC = struct.Struct("4ifI")
_ACTS = {"none": 0, "silu": 1}


def _norm(x, groups, weight, bias, gate, act, eps):
    """(desc, rows of x, of gate or None, addresses of weight and bias, C, device)."""
    flags = _row_type(x)
    if x.dim() not in (2, 3):
        raise ValueError("x must be [T,C] or [B,L,C]")
    C, dev = x.shape[-1], x.device
    T = math.prod(x.shape[:-1])
    groups = int(groups)
    if C < 1 or groups < 1 or C % groups != 0:
        raise ValueError("groups must divide the %d channels, got %d" % (C, groups))
    if act not in _ACTS:
        raise ValueError("act must be 'none' or 'silu', got %r" % (act,))
    eps = float(eps)
    if not 0.0 <= eps < math.inf:
        raise ValueError("eps must be finite and not negative")
    _int32(T, C)
    rows = _rows(x, "x", x.dtype, x.shape, dev)
    gate_rows = None if gate is None else _rows(gate, "gate", x.dtype, x.shape, dev)
    w_at = None if weight is None else _tensor(weight, "weight", torch.float32, (C,), dev)
    b_at = None if bias is None else _tensor(bias, "bias", torch.float32, (C,), dev)
    return _NORM_DESC.pack(T, C, groups, _ACTS[act], eps, flags), rows, gate_rows, w_at, b_at, C, dev


@_on_its_device
def group_norm(x, groups, weight=None, bias=None, gate=None, act="none", eps=1e-5, stream=None):
    """Group norm of every row of x [T,C] or [B,L,C] over `groups` groups of
    neighbouring channels, u = (x - mean) / sqrt(var + eps) * weight + bias, and
    behind it act(u) or, with a gate (rows as x), u * act(gate); act is "none" or
    "silu".  weight and bias [C] are float32.  Returns y, dense, in x's type."""
    d, rows, gate_rows, w_at, b_at, _, dev = _norm(x, groups, weight, bias, gate, act, eps)
    y = torch.empty_like(x, memory_format=torch.contiguous_format)
    s = _on(stream, dev, (x, weight, bias, gate, y))
    _done(load().pdssm_group_norm(d, rows, gate_rows, w_at, b_at, y.data_ptr(), s), None, "pdssm_group_norm")
    return y


@_on_its_device
def group_norm_bwd(x, dy, groups, weight=None, bias=None, gate=None, act="none", eps=1e-5, stream=None):
    """Gradients of group_norm from dy (rows as y): (dx, dweight [C], dbias [C],
    dgate); dgate is None without a gate, dweight and dbias without theirs."""
    d, rows, gate_rows, w_at, b_at, C, dev = _norm(x, groups, weight, bias, gate, act, eps)
    dy_rows = _rows(dy, "dy", x.dtype, x.shape, dev)
    dx = torch.empty_like(x, memory_format=torch.contiguous_format)
    dgate = None if gate is None else torch.empty_like(dx)
    dw = None if weight is None else torch.empty_like(weight)
    db = None if bias is None else torch.empty_like(bias)
    n = 0
    if dw is not None or db is not None:
        n = load().pdssm_group_norm_workspace_size(d)
        if n == OP_SIZE_ERROR:
            raise PdssmError(ERR_UNSUPPORTED, "group_norm_workspace_size")
    ws = torch.empty(n, dtype=torch.uint8, device=dev) if n else None
    s = _on(stream, dev, (x, dy, weight, bias, gate, dx, dgate, dw, db, ws))
    _done(load().pdssm_group_norm_bwd(d, rows, gate_rows, dy_rows, w_at, b_at, dx.data_ptr(), _at(dgate), _at(dw), _at(db),
                                      _at(ws), n, s), None, "pdssm_group_norm_bwd")
    return dx, dw, db, dgate
