"""Host checks of linear attention and of the group norm (no GPU): bad arguments
are refused before anything is enqueued, by the C entry points and by the
binding.  The addresses are made up; nothing reads them."""
import ctypes
import inspect
import math
import os

import pytest
import torch

from paper_2605_19150_amd import pdssm
from paper_2605_19150_amd.pdssm import (ERR_INVALID_ARG, ERR_UNSUPPORTED, ERR_WORKSPACE, FLAG_BF16_IO, OP_BWD, OP_FWD, AttnDesc,
                                        Heads, NormDesc, Rows)

P = ctypes.byref
MB = 1 << 20
BAD = ctypes.c_size_t(-1).value


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(pdssm.lib_path()):
        from paper_2605_19150_amd.build import build_library
        build_library()
    return pdssm.load()


def _at(k):
    """A made-up address, 64 MiB apart from the others."""
    return None if k is None else (1 << 32) + 64 * MB * k


class Attn:
    """Arguments of a good call; attributes are changed to make it a bad one."""

    def __init__(self, lib, T=300, S=3, H=4, Hq=4, Hk=2, Hv=1, Dk=17, Dv=33, scale=0.5, flags=0):
        self.lib, self.d = lib, AttnDesc(T, S, H, Hq, Hk, Hv, Dk, Dv, scale, flags)
        self.q, self.k, self.v, self.do = (Heads(_at(k), 1000, 40, ) for k in (1, 2, 3, 4))
        self.rate, self.cu, self.h0, self.o, self.fin, self.ws, self.dhf = (_at(k) for k in range(5, 12))
        self.dq, self.dk, self.dv, self.dh0, self.status, self.slots, self.h_out = (_at(k) for k in range(12, 19))
        self.ws_bytes = 64 * MB

    def fwd(self):
        return self.lib.pdssm_decay_attn_fwd(P(self.d), P(self.q), P(self.k), P(self.v), self.rate, self.cu, self.h0, self.o,
                                             self.fin, self.ws, self.ws_bytes, self.status, None)

    def bwd(self):
        return self.lib.pdssm_decay_attn_bwd(P(self.d), P(self.q), P(self.k), P(self.v), P(self.do), self.rate, self.cu, self.h0,
                                             self.dhf, self.dq, self.dk, self.dv, self.dh0, self.ws, self.ws_bytes, self.status,
                                             None)

    def step(self):
        return self.lib.pdssm_decay_attn_step(P(self.d), P(self.q), P(self.k), P(self.v), self.rate, self.slots, self.h0,
                                              self.h_out, self.o, self.status, None)


SIZES = [("T", -1, ERR_INVALID_ARG), ("S", 0, ERR_INVALID_ARG), ("H", 0, ERR_INVALID_ARG), ("Hq", 3, ERR_INVALID_ARG),
         ("Hk", 0, ERR_INVALID_ARG), ("Hv", -4, ERR_INVALID_ARG), ("Dk", 0, ERR_INVALID_ARG), ("Dv", -1, ERR_INVALID_ARG),
         ("scale", math.inf, ERR_INVALID_ARG), ("scale", math.nan, ERR_INVALID_ARG), ("flags", 1, ERR_INVALID_ARG),
         ("flags", FLAG_BF16_IO | 8, ERR_INVALID_ARG), ("Dk", 257, ERR_UNSUPPORTED), ("Dv", 1024, ERR_UNSUPPORTED),
         ("T", (1 << 30) + 1, ERR_UNSUPPORTED), ("S", (1 << 30) + 1, ERR_UNSUPPORTED), ("H", 65536, ERR_UNSUPPORTED)]


@pytest.mark.parametrize("name,value,status", SIZES)
def test_sizes(lib, name, value, status):
    c = Attn(lib)
    setattr(c.d, name, value)
    assert c.fwd() == c.bwd() == c.step() == status
    assert lib.pdssm_decay_attn_workspace_size(P(c.d), 1, OP_FWD) == BAD


@pytest.mark.parametrize("name", ["q", "k", "v", "do"])
@pytest.mark.parametrize("change", [dict(p=None), dict(ld=-1), dict(hs=-1), dict(ld=(1 << 24) + 1), dict(hs=(1 << 40) + 1),
                                    dict(p=(1 << 40) + 2)], ids=str)
def test_rows(lib, name, change):
    c = Attn(lib)
    for f, v in change.items():
        setattr(getattr(c, name), f, v)
    assert c.bwd() == ERR_INVALID_ARG
    if name != "do":
        assert c.fwd() == c.step() == ERR_INVALID_ARG


@pytest.mark.parametrize("name,calls", [("rate", "fbs"), ("o", "fs"), ("dq", "b"), ("dk", "b"), ("dv", "b"), ("h0", "s"),
                                        ("h_out", "s")])
def test_missing_and_misaligned(lib, name, calls):
    for value in (None, _at(60) + 1):
        c = Attn(lib)
        setattr(c, name, value)
        for f, call in (("f", c.fwd), ("b", c.bwd), ("s", c.step)):
            if f in calls:
                assert call() == ERR_INVALID_ARG


@pytest.mark.parametrize("name,calls", [("cu", "fb"), ("h0", "fb"), ("fin", "f"), ("dhf", "b"), ("dh0", "b"), ("slots", "s"),
                                        ("status", "fbs")])
def test_misaligned_words(lib, name, calls):
    c = Attn(lib)
    setattr(c, name, _at(60) + 2)
    for f, call in (("f", c.fwd), ("b", c.bwd), ("s", c.step)):
        if f in calls:
            assert call() == ERR_INVALID_ARG


def test_missing_arguments(lib):
    c = Attn(lib)
    n = None
    assert lib.pdssm_decay_attn_fwd(n, n, n, n, n, n, n, n, n, n, 0, n, n) == ERR_INVALID_ARG
    assert lib.pdssm_decay_attn_fwd(P(c.d), n, P(c.k), P(c.v), c.rate, c.cu, n, c.o, n, c.ws, c.ws_bytes, n, n) == ERR_INVALID_ARG
    assert lib.pdssm_decay_attn_workspace_size(n, 0, OP_FWD) == BAD
    assert lib.pdssm_decay_attn_workspace_size(P(c.d), 0, 3) == BAD
    c.cu, c.d.S = None, 7  # 300 rows in 7 sequences
    assert c.fwd() == c.bwd() == ERR_INVALID_ARG
    c.slots = None  # 300 rows, 7 states
    assert c.step() == ERR_INVALID_ARG
    c.slots, c.d.T = _at(17), 65536
    assert c.step() == ERR_UNSUPPORTED


@pytest.mark.parametrize("out,into,calls", [("o", "q", "fs"), ("o", "h0", "fs"), ("fin", "h0", "f"), ("fin", "o", "f"),
                                            ("ws", "v", "fb"), ("ws", "cu", "fb"), ("dq", "q", "b"), ("dv", "dk", "b"),
                                            ("dh0", "dhf", "b"), ("dk", "do", "b"), ("dq", "rate", "b"), ("h_out", "k", "s")])
def test_overlaps(lib, out, into, calls):
    c = Attn(lib, T=4000, S=2)
    there = getattr(c, into)
    setattr(c, out, there.p if isinstance(there, Heads) else there)
    for f, call in (("f", c.fwd), ("b", c.bwd), ("s", c.step)):
        if f in calls:
            assert call() == ERR_INVALID_ARG


def test_part_overlap_of_a_pool(lib):
    c = Attn(lib)
    c.h_out = c.h0 + 64
    assert c.step() == ERR_INVALID_ARG


def test_workspace(lib):
    """Long sequences of few heads are cut into segments, whose states need room; shared heads need room for their users' gradients."""
    c = Attn(lib, T=30000, S=1, H=1, Hq=1, Hk=1, Hv=1, Dk=64, Dv=64)
    c.cu = None
    for call, op in ((c.fwd, OP_FWD), (c.bwd, OP_BWD)):
        need = lib.pdssm_decay_attn_workspace_size(P(c.d), 0, op)
        assert 0 < need < 64 * MB
        c.ws_bytes = need - 1
        assert call() == ERR_WORKSPACE
        c.ws_bytes, c.ws = need, None
        assert call() == ERR_WORKSPACE
        c.ws = _at(10) + 16
        assert call() == ERR_INVALID_ARG
        c.ws = _at(10)
    short = AttnDesc(64, 1, 16, 16, 16, 16, 64, 64, 1.0, 0)
    assert lib.pdssm_decay_attn_workspace_size(P(short), 0, OP_FWD) == lib.pdssm_decay_attn_workspace_size(P(short), 0, OP_BWD) == 0
    short.Hk = 4
    assert lib.pdssm_decay_attn_workspace_size(P(short), 0, OP_FWD) == 0
    assert lib.pdssm_decay_attn_workspace_size(P(short), 0, OP_BWD) > 0


def test_launches_past_the_grid(lib):
    d = AttnDesc(1 << 29, 1 << 29, 64, 64, 64, 64, 64, 64, 1.0, 0)
    assert lib.pdssm_decay_attn_workspace_size(P(d), 0, OP_FWD) == BAD
    c = Attn(lib)
    c.d = d
    c.cu = None
    assert c.fwd() == c.bwd() == ERR_UNSUPPORTED
    c.d = AttnDesc(65535, 65535, 65535, 65535, 65535, 65535, 1, 1, 1.0, 0)
    assert c.step() == ERR_UNSUPPORTED


M = 1 << 20


@pytest.mark.parametrize("H,Dk,Dv,T,op,fits,refused", [
    (8, 1, 72, 1000, OP_FWD, M - 8, M - 7),               # 7 segments more than sequences: states alone, more than 64 columns
    (1, 1, 72, 1000, OP_BWD, 4 * M - 15, 4 * M - 7),      # two scans of states alone
    (8, 129, 65, None, OP_FWD, M - 1, M),                 # rows past 128 entries
    (2, 130, 256, None, OP_BWD, 699048, 699052),          # six workgroups a head
    (8, 1, 72, 100, OP_FWD, 2 * M - 1, 2 * M),            # 256 threads each: nothing is cut
    (8, 128, 65, None, OP_FWD, 2 * M - 1, 2 * M)], ids=str)
def test_launches_of_512_threads(lib, H, Dk, Dv, T, op, fits, refused):
    """2^32 threads and more are refused: 2^23 workgroups of the scan where they have 512 threads, 2^24 where they have 256.
    T rows of packed sequences, or a row for each."""
    for S, bad in ((fits, False), (refused, True)):
        d = AttnDesc(T or S, S, H, H, H, H, Dk, Dv, 1.0, 0)
        assert (lib.pdssm_decay_attn_workspace_size(P(d), int(T is not None), op) == BAD) == bad
    c = Attn(lib)
    c.d, c.ws, c.h0, c.fin, c.dhf, c.dh0 = d, _at(10), None, None, None, None
    c.cu = c.cu if T else None
    assert (c.fwd if op == OP_FWD else c.bwd)() == ERR_UNSUPPORTED


class Norm:
    def __init__(self, lib, T=300, C=96, G=6, act=1, eps=1e-5, flags=0):
        self.lib, self.d = lib, NormDesc(T, C, G, act, eps, flags)
        self.x, self.gate, self.dy = (Rows(_at(k), C, None) for k in (1, 2, 3))
        self.w, self.b, self.y, self.dx, self.dgate, self.dw, self.db, self.ws = (_at(k) for k in range(4, 12))
        self.ws_bytes = 64 * MB

    def fwd(self):
        return self.lib.pdssm_group_norm(P(self.d), P(self.x), P(self.gate), self.w, self.b, self.y, None)

    def bwd(self):
        return self.lib.pdssm_group_norm_bwd(P(self.d), P(self.x), P(self.gate), P(self.dy), self.w, self.b, self.dx, self.dgate,
                                             self.dw, self.db, self.ws, self.ws_bytes, None)


@pytest.mark.parametrize("name,value,status", [
    ("T", -1, ERR_INVALID_ARG), ("C", 0, ERR_INVALID_ARG), ("G", 0, ERR_INVALID_ARG), ("G", 5, ERR_INVALID_ARG),
    ("act", 2, ERR_INVALID_ARG), ("act", -1, ERR_INVALID_ARG), ("eps", -1e-9, ERR_INVALID_ARG), ("eps", math.inf, ERR_INVALID_ARG),
    ("eps", math.nan, ERR_INVALID_ARG), ("flags", 8, ERR_INVALID_ARG), ("T", (1 << 30) + 1, ERR_UNSUPPORTED)])
def test_norm_sizes(lib, name, value, status):
    c = Norm(lib)
    setattr(c.d, name, value)
    assert c.fwd() == c.bwd() == status and lib.pdssm_group_norm_workspace_size(P(c.d)) == BAD


def test_norm_sizes_past_the_grid(lib):
    for d in (NormDesc(4, 1 << 25, 1, 0, 0.0, 0), NormDesc(1024, 1 << 20, 1 << 20, 0, 0.0, 0)):
        c = Norm(lib)
        c.d = d
        for r in (c.x, c.gate, c.dy):
            r.ld = 1 << 24
        assert c.fwd() == c.bwd() == ERR_UNSUPPORTED


@pytest.mark.parametrize("name", ["x", "gate", "dy"])
@pytest.mark.parametrize("change", [dict(p=None), dict(ld=95), dict(ld=(1 << 24) + 1), dict(p=_at(1) + 2), dict(e=_at(50))], ids=str)
def test_norm_rows(lib, name, change):
    c = Norm(lib)
    for f, v in change.items():
        setattr(getattr(c, name), f, v)
    assert c.bwd() == ERR_INVALID_ARG
    if name != "dy":
        assert c.fwd() == ERR_INVALID_ARG


def test_norm_pointers(lib):
    for name, value, calls in (("y", None, "f"), ("y", _at(30) + 2, "f"), ("w", _at(30) + 2, "fb"), ("b", _at(30) + 1, "fb"),
                               ("dx", None, "b"), ("dgate", None, "b"), ("dw", _at(30) + 2, "b"), ("db", _at(30) + 2, "b"),
                               ("y", _at(1), "f"), ("y", _at(4), "f"), ("dx", _at(3), "b"), ("dgate", _at(7), "b"),
                               ("dw", _at(10), "b"), ("ws", _at(2), "b"), ("ws", _at(30) + 8, "b")):
        c = Norm(lib)
        setattr(c, name, value)
        for f, call in (("f", c.fwd), ("b", c.bwd)):
            if f in calls:
                assert call() == ERR_INVALID_ARG, (name, value)
    c = Norm(lib)
    c.ws_bytes = lib.pdssm_group_norm_workspace_size(P(c.d)) - 1
    assert c.bwd() == ERR_WORKSPACE


# ---- the binding -----------------------------------------------------------------------------------------------------

FUNCTIONS = [pdssm.decay_attn_fwd, pdssm.decay_attn_bwd, pdssm.decay_attn_step, pdssm.group_norm, pdssm.group_norm_bwd]


def _arguments(f):
    step = f is pdssm.decay_attn_step
    rows = torch.zeros(4, 2, 16) if step else torch.zeros(1, 4, 2, 16) if "attn" in f.__name__ else torch.zeros(4, 16)
    special = dict(rate=torch.zeros(2), h=torch.zeros(4, 2, 16, 16), groups=2)
    return {p.name: special.get(p.name, rows) for p in inspect.signature(f).parameters.values() if p.default is p.empty}


@pytest.mark.parametrize("f", FUNCTIONS, ids=lambda f: f.__name__)
def test_every_argument_by_its_name(lib, f):
    """Both forms of a call end at the same check: these tensors are not on a GPU."""
    kw = _arguments(f)
    with pytest.raises(ValueError, match="must be on") as by_place:
        f(*kw.values())
    with pytest.raises(ValueError, match="must be on") as by_name:
        f(**kw)
    assert str(by_place.value) == str(by_name.value)


def test_packed_arguments_are_the_structures():
    assert pdssm._ATTN_DESC.size == ctypes.sizeof(AttnDesc) and pdssm._HEADS.size == ctypes.sizeof(Heads)
    assert pdssm._NORM_DESC.size == ctypes.sizeof(NormDesc)
    a = AttnDesc.from_buffer_copy(pdssm._ATTN_DESC.pack(1, 2, 3, 4, 5, 6, 7, 8, 0.5, 2))
    assert [getattr(a, n) for n, _ in AttnDesc._fields_] == [1, 2, 3, 4, 5, 6, 7, 8, 0.5, 2]
    n = NormDesc.from_buffer_copy(pdssm._NORM_DESC.pack(1, 2, 3, 1, 0.25, 2))
    assert [getattr(n, f) for f, _ in NormDesc._fields_] == [1, 2, 3, 1, 0.25, 2]


class _Fake(torch.Tensor):
    """A tensor of the CPU that says that it is on a GPU: the checks before the library see it."""

    @property
    def is_cuda(self):
        return True

    @property
    def device(self):
        return torch.device("cuda", 0)


def _fake(*shape, dtype=torch.float32):
    return torch.zeros(*shape, dtype=dtype).as_subclass(_Fake)


@pytest.mark.parametrize("change,error,match", [
    (dict(k=_fake(1, 4, 3, 16)), ValueError, "divide"), (dict(k=_fake(1, 4, 2, 8)), ValueError, "shape"),
    (dict(v=_fake(1, 5, 2, 16)), ValueError, "shape"), (dict(v=_fake(4, 2, 16)), ValueError, "v must be rows"),
    (dict(q=_fake(4, 2, 16)), ValueError, "rows must be"), (dict(q=_fake(1, 4, 2, 16, dtype=torch.float16)), TypeError, "float32"),
    (dict(k=_fake(1, 4, 2, 16, dtype=torch.bfloat16)), TypeError, "k must be"), (dict(rate=_fake(2, 1)), ValueError, "rate"),
    (dict(rate=_fake(2, dtype=torch.float64)), TypeError, "rate"), (dict(scale=math.inf), ValueError, "scale"),
    (dict(cu=_fake(3, dtype=torch.int32)), ValueError, "rows must be"), (dict(k=_fake(1, 4, 2, 32)[..., ::2]), ValueError, "next to"),
    (dict(q=_fake(2, 2, 4, 16)[:, :, :2], k=_fake(2, 4, 2, 16)[:, :2], v=_fake(2, 2, 2, 16)), ValueError, "evenly"),
    (dict(q=_fake(1, 4, 2, 300), k=_fake(1, 4, 2, 300)), ValueError, "256"), (dict(h0=_fake(1, 2, 16, 8)), ValueError, "h0"),
    (dict(v=None), ValueError, "v must be"), (dict(rate=None), ValueError, "rate")], ids=lambda c: str(c)[:40] if isinstance(c, dict) else "")
def test_attention_refuses(lib, change, error, match):
    kw = dict(q=_fake(1, 4, 2, 16), k=_fake(1, 4, 2, 16), v=_fake(1, 4, 2, 16), rate=_fake(2))
    with pytest.raises(error, match=match):
        pdssm.decay_attn_fwd.__wrapped__(**{**kw, **change})


@pytest.mark.parametrize("change,error,match", [
    (dict(groups=3), ValueError, "groups"), (dict(groups=0), ValueError, "groups"), (dict(act="relu"), ValueError, "act"),
    (dict(eps=-1.0), ValueError, "eps"), (dict(eps=math.nan), ValueError, "eps"), (dict(x=_fake(16)), ValueError, "x must be"),
    (dict(weight=_fake(8)), ValueError, "weight"), (dict(bias=_fake(16, dtype=torch.bfloat16)), TypeError, "bias"),
    (dict(gate=_fake(4, 8)), ValueError, "gate"), (dict(gate=_fake(4, 16, dtype=torch.bfloat16)), TypeError, "gate"),
    (dict(x=_fake(4, 32)[:, ::2]), ValueError, "next to")], ids=lambda c: str(c)[:40] if isinstance(c, dict) else "")
def test_norm_refuses(lib, change, error, match):
    with pytest.raises(error, match=match):
        pdssm.group_norm.__wrapped__(**{**dict(x=_fake(4, 16), groups=2), **change})
