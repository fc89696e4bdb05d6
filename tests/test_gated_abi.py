"""Host checks of the gated recurrent operators' C entry points (no GPU): bad
arguments are refused before anything is enqueued.  The addresses are made up;
nothing reads them."""
import ctypes
import os

import pytest

from paper_2605_19150_amd import pdssm
from paper_2605_19150_amd.pdssm import ERR_INVALID_ARG, ERR_UNSUPPORTED, ERR_WORKSPACE, FLAG_BF16_IO, GatedDesc, Rows

P = ctypes.byref
MB = 1 << 20


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(pdssm.lib_path()):
        from paper_2605_19150_amd.build import build_library
        build_library()
    return pdssm.load()


def _at(k):
    """A made-up address, 64 MiB apart from the others."""
    return None if k is None else (1 << 32) + 64 * MB * k


class Call:
    """Arguments of a good call; attributes are changed to make it a bad one."""

    def __init__(self, lib, T=300, C=65, S=3, flags=0):
        self.lib, self.d = lib, GatedDesc(T, C, S, flags)
        self.x, self.ga, self.gi, self.dy = (Rows(_at(k), C, None) for k in (1, 2, 3, 4))
        self.rate, self.cu, self.h0, self.y, self.fin, self.saved, self.ws = (_at(k) for k in range(5, 12))
        self.q = [_at(12), _at(13), _at(14)]
        self.e = [_at(15), _at(16), _at(17)]
        self.dhf, self.drate, self.dh0, self.status = (_at(k) for k in (18, 19, 20, 21))
        self.dd, self.ldd = [_at(22), _at(23), _at(24)], C
        self.slots, self.h_out = _at(25), _at(26)
        self.ws_bytes = 64 * MB

    @staticmethod
    def _three(v):
        return None if v is None else (ctypes.c_void_p * 3)(*v)

    def fwd(self):
        return self.lib.pdssm_gated_fwd(P(self.d), P(self.x), P(self.ga), P(self.gi), self.rate, self.cu, self.h0, self.y,
                                        self.fin, self.saved, self._three(self.q), self._three(self.e), self.ws,
                                        self.ws_bytes, self.status, None)

    def bwd(self):
        return self.lib.pdssm_gated_bwd(P(self.d), P(self.x), P(self.ga), P(self.gi), self.rate, self.cu, self.h0,
                                        self.saved, P(self.dy), self.dhf, self._three(self.dd), self.ldd, self.drate,
                                        self.dh0, self.ws, self.ws_bytes, self.status, None)

    def step(self):
        return self.lib.pdssm_gated_step(P(self.d), P(self.x), P(self.ga), P(self.gi), self.rate, self.slots, self.h0,
                                         self.h_out, self.y, self.status, None)


@pytest.mark.parametrize("change,code", [
    (lambda c: setattr(c.d, "flags", 1), ERR_INVALID_ARG),
    (lambda c: setattr(c.d, "flags", 4), ERR_INVALID_ARG),
    (lambda c: setattr(c.d, "T", -1), ERR_INVALID_ARG),
    (lambda c: setattr(c.d, "C", 0), ERR_INVALID_ARG),
    (lambda c: setattr(c.d, "S", 0), ERR_INVALID_ARG),
    (lambda c: (setattr(c.d, "C", 1 << 30), setattr(c.d, "T", 1 << 30)), ERR_UNSUPPORTED),
    (lambda c: setattr(c.d, "T", (1 << 30) + 1), ERR_UNSUPPORTED),
    (lambda c: setattr(c.d, "T", 1 << 30), ERR_UNSUPPORTED),  # 2^32 threads and more
    (lambda c: setattr(c.d, "S", (1 << 30) + 1), ERR_UNSUPPORTED),
    (lambda c: (setattr(c.d, "C", (1 << 24) + 1), setattr(c.d, "T", 1)), ERR_UNSUPPORTED),
    (lambda c: setattr(c.x, "ld", (1 << 24) + 1), ERR_INVALID_ARG),
    (lambda c: setattr(c.x, "p", None), ERR_INVALID_ARG),
    (lambda c: setattr(c.ga, "ld", 64), ERR_INVALID_ARG),
    (lambda c: setattr(c.gi, "p", _at(3) + 2), ERR_INVALID_ARG),
    (lambda c: setattr(c.x, "e", _at(30)), ERR_INVALID_ARG),
    (lambda c: setattr(c, "rate", None), ERR_INVALID_ARG),
    (lambda c: setattr(c, "rate", _at(5) + 1), ERR_INVALID_ARG),
    (lambda c: setattr(c, "cu", _at(6) + 2), ERR_INVALID_ARG),
    (lambda c: (setattr(c, "cu", None), setattr(c.d, "S", 7)), ERR_INVALID_ARG),   # 300 rows are not 7 sequences
    (lambda c: setattr(c, "h0", _at(7) + 2), ERR_INVALID_ARG),
])
def test_refused_by_both_passes(lib, change, code):
    for name in ("fwd", "bwd"):
        c = Call(lib)
        change(c)
        assert getattr(c, name)() == code, name


@pytest.mark.parametrize("change", [
    lambda c: setattr(c, "y", None), lambda c: setattr(c, "y", _at(8) + 2), lambda c: setattr(c, "e", None),
    lambda c: setattr(c, "q", [_at(12), None, _at(14)]), lambda c: setattr(c, "y", _at(1) + 400),
    lambda c: setattr(c, "saved", _at(8) + 4000), lambda c: setattr(c, "fin", _at(7)),
    lambda c: setattr(c, "e", [_at(15), _at(16), _at(12) + 60]),
])
def test_refused_by_the_forward(lib, change):
    c = Call(lib)
    change(c)
    assert c.fwd() == ERR_INVALID_ARG


@pytest.mark.parametrize("change", [
    lambda c: setattr(c, "saved", None), lambda c: setattr(c.dy, "p", None), lambda c: setattr(c.dy, "e", _at(30)),
    lambda c: setattr(c, "ldd", 64), lambda c: setattr(c, "dd", [_at(22), _at(23), None]),
    lambda c: setattr(c.ga, "e", _at(30)),                                     # one of three in the 8-bit form
    lambda c: setattr(c, "dd", [_at(22), _at(22) + 64 * 4, _at(24)]),          # parts of a row that overlap
    lambda c: (setattr(c, "ldd", 195), setattr(c, "dd", [_at(22), _at(22) + 65 * 4, _at(22) + 129 * 4])),
    lambda c: (setattr(c, "ldd", 194), setattr(c, "dd", [_at(22), _at(22) + 65 * 4, _at(22) + 130 * 4])),
    lambda c: setattr(c, "dd", [_at(4), _at(23), _at(24)]), lambda c: setattr(c, "drate", _at(5)),
    lambda c: setattr(c, "dh0", _at(18)), lambda c: setattr(c, "drate", _at(22) + 260),
])
def test_refused_by_the_backward(lib, change):
    c = Call(lib)
    change(c)
    assert c.bwd() == ERR_INVALID_ARG


@pytest.mark.parametrize("op,name", [(pdssm.OP_FWD, "fwd"), (pdssm.OP_BWD, "bwd")])
def test_workspace(lib, op, name):
    c = Call(lib)
    need = lib.pdssm_gated_workspace_size(P(c.d), op)
    if need:
        c.ws_bytes = need - 1
        assert getattr(c, name)() == ERR_WORKSPACE
        c.ws = None
        assert getattr(c, name)() == ERR_WORKSPACE
        c = Call(lib)
        c.ws += 16
        assert getattr(c, name)() == ERR_INVALID_ARG
        c.ws = c.y if op == pdssm.OP_FWD else c.dd[0]
        assert getattr(c, name)() == ERR_INVALID_ARG
    bad = ctypes.c_size_t(-1).value
    assert lib.pdssm_gated_workspace_size(P(c.d), 0) == bad
    assert lib.pdssm_gated_workspace_size(P(c.d), pdssm.OP_COMPOSE) == bad
    assert lib.pdssm_gated_workspace_size(None, op) == bad
    assert lib.pdssm_gated_workspace_size(P(GatedDesc(4, 0, 1, 0)), op) == bad


@pytest.mark.parametrize("change,code", [
    (lambda c: setattr(c.d, "T", 65536), ERR_UNSUPPORTED),
    (lambda c: setattr(c, "slots", None), ERR_INVALID_ARG),       # 300 rows, 3 states
    (lambda c: setattr(c, "slots", _at(25) + 1), ERR_INVALID_ARG),
    (lambda c: setattr(c, "h0", None), ERR_INVALID_ARG),
    (lambda c: setattr(c, "h_out", None), ERR_INVALID_ARG),
    (lambda c: setattr(c, "h_out", _at(7) + 4), ERR_INVALID_ARG),  # neither in place nor apart
    (lambda c: setattr(c, "y", _at(7)), ERR_INVALID_ARG),
    (lambda c: setattr(c, "h_out", _at(2)), ERR_INVALID_ARG),
    (lambda c: setattr(c.x, "e", _at(30)), ERR_INVALID_ARG),
])
def test_refused_by_the_step(lib, change, code):
    c = Call(lib)
    change(c)
    assert c.step() == code


def test_step_without_rows(lib):
    c = Call(lib, T=0)
    c.x.p = c.ga.p = c.gi.p = c.y = None
    assert c.step() == 0


def test_pack_and_unpack(lib):
    u = Rows(_at(1), 40, None)
    assert lib.pdssm_pack8(0, 40, 0, P(Rows(None, 40, None)), None, None, None) == 0
    assert lib.pdssm_unpack8(0, 40, FLAG_BF16_IO, None, None, None, None) == 0
    for args in ((-1, 40, 0, P(u), _at(2), _at(3)), (9, 0, 0, P(u), _at(2), _at(3)), (9, 40, 1, P(u), _at(2), _at(3)),
                 (9, 41, 0, P(u), _at(2), _at(3)), (9, 40, 0, P(u), None, _at(3)), (9, 40, 0, P(u), _at(2), None),
                 (9, 40, 0, P(u), _at(1) + 9 * 160 - 1, _at(3)), (9, 40, 0, P(u), _at(2), _at(2) + 359),
                 (9, 40, 0, P(Rows(_at(1) + 2, 40, None)), _at(2), _at(3)), (9, 40, 0, P(Rows(_at(1), 40, _at(9))), _at(2), _at(3))):
        assert lib.pdssm_pack8(*args, None) == ERR_INVALID_ARG, args[:3]
    for args in ((9, 40, 0, None, _at(2), _at(3)), (9, 40, 0, _at(1), None, _at(3)), (9, 40, 0, _at(1), _at(2), None),
                 (9, 40, 0, _at(1), _at(2), _at(3) + 1), (9, 40, FLAG_BF16_IO, _at(1), _at(2), _at(3) + 1),
                 (9, 40, 2 + 4, _at(1), _at(2), _at(3)), (9, 40, 0, _at(1), _at(2), _at(1) + 356)):
        assert lib.pdssm_unpack8(*args, None) == ERR_INVALID_ARG, args[:3]
    for T, C in (((1 << 30) + 1, 1), (1, (1 << 24) + 1), (1 << 30, 64), (1 << 24, 1 << 12)):
        assert lib.pdssm_pack8(T, C, 0, P(Rows(_at(1), C, None)), _at(2), _at(3), None) == ERR_UNSUPPORTED
        assert lib.pdssm_unpack8(T, C, 0, _at(1), _at(2), _at(3), None) == ERR_UNSUPPORTED


def test_weight_gradient(lib):
    size = lib.pdssm_project_wgrad_workspace_size
    bad = ctypes.c_size_t(-1).value
    for T, M, Dm, code in ((-1, 16, 16, ERR_INVALID_ARG), (4, 0, 16, ERR_INVALID_ARG), (4, 16, 0, ERR_INVALID_ARG),
                           (4, 12, 16, ERR_UNSUPPORTED), (4, 16, 24, ERR_UNSUPPORTED), (4, 1 << 16, 1 << 16, ERR_UNSUPPORTED),
                           ((1 << 31) - 1, 1 << 10, 16, ERR_UNSUPPORTED), ((1 << 30) + 1, 16, 16, ERR_UNSUPPORTED),
                           (4, 1 << 21, 16, ERR_UNSUPPORTED)):
        assert size(T, M, Dm) == bad
        assert lib.pdssm_project_wgrad(T, M, Dm, _at(1), _at(2), _at(3), _at(4), _at(5), 64 * MB, None) == code
    T, M, Dm = 5000, 16, 32
    need = size(T, M, Dm)
    good = [_at(1), _at(2), _at(3), _at(4), _at(5), 64 * MB]
    for k, v in ((0, None), (1, None), (2, None), (3, None), (0, _at(1) + 8), (1, _at(2) + 8), (2, _at(3) + 8), (3, _at(4) + 4),
                 (3, _at(1)), (3, _at(2) + 64), (3, _at(3))):
        args = list(good)
        args[k] = v
        assert lib.pdssm_project_wgrad(T, M, Dm, *args, None) == ERR_INVALID_ARG, (k, v)
    if need:
        assert lib.pdssm_project_wgrad(T, M, Dm, *good[:4], None, 64 * MB, None) == ERR_WORKSPACE
        assert lib.pdssm_project_wgrad(T, M, Dm, *good[:5], need - 1, None) == ERR_WORKSPACE
        assert lib.pdssm_project_wgrad(T, M, Dm, *good[:4], _at(5) + 64, 64 * MB, None) == ERR_INVALID_ARG


@pytest.mark.parametrize("sizes", [((1 << 32) + 5, 4, 1), (4, (1 << 32) + 5, 1), (4, 4, (1 << 32) + 1)])
def test_sizes_past_32_bits_are_not_cut(sizes):
    """They would otherwise arrive in the library as their low 32 bits."""
    with pytest.raises(pdssm.PdssmError, match="UNSUPPORTED"):
        pdssm._desc(*sizes, 0)
    with pytest.raises(pdssm.PdssmError, match="UNSUPPORTED"):
        pdssm._kept((None, None), "u", *sizes[:2], None) if max(sizes[:2]) > 4 else pdssm._int32(*sizes)
