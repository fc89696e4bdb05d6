"""How the binding of the gated operators is called (no GPU): what it checks
before it reaches the library."""
import ctypes
import inspect

import pytest
import torch

from paper_2605_19150_amd import pdssm

FUNCTIONS = [pdssm.gated_fwd, pdssm.gated_bwd, pdssm.gated_step, pdssm.pack8, pdssm.unpack8, pdssm.project_wgrad]


@pytest.mark.parametrize("f", FUNCTIONS, ids=lambda f: f.__name__)
def test_every_argument_by_its_name(f):
    """Both forms of a call end at the same check: these tensors are not on a GPU."""
    rows, pair = torch.zeros(1, 4, 16), (torch.zeros(4, 16, dtype=torch.int8), torch.zeros(1, 16, dtype=torch.int8))
    special = dict(rate=torch.zeros(16), saved=torch.zeros(1, 16), h=torch.zeros(4, 16), pair=pair, u8=pair,
                   dP=torch.zeros(4, 8, dtype=torch.bfloat16))
    names = [p.name for p in inspect.signature(f).parameters.values() if p.default is p.empty]
    kw = {n: special.get(n, rows[0] if f is pdssm.gated_step else rows) for n in names}
    with pytest.raises(ValueError, match="must be on") as by_place:
        f(*kw.values())
    with pytest.raises(ValueError, match="must be on") as by_name:
        f(**kw)
    assert str(by_place.value) == str(by_name.value)


def test_a_call_without_arguments_names_them():
    with pytest.raises(TypeError, match="'u'"):
        pdssm.pack8()


class _Stream:
    """As much of a torch.cuda.Stream as the binding looks at."""

    def __init__(self, device, cuda_stream):
        self.device, self.cuda_stream = torch.device(device), cuda_stream

    def wait_stream(self, other):
        self.waited = other


def test_a_stream_of_another_device_is_refused(monkeypatch):
    """A kernel launched there would run on that device, on memory of this one."""
    monkeypatch.setattr(pdssm, "_raw_stream", lambda index: 0)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: "current")
    dev = torch.device("cuda", 0)
    for raw in (0, 4096):  # the default stream of every device has the number 0
        with pytest.raises(ValueError, match="stream"):
            pdssm._on(_Stream("cuda:1", raw), dev, ())
    own = _Stream("cuda:0", 4096)
    assert pdssm._on(own, dev, ()) == 4096 and own.waited == "current"
    assert pdssm._on(_Stream("cuda:0", 0), dev, ()) == 0 and pdssm._on(None, dev, ()) == 0


def test_flags_of_the_passes_and_the_step():
    """Zeros behind the last sequence are for the two passes; the step has no such rows."""
    lib = pdssm.load()
    bad = ctypes.c_size_t(-1).value
    for flags in (pdssm.FLAG_ZERO_REST, pdssm.FLAG_ZERO_REST | pdssm.FLAG_BF16_IO):
        d, r = pdssm._DESC.pack(4, 16, 4, flags), pdssm._ROW.pack(1 << 32, 16, 0)
        for op in (pdssm.OP_FWD, pdssm.OP_BWD):
            assert lib.pdssm_gated_workspace_size(d, op) != bad
        far = [(1 << 33) + (k << 26) for k in range(5)]
        assert lib.pdssm_gated_step(d, r, r, r, far[0], None, far[1], far[2], far[3], None, None) == pdssm.ERR_INVALID_ARG
    assert lib.pdssm_gated_workspace_size(pdssm._DESC.pack(4, 16, 4, 16), pdssm.OP_FWD) == bad


def test_packed_arguments_are_the_structures():
    """The binding packs pdssm_gated_desc and pdssm_rows itself; the ctypes structures say the same."""
    assert pdssm._DESC.pack(1000, 65, 7, 10) == bytes(pdssm.GatedDesc(1000, 65, 7, 10))
    assert pdssm._ROW.pack(1 << 40, 77, 1 << 33) == bytes(pdssm.Rows(1 << 40, 77, 1 << 33))
    assert pdssm._ROW.pack(1 << 40, 77, 0) == bytes(pdssm.Rows(1 << 40, 77, None))
