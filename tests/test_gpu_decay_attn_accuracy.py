"""Attention with bf16 rows as a whole, head by head: row outputs are off by the
rounding of the output and little else, states by what fp32 sums make
(oracle.decay_attn.ROWS_OFF and STATES_OFF, which say why; what they see is
tested without a GPU)."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import decay_attn as R
from paper_2605_19150_amd import pdssm
from test_gpu_decay_attn import DEV, Case, _np

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


def _fill(H, D, bounds, share=1, seed=0, **kw):
    return Case(bounds, H, *D, BF16, heads=(H, H // share, H // share), seed=seed, **kw)


def _check(c, got, grads, picked, share=1):
    """Heads of keys and values in picked, and the users of each, against the reference."""
    users = [h * share + k for h in picked for k in range(share)]
    of = lambda t, heads: _np(t.reshape(c.T, -1, t.shape[-1])[:, heads])  # noqa: E731
    q, k, v, do = of(c.q, users), of(c.k, picked), of(c.v, picked), of(c.do, users)
    rate, h0, dhf = _np(c.rate)[users], _np(c.h0[:, users]), _np(c.dhf[:, users])
    o, fin = R.fwd(q, k, v, rate, c.scale, c.bounds, h0)
    want = R.bwd(q, k, v, rate, do, c.scale, c.bounds, h0, dhf)
    for name, x, heads, y in (("o", got[0], users, o), ("dq", grads[0], users, want["dq"]), ("dk", grads[1], picked, want["dk"]),
                              ("dv", grads[2], picked, want["dv"])):
        off = R.rows_off(of(x, heads), y)
        assert (off < R.ROWS_OFF).all(), (name, off)
    for name, x, y in (("h_final", got[1], fin), ("dh0", grads[3], want["dh0"])):
        off = R.states_off(_np(x[:, users]), y)
        assert (off < _states_bound(c)).all(), (name, off)


def _states_bound(c):
    # weights of chunks, rounded to fp32, multiply where a state outlives several of them
    return R.STATES_OFF + 2.0 ** -24 * min(c.longest / 64, 1 / (64 * float(c.rate.min())))


@pytest.mark.parametrize("H,D,share", [(300, (64, 64), 1), (300, (40, 64), 1), (140, (128, 128), 1), (140, (96, 72), 2),
                                       (130, (200, 72), 1), (130, (72, 256), 1), (320, (64, 64), 4)], ids=str)
def test_calls_that_fill_the_card(H, D, share):
    c = _fill(H, D, [0, 70, 271], share, seed=H)
    _check(c, c.fwd(), c.bwd(), [0, H // share // 2, H // share - 1], share)


@pytest.mark.parametrize("H,D,share,pad", [(2, (64, 64), 1, 0), (4, (40, 64), 2, 1), (2, (128, 96), 1, 2), (1, (256, 256), 1, 0)],
                         ids=str)
def test_calls_that_leave_cus_idle(H, D, share, pad):
    """Few heads, some of whose sequences are cut; rows at odd addresses, too."""
    c = _fill(H, D, [0, 0, 1200, 1200, 1500], share, pad=pad, seed=pad, rate=[2.0 ** -3 / 4 ** h for h in range(H)])
    _check(c, c.fwd(), c.bwd(), list(range(H // share)), share)


@pytest.mark.parametrize("H", [1, 300])
@pytest.mark.parametrize("centre", [1.0, 4.0, 10.0])
@pytest.mark.parametrize("which", ["qk", "vdo"])
def test_rows_that_cancel(which, centre, H):
    """Keys or values off centre, and what they are multiplied by without a constant part, as the gradient of a norm is: the
    state's entries are much larger than their sum."""
    c = _fill(H, (64, 64), [0, 1024], states=False, rate=[2.0 ** -9] if H == 1 else np.geomspace(2.0 ** -2, 2.0 ** -9, H, dtype=np.float32))
    c.h0 = torch.zeros(1, H, 64, 64, device=DEV)
    c.dhf = torch.zeros_like(c.h0)
    flat, shifted = (c.q, c.k) if which == "qk" else (c.do, c.v)
    flat.copy_(flat.float() - flat.float().mean(2, keepdim=True))
    shifted.copy_(shifted.float() + centre)
    _check(c, c.fwd(), c.bwd(), [0, H // 2, H - 1] if H > 1 else [0])

def test_rows_do_not_depend_on_whether_states_are_asked_for():
    """The C entries without h_final and without dh0, in a call that fills the card."""
    H, D, T = 300, 64, 200
    c = _fill(H, (D, D), [0, 70, T])
    (o, _), (dq, dk, dv, _) = c.fwd(), c.bwd()
    desc = ctypes.byref(pdssm.AttnDesc(T, 2, H, H, H, H, D, D, c.scale, pdssm.FLAG_BF16_IO))
    heads = [ctypes.byref(pdssm.Heads(t.data_ptr(), t.stride(0), t.stride(1))) for t in (c.q, c.k, c.v, c.do)]
    lib, at = pdssm.load(), lambda t: t.data_ptr()  # noqa: E731
    ws = [torch.empty(max(lib.pdssm_decay_attn_workspace_size(desc, 1, op), 1), dtype=torch.uint8, device=DEV)
          for op in (pdssm.OP_FWD, pdssm.OP_BWD)]
    outs = [torch.empty_like(t) for t in (o, dq, dk, dv)]
    s = torch.cuda.current_stream().cuda_stream
    assert lib.pdssm_decay_attn_fwd(desc, *heads[:3], at(c.rate), at(c.cu), at(c.h0), at(outs[0]), None, at(ws[0]), ws[0].numel(),
                                    None, s) == 0
    assert lib.pdssm_decay_attn_bwd(desc, *heads, at(c.rate), at(c.cu), at(c.h0), at(c.dhf), *(at(t) for t in outs[1:]), None,
                                    at(ws[1]), ws[1].numel(), None, s) == 0
    for name, x, y in zip(("o", "dq", "dk", "dv"), outs, (o, dq, dk, dv)):
        assert torch.equal(x, y), name



@pytest.mark.parametrize("H,D,share", [(29, 40, 1), (23, 48, 1), (12, 96, 1), (12, 104, 2)], ids=str)
def test_large_outputs_whose_rows_are_no_whole_lines(H, D, share):
    """64 MB and more of rows of 80, 96, 192 and 208 bytes; two heads of two sequences against the reference."""
    L, S = 2048, 16
    c = Case(list(range(0, S * L + 1, L)), H, D, D, BF16, heads=(H, H // share, H // share), dense=True, seed=D)
    got, grads = c.fwd(), c.bwd()
    picked = [1, H // share - 1]
    users = [h * share + k for h in picked for k in range(share)]
    part = Case([0, L, 2 * L], len(users), D, D, BF16, heads=(len(users), len(picked), len(picked)), dense=True, states=False)
    of = lambda t, heads: t.reshape(S * L, -1, D)[2 * L:4 * L, heads]  # noqa: E731
    part.q, part.k, part.v, part.do = of(c.q, users), of(c.k, picked), of(c.v, picked), of(c.do, users)
    part.rate, part.h0, part.dhf = c.rate[users], c.h0[2:4, users], c.dhf[2:4, users]
    _check(part, (of(got[0], users), got[1][2:4, users]), (of(grads[0], users), of(grads[1], picked), of(grads[2], picked),
                                                          grads[3][2:4, users]), list(range(len(picked))), share)


def test_sums_of_shared_heads_by_more_than_2_32_threads():
    """Three tensors of gradients, each the sum over two heads: 2734 x 2048 x 3 workgroups of 256.  Two pairs against the
    reference."""
    H, D, T, share = 5488, 255, 2048, 2
    g = torch.Generator(DEV).manual_seed(3)
    q, k, v, do = (torch.randn(T, n, D, generator=g, device=DEV, dtype=BF16) for n in (H // share,) * 3 + (H,))
    rate = torch.linspace(2.0 ** -5, 1.0, H, device=DEV)
    cu = torch.tensor([0, T], dtype=torch.int32, device=DEV)
    grads = pdssm.decay_attn_bwd(q, k, v, rate, do, scale=D ** -0.5, cu=cu)
    for h in (0, H // share - 1):
        users = [2 * h, 2 * h + 1]
        want = R.bwd(*(_np(t[:, [h]]) for t in (q, k, v)), _np(rate[users]), _np(do[:, users]), D ** -0.5, [0, T])
        for name, t in zip(("dq", "dk", "dv"), grads):
            off = R.rows_off(_np(t[:, [h]]), want[name])
            assert (off < R.ROWS_OFF).all(), (h, name, off)
