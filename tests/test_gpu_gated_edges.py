"""Edges of the gated recurrent operators on the GPU: rates that no recurrence
has, infinite gates, rows behind the last sequence, very many sequences, and
weight gradients whose sums are exact."""
import math

import numpy as np
import pytest
import torch

from oracle import gated as G
from paper_2605_19150_amd import pdssm
from test_gpu_gated import DEV, Case, _all_ops, _check_bwd, _check_fwd, _near, _np

pytestmark = pytest.mark.gpu


def _dirty(*shapes):
    """Leaves memory of these sizes behind that holds NaN in every type."""
    keep = [torch.full((n,), 0xff, dtype=torch.uint8, device=DEV) for n in shapes for _ in range(4)]
    del keep


# ---- rates -----------------------------------------------------------------

BAD_RATES = [0.0, -0.0, -1.0, -1e-30, -3e38, math.inf, -math.inf, math.nan]


@pytest.mark.parametrize("dtype,C", [(torch.float32, 65), (torch.bfloat16, 65), (torch.bfloat16, 66)])
@pytest.mark.parametrize("bounds", [[0, 100], [0, 90, 400, 700]], ids=["one chunk", "chunks"])
def test_rates_that_are_not_positive_and_finite(bounds, dtype, C):
    """NaN in the rows of those channels, held ones among them, and in nothing else."""
    case = Case(bounds, C, dtype=dtype, wide=C % 2 == 1, seed=C)
    case.ga[5], case.ga[50] = -math.inf, -100.0
    good = case.rate
    y0, f0, s0, k0 = case.fwd(hold8=True)
    g0 = case.bwd(s0), case.bwd(s0, k0)
    case.rate = good.clone()
    bad = list(range(0, C, 8))
    for n, c in enumerate(bad):
        case.rate[c] = BAD_RATES[n % len(BAD_RATES)]
    rest = [c for c in range(C) if c not in bad]
    y, fin, saved, kept = case.fwd(hold8=True)
    for v, v0 in ((y, y0), (fin, f0)):
        assert torch.isnan(v[:, bad]).all() and torch.equal(v[:, rest], v0[:, rest])
    for a, b in zip(kept, k0):  # the form of the inputs knows no rate
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    for got, want in zip((case.bwd(saved), case.bwd(saved, kept)), g0):
        for v, v0 in zip(got, want):
            assert torch.isnan(v[..., bad]).all() and torch.equal(v[..., rest], v0[..., rest])
    h = torch.randn(case.T, C, device=DEV)
    h0 = h.clone()
    _, ys = pdssm.gated_step(case.x, case.ga, case.gi, case.rate, h)
    _, y1 = pdssm.gated_step(case.x, case.ga, case.gi, good, h0)
    for v, v0 in ((h, h0), (ys, y1)):
        assert torch.isnan(v[:, bad]).all() and torch.equal(v[:, rest], v0[:, rest])


def test_bad_rates_without_rows():
    """drate says so where no row does: in chunks of a call whose sequences are all empty, and in a call without rows."""
    rate = torch.tensor([0.5, 0.0, -1.0, math.inf, math.nan], device=DEV)
    for T in (0, 100, 300):
        z, cu = torch.randn(T, 5, device=DEV), torch.zeros(3, dtype=torch.int32, device=DEV)
        h0 = torch.randn(2, 5, device=DEV)
        _, fin, saved = pdssm.gated_fwd(z, z, z, rate, cu=cu, h0=h0)
        got = pdssm.gated_bwd(z, z, z, rate, saved, z, cu=cu, h0=h0, dh_final=h0)
        assert torch.equal(fin, h0) and torch.equal(got[4], h0)
        assert got[3][0] == 0 and torch.isnan(got[3][1:]).all()


# ---- rows behind the last sequence -----------------------------------------

@pytest.mark.parametrize("dtype,C", [(torch.float32, 33), (torch.bfloat16, 65), (torch.bfloat16, 66), (torch.float32, 64)])
@pytest.mark.parametrize("bounds,T", [([0, 40, 130], 300), ([0, 128], 129), ([0, 5], 6), ([0, 96, 96], 256), ([0, 0], 40),
                                      ([0, 0, 0], 300), ([0, 31], 500)])
def test_rows_behind_the_last_sequence_are_zero(bounds, T, dtype, C):
    """The binding's outputs there, whatever the inputs and the memory held."""
    case = Case(bounds, C, T=T, dtype=dtype, wide=C % 2 == 1, seed=T)
    end, first = bounds[-1], -(-bounds[-1] // 32)
    for t in (case.x, case.ga, case.gi, case.dy):
        t[end:] = math.nan
    n = T * C
    _dirty(n, 2 * n, 4 * n, 6 * n, 12 * n, -(-T // 32) * C, -(-T // 128) * C * 4)
    y, fin, saved, kept = case.fwd(hold8=True)
    assert (y[end:] == 0).all() and (saved[-(-end // 128):] == 0).all()
    for q, e in kept:
        assert (q[end:] == 0).all() and (e[first:] == -126).all()
        assert (pdssm.unpack8((q, e))[end:] == 0).all()
    for k in (None, kept):
        _dirty(6 * n, 12 * n)
        got = case.bwd(saved, k)
        assert all((t[end:] == 0).all() for t in got[:3])
    y, _, saved = case.fwd()
    assert (y[end:] == 0).all()
    if end:
        h, size = _check_fwd(case, y, fin)
        _check_bwd(case, case.bwd(saved), h, size)


def test_weight_gradient_of_packed_rows():
    """The gradients and the kept rows as they are returned, rows behind the last sequence included."""
    case = Case([0, 130, 130, 1000], 80, T=1500, dtype=torch.bfloat16, wide=False, seed=6)
    for t in (case.x, case.ga, case.gi, case.dy):
        t[1000:] = math.nan
    _dirty(1500 * 240 * 2, 1500 * 80)
    y, fin, saved, kept = case.fwd(hold8=True)
    _dirty(1500 * 240 * 2)
    dP = torch.cat(case.bwd(saved, kept)[:3], 1)
    p, u = _np(dP)[:1000], G.unpack8(*(t.cpu().numpy() for t in kept[0]))[:1000]
    # 1500 products, a rounding each; the last 500 are zero
    _near("dW", _np(pdssm.project_wgrad(dP, kept[0])), p.T @ u, np.abs(p).T @ np.abs(u), 1502)


def test_captured_set_with_its_weight_gradient():
    """Every output of a replayed graph, the weight gradient too."""
    case = Case([0, 130, 130, 1000], 80, T=1003, dtype=torch.bfloat16, seed=6)
    _all_ops(case)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = _all_ops(case)
    for _ in range(4):
        case.x.copy_(torch.randn_like(case.x))
        case.dy.copy_(torch.randn_like(case.dy))
        g.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in out]
        _dirty(1003 * 240 * 2, 1003 * 80)
        want = _all_ops(case)
        torch.cuda.synchronize()
        for n, (a, b) in enumerate(zip(got, want)):
            assert torch.equal(a, b), n


# ---- very many sequences ---------------------------------------------------

def test_very_many_sequences():
    """2^17 sequences, most without rows, between long ones: their states, a bound out of order among the last, and
    no more time than their share of the memory takes."""
    T, S, C = 1 << 17, 1 << 17, 64
    g = torch.Generator().manual_seed(31)
    x, ga, gi, dy = (torch.randn(T, C, generator=g).to(torch.bfloat16).to(DEV) for _ in range(4))
    rate = torch.full((C,), 0.05, device=DEV)
    cuts = sorted(np.random.default_rng(31).choice(S, 40, replace=False).tolist())  # sequences that have rows
    n = np.zeros(S, np.int64)
    n[cuts] = T // 40
    cu = torch.from_numpy(np.concatenate([[0], np.cumsum(n)]).astype(np.int32)).to(DEV)
    few = torch.tensor([0, *(T // 40 * (k + 1) for k in range(40))], dtype=torch.int32, device=DEV)
    h0, dhf = (torch.randn(S, C, generator=g).to(DEV) for _ in range(2))
    at = torch.tensor(cuts, device=DEV)
    rest = torch.ones(S, dtype=torch.bool, device=DEV)
    rest[at] = False
    few0, fewf = h0[at].contiguous(), dhf[at].contiguous()

    y, fin, saved = pdssm.gated_fwd(x, ga, gi, rate, cu=cu, h0=h0)
    y1, fin1, saved1 = pdssm.gated_fwd(x, ga, gi, rate, cu=few, h0=few0)
    end = T // 40 * 40
    assert torch.equal(y[:end], y1[:end]) and torch.equal(fin[at], fin1) and torch.equal(fin[rest], h0[rest])
    d = pdssm.gated_bwd(x, ga, gi, rate, saved, dy, cu=cu, h0=h0, dh_final=dhf)
    d1 = pdssm.gated_bwd(x, ga, gi, rate, saved1, dy, cu=few, h0=few0, dh_final=fewf)
    assert all(torch.equal(a[:end], b[:end]) for a, b in zip(d[:3], d1[:3])) and torch.equal(d[3], d1[3])
    assert torch.equal(d[4][at], d1[4]) and torch.equal(d[4][rest], dhf[rest])
    for place in (S - 1, S, S // 2 + 17):
        bad = cu.clone()
        bad[place] = T + 1
        with pytest.raises(pdssm.PdssmError, match="INDEX"):
            pdssm.gated_fwd(x, ga, gi, rate, cu=bad, h0=h0)
        with pytest.raises(pdssm.PdssmError, match="INDEX"):
            pdssm.gated_bwd(x, ga, gi, rate, saved, dy, cu=bad, h0=h0, dh_final=dhf)

    def took(f):
        best = math.inf
        for _ in range(6):
            a, b = (torch.cuda.Event(enable_timing=True) for _ in range(2))
            a.record()
            f()
            b.record()
            torch.cuda.synchronize()
            best = min(best, a.elapsed_time(b))
        return best

    def fwd(cu, h0):
        return took(lambda: pdssm.gated_fwd(x, ga, gi, rate, cu=cu, h0=h0, check=False))

    def bwd(cu, h0, dhf, saved):
        return took(lambda: pdssm.gated_bwd(x, ga, gi, rate, saved, dy, cu=cu, h0=h0, dh_final=dhf, check=False))

    # 2^17 states of 64 channels are 32 MB to read and as many to write, about as much as the rows; by one wave they took
    # a hundred times as long
    times = fwd(cu, h0), fwd(few, few0), bwd(cu, h0, dhf, saved), bwd(few, few0, fewf, saved1)
    print("forward %.3f (few sequences: %.3f), backward %.3f (%.3f) ms" % times)
    assert times[0] < 10 * times[1] and times[2] < 10 * times[3]


@pytest.mark.parametrize("T,S", [(0, 3000), (5, 1000), (128, 700), (129, 513), (3000, 20000)])
def test_more_sequences_than_rows(T, S):
    C = 70
    g = torch.Generator().manual_seed(S)
    x, ga, gi, dy = (torch.randn(T, C, generator=g).to(DEV) for _ in range(4))
    cu = torch.cat([torch.tensor([0]), torch.randint(0, T + 1, (S - 1,), generator=g).sort().values, torch.tensor([T])])
    h0, dhf = (torch.randn(S, C, generator=g).to(DEV) for _ in range(2))
    rate = torch.full((C,), 0.3, device=DEV)
    cud = cu.to(torch.int32).to(DEV)
    _, fin, saved = pdssm.gated_fwd(x, ga, gi, rate, cu=cud, h0=h0)
    got = pdssm.gated_bwd(x, ga, gi, rate, saved, dy, cu=cud, h0=h0, dh_final=dhf)
    none = (cu.diff() == 0).to(DEV)
    assert torch.equal(fin[none], h0[none]) and torch.equal(got[4][none], dhf[none])
    args = [_np(t) for t in (x, ga, gi, rate)]
    n = int(cu.diff().max())
    h, want = G.gated_fwd(*args, cu.tolist(), _np(h0))
    size, fin_size = G.gated_fwd(*args, cu.tolist(), _np(h0), absolute=True)
    _near("h_final", _np(fin), want, fin_size, 2 * n + 32)
    before = G.states_before(h, cu.tolist(), _np(h0))
    w = G.gated_bwd(*args, cu.tolist(), before, _np(dy), _np(dhf))
    m = G.gated_bwd(*args, cu.tolist(), np.abs(before), _np(dy), _np(dhf), absolute=True)
    _near("dh0", _np(got[4]), w["dh0"], m["dh0"], 4 * n + 64)
    _near("dx", _np(got[0]), w["dx"], m["dx"], 4 * n + 64)


def test_many_sequences_of_length_zero():
    z, rate, h0 = torch.empty(2500, 0, 70, device=DEV), torch.ones(70, device=DEV), torch.randn(2500, 70, device=DEV)
    _, fin, saved = pdssm.gated_fwd(z, z, z, rate, h0=h0)
    assert torch.equal(fin, h0)
    got = pdssm.gated_bwd(z, z, z, rate, saved, z, dh_final=h0)
    assert torch.equal(got[4], h0) and (got[3] == 0).all()


# ---- infinite gates --------------------------------------------------------

@pytest.mark.parametrize("dtype,C", [(torch.float32, 65), (torch.bfloat16, 65), (torch.bfloat16, 66)])
def test_infinite_gates_in_the_eight_bit_form(dtype, C):
    """A gate that is open or an input that is masked altogether has the finite gradients of the plain rows, and leaves
    its neighbours' as good as they are without it."""
    case = Case([0, 60, 300, 470], C, T=475, dtype=dtype, wide=C % 2 == 1, masked=True, seed=C)
    pick = torch.Generator().manual_seed(5)
    # rows whose values count: held ones may hold anything
    live = torch.from_numpy(_np(case.ga) > G.HOLD).to(DEV)
    for t, v, share in ((case.gi, -math.inf, 0.2), (case.gi, math.inf, 0.02), (case.ga, math.inf, 0.02)):
        at = (torch.rand(case.T, C, generator=pick) < share).to(DEV) & live
        t[at] = v
    y, fin, saved, kept = case.fwd(hold8=True)
    h, size = _check_fwd(case, y, fin)
    plain = case.bwd(saved)
    want = G.kept(*(_np(t) for t in (case.x, case.ga, case.gi)), case.end)
    blocks = -(-case.end // 32)
    for (q, e), w in zip(kept, want):
        assert np.array_equal(G.unpack8(q.cpu().numpy()[:case.end], e.cpu().numpy()[:blocks]), w[:case.end])
        assert np.array_equal(_np(pdssm.unpack8((q, e)))[:case.end], w[:case.end])
    got = case.bwd(saved, kept)
    for t in (*plain, *got):
        rows = case.end if t.shape[0] == case.T else t.shape[0]
        assert torch.isfinite(t[:rows]).all()
    # the kept value of an open gate is 31.75 or more, where the sigmoid is 1 in 32 bits as it is at infinity
    args = [w.copy() for w in want]
    for w, t in ((args[1], case.ga), (args[2], case.gi)):
        w[_np(t) == math.inf] = math.inf
    _check_bwd(case, got, h, size, kept=args)
    shut = _np(case.gi)[:case.end] == -math.inf
    shut &= _np(case.ga)[:case.end] > G.HOLD
    assert shut.sum() > 1000 and all((_np(got[k])[:case.end][shut] == 0).all() for k in (0, 2))


@pytest.mark.parametrize("dtype,C", [(torch.float32, 65), (torch.bfloat16, 65), (torch.bfloat16, 66)])
@pytest.mark.parametrize("shut", ["lowest", -1e9, -1e4, -100.0, -89.0])
def test_gates_far_out_in_the_eight_bit_form(shut, dtype, C):
    """An input masked with the type's lowest value or any other that shuts its gate, and gates wide open, do not cost
    the logits beside them their codes."""
    case = Case([0, 60, 300, 470], C, T=475, dtype=dtype, wide=C % 2 == 1, seed=C)
    clean = [_np(t) for t in (case.ga, case.gi)]
    v = torch.finfo(dtype).min if shut == "lowest" else shut
    pick = torch.Generator().manual_seed(6)
    far = []
    for t, v, share in ((case.ga, -v, 0.02), (case.gi, -v, 0.02), (case.gi, v, 0.2)):
        at = (torch.rand(case.T, C, generator=pick) < share).to(DEV)
        t[at] = v
        far.append(_np(at) > 0)
    y, fin, saved, kept = case.fwd(hold8=True)
    h, size = _check_fwd(case, y, fin)
    want = G.kept(*(_np(t) for t in (case.x, case.ga, case.gi)), case.end)
    got = []
    for (q, e), w in zip(kept, want):
        got.append(_np(pdssm.unpack8((q, e))))
        assert np.array_equal(got[-1][:case.end], w[:case.end])
    # half a step of a block that reaches 31.75, and 2^-7 of what the largest of the others is
    for v, c, out in ((got[1], clean[0], far[0]), (got[2], clean[1], far[1] | far[2])):
        ok = ~out[:case.end]
        assert np.abs(v[:case.end] - c[:case.end])[ok].max() <= 0.125
    args = [w.copy() for w in want]
    for w, out in ((args[1], far[0]), (args[2], far[1] & ~far[2])):
        w[:case.end][out[:case.end]] = math.inf  # 1 in 32 bits, as there
    _check_bwd(case, case.bwd(saved, kept), h, size, kept=args)


def test_infinite_gates_beside_a_nan():
    """A block with a NaN is marked whatever else it holds, and infinite inputs mark theirs as before."""
    case = Case([0, 200], 66, seed=11)
    case.gi[40, 3], case.gi[41, 3], case.ga[70, 5], case.ga[71, 5] = math.nan, -math.inf, math.nan, math.inf
    case.x[100, 7], case.gi[0, 9] = math.inf, -math.inf
    _, _, _, kept = case.fwd(hold8=True)
    bad = [(100, 7), (70, 5), (40, 3)]
    for (q, e), (t, c) in zip(kept, bad):
        v = _np(pdssm.unpack8((q, e)))
        block = np.zeros_like(v, bool)
        block[t // 32 * 32:t // 32 * 32 + 32, c] = True
        assert np.isnan(v[block]).all() and not np.isnan(v[~block]).any()
        assert (e[:, c].cpu().numpy() == -128).sum() == 1


# ---- weight gradient -------------------------------------------------------

@pytest.mark.parametrize("T,M,Dm", [(98401, 264, 272), (6200, 4096, 1024), (131072, 512, 512), (100, 3592, 3344),
                                    (5000, 520, 64), (20000, 64, 32), (3000, 2048, 2048), (1600, 1024, 1040), (777, 40, 48)])
def test_weight_gradient_whose_sums_are_exact(T, M, Dm):
    """Whole numbers, so that every partial sum is one below 2^24: a share of the tokens that is lost, counted twice or
    cut at the wrong row changes the result.  Both tiles, with and without shares, few and many of them."""
    g = torch.Generator(device=DEV).manual_seed(T)
    dP = torch.randint(-3, 4, (T, M), generator=g, device=DEV)
    u = torch.randint(-5, 6, (T, Dm), generator=g, device=DEV)
    u8 = pdssm.pack8(u.to(torch.bfloat16))
    assert torch.equal(pdssm.unpack8(u8), u.float()) and 15 * T < 1 << 24
    want = dP.double().t().contiguous() @ u.double()
    assert torch.equal(pdssm.project_wgrad(dP.to(torch.bfloat16), u8).double(), want)
