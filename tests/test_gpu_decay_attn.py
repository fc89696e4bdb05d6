"""Linear attention with a decay for each head on the GPU against its float64
reference.

Tolerances.  An entry is a sum of terms; the reference gives the sum of their
magnitudes m.  With u = 2^-24 (half a step of fp32) an fp32 result is off by at
most (D + 64 + 2 n/32 + 32) u m: the products' sums over D entries and up to 64
rows of a chunk, a product and a sum for each of a sequence's n/32 chunks, and
some 30 roundings of weights.  With bf16 rows scores and states are rounded to
bf16 (2^-8 of themselves) at most once where a row output is made from them, and
weighted rows of a state enter as two bf16 numbers (2^-16): row outputs are off
by 2^-8 m, and 2^-8 of themselves for their own rounding; states by 2^-16 m.
"""
import math

import numpy as np
import pytest
import torch

from oracle import decay_attn as R
from paper_2605_19150_amd import pdssm

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
DEV = "cuda"
TYPES = pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["fp32", "bf16"])


def _np(t):
    return None if t is None else t.detach().double().cpu().numpy()


class Case:
    """Inputs of one call on the GPU; q, k and v are parts of one wider row tensor."""

    def __init__(self, bounds, H, Dk, Dv, dtype, heads=None, T=None, dense=False, states=True, pad=0, seed=0, rate=None, scale=None):
        g = torch.Generator().manual_seed(seed)
        self.bounds, self.H, self.dtype, self.dense = list(bounds), H, dtype, dense
        self.heads = heads or (H, H, H)
        self.Dk, self.Dv, self.S = Dk, Dv, len(bounds) - 1
        T = self.T = bounds[-1] if T is None else T
        sizes = [n * D for n, D in zip(self.heads, (Dk, Dk, Dv))]
        rows = torch.randn(T, sum(sizes) + pad, generator=g)
        rows[bounds[-1]:] = math.nan  # nothing reads them
        rows = rows.to(dtype).to(DEV)
        parts = rows[:, pad:].split(sizes, 1)
        self.q, self.k, self.v = (p.unflatten(1, (n, D)) for p, n, D in zip(parts, self.heads, (Dk, Dk, Dv)))
        self.do = torch.randn(T, H, Dv, generator=g)
        self.do[bounds[-1]:] = math.nan
        self.do = self.do.to(dtype).to(DEV)
        self.rate = (torch.exp(torch.empty(H).uniform_(math.log(2.0 ** -10), math.log(1.0), generator=g)) if rate is None
                     else torch.tensor(rate)).to(DEV)
        self.h0 = torch.randn(self.S, H, Dk, Dv, generator=g).to(DEV) if states else None
        self.dhf = torch.randn(self.S, H, Dk, Dv, generator=g).to(DEV) if states else None
        self.cu = None if dense else torch.tensor(bounds, dtype=torch.int32, device=DEV)
        self.scale = Dk ** -0.5 if scale is None else scale
        self.longest = max(b - a for a, b in zip(bounds, bounds[1:]))

    def rows(self, t):
        return t.unflatten(0, (self.S, self.T // self.S)) if self.dense else t

    def fwd(self, **kw):
        return pdssm.decay_attn_fwd(self.rows(self.q), self.rows(self.k), self.rows(self.v), self.rate, scale=self.scale,
                                    cu=self.cu, h0=self.h0, **kw)

    def bwd(self, **kw):
        return pdssm.decay_attn_bwd(self.rows(self.q), self.rows(self.k), self.rows(self.v), self.rate, self.rows(self.do),
                                    scale=self.scale, cu=self.cu, h0=self.h0, dh_final=self.dhf, **kw)

    def _used(self, t):
        return _np(t[:self.bounds[-1]])

    def check_fwd(self, o, fin):
        args = [self._used(t) for t in (self.q, self.k, self.v)] + [_np(self.rate), self.scale, self.bounds, _np(self.h0)]
        want, wfin = R.fwd(*args)
        size, fsize = R.fwd(*args, absolute=True)
        self.near("o", o, want, size, self.Dk)
        near("h_final", _np(fin), wfin, fsize * self.state_units())

    def check_bwd(self, got):
        args = [self._used(t) for t in (self.q, self.k, self.v)] + [_np(self.rate), self._used(self.do), self.scale, self.bounds,
                                                                    _np(self.h0), _np(self.dhf)]
        want, size = R.bwd(*args), R.bwd(*args, absolute=True)
        for name, t in zip(("dq", "dk", "dv"), got):
            self.near(name, t, want[name], size[name], max(self.Dk, self.Dv) + self.H)
        near("dh0", _np(got[3]), want["dh0"], size["dh0"] * self.state_units())

    def units(self, D):
        return (D + 96 + 2 * (self.longest // 32)) * U

    def state_units(self):
        return self.units(0) + (2.0 ** -16 if self.dtype == torch.bfloat16 else 0)

    def near(self, name, got, want, size, D):
        got = _np(got).reshape(self.T, *want.shape[1:])
        assert not got[self.bounds[-1]:].any(), name + " behind the last sequence"
        tol = self.units(D) * size
        if self.dtype == torch.bfloat16:
            tol = tol + 2.0 ** -8 * size + 2.0 ** -8 * np.abs(want)
        near(name, got[:self.bounds[-1]], want, tol)


def near(name, got, want, tol):
    bad = ~(np.abs(got - want) <= tol + 1e-30)
    assert not bad.any(), "%s: %d of %d, worst %.3g of its tolerance" % (name, bad.sum(), bad.size,
                                                                        np.nanmax(np.abs(got - want) / (tol + 1e-30)))


BOUNDS = {"one": [0, 1], "chunk": [0, 64], "chunk+1": [0, 65], "ones": list(range(9)),
          "empty": [0, 0, 31, 32, 32, 97, 97, 225, 230], "edges": [0, 63, 127, 255, 384], "long": [0, 5, 700]}


@TYPES
@pytest.mark.parametrize("which", sorted(BOUNDS))
@pytest.mark.parametrize("D", [(1, 1), (7, 130), (64, 64), (72, 37), (128, 128), (129, 16), (256, 256)], ids=str)
def test_packed_sequences(which, D, dtype):
    b = BOUNDS[which]
    c = Case(b, 2, *D, dtype, T=b[-1] + 3, states=D[0] != 7, seed=len(b) + D[0])
    c.check_fwd(*c.fwd())
    c.check_bwd(c.bwd())


@TYPES
@pytest.mark.parametrize("pad", [0, 1, 2])
@pytest.mark.parametrize("D", [(256, 16), (16, 256), (256, 64), (200, 48), (255, 33), (136, 8), (128, 48), (96, 20)], ids=str)
def test_long_rows_of_few_columns(D, pad, dtype):
    """Products whose results are read at once: every entry of a row counts."""
    c = Case([0, 14, 28, 60, 190, 400], 2, *D, dtype, pad=pad, seed=D[0])
    c.check_fwd(*c.fwd())
    c.check_bwd(c.bwd())


@TYPES
@pytest.mark.parametrize("B,L", [(1, 1), (3, 64), (2, 201)])
@pytest.mark.parametrize("heads", [(4, 4, 4), (4, 2, 2), (1, 1, 4), (2, 4, 1)], ids=str)
def test_dense_batches_and_shared_heads(B, L, heads, dtype):
    c = Case(list(range(0, B * L + 1, L)), 4, 32, 48, dtype, heads=heads, dense=True, seed=B + L)
    o, fin = c.fwd()
    assert o.shape == (B, L, 4, 48) and fin.shape == (B, 4, 32, 48)
    c.check_fwd(o, fin)
    got = c.bwd()
    assert [t.shape for t in got[:3]] == [(B, L, heads[0], 32), (B, L, heads[1], 32), (B, L, heads[2], 48)]
    c.check_bwd(got)


@TYPES
def test_shared_heads_behind_the_last_sequence(dtype):
    c = Case([0, 40, 70], 4, 16, 16, dtype, heads=(2, 1, 4), T=83)
    c.check_bwd(c.bwd())


@TYPES
def test_shared_heads_of_odd_sizes(dtype):
    c = Case([0, 3, 90], 6, 7, 9, dtype, heads=(6, 2, 3))
    c.check_fwd(*c.fwd())
    c.check_bwd(c.bwd())


@TYPES
@pytest.mark.parametrize("H,D,share", [(300, (24, 40), 1), (300, (64, 64), 4), (140, (128, 128), 1), (140, (96, 72), 2),
                                       (130, (200, 72), 1), (130, (72, 256), 1)], ids=str)
def test_many_heads(H, D, share, dtype):
    """Calls that fill the card (bf16: scores and states rounded once); three heads of them against the reference."""
    bounds = [0, 70, 201]
    c = Case(bounds, H, *D, dtype, heads=(H, H // share, H // share), seed=H)
    (o, fin), grads = c.fwd(), c.bwd()
    picked = [0, H // 2 // share * share, H - share]
    users = [h + k for h in picked for k in range(share)]
    part = Case(bounds, len(users), *D, dtype, heads=(len(users), len(picked), len(picked)), states=False)
    of = lambda t, heads: t[:, torch.tensor(heads, device=DEV)]  # noqa: E731
    shared = [h // share for h in picked]
    part.q, part.k, part.v, part.do = of(c.q, users), of(c.k, shared), of(c.v, shared), of(c.do, users)
    part.rate, part.h0, part.dhf = c.rate[users], of(c.h0, users), of(c.dhf, users)
    part.check_fwd(of(o, users), of(fin, users))
    part.check_bwd((of(grads[0], users), of(grads[1], shared), of(grads[2], shared), of(grads[3], users)))


def test_rows_of_eight_million_entries():
    """Very many heads: the fp32 rows of a chunk, from which shared heads' gradients are summed, take 2^31 bytes and
    more.  Six heads against the reference."""
    H, D, T, share = 40000, 216, 64, 2
    g = torch.Generator(DEV).manual_seed(4)
    q, k, v, do = (torch.randn(T, n, D, generator=g, device=DEV, dtype=torch.bfloat16) for n in (H, H // share, H // share, H))
    rate = torch.linspace(2.0 ** -8, 1.0, H, device=DEV)
    cu = torch.tensor([0, T], dtype=torch.int32, device=DEV)
    o, fin = pdssm.decay_attn_fwd(q, k, v, rate, scale=D ** -0.5, cu=cu)
    grads = pdssm.decay_attn_bwd(q, k, v, rate, do, scale=D ** -0.5, cu=cu)
    picked = [0, H // 2, H - share]
    users, shared = [h + i for h in picked for i in range(share)], [h // share for h in picked]
    part = Case([0, T], len(users), D, D, torch.bfloat16, heads=(len(users), len(shared), len(shared)), states=False)
    part.q, part.k, part.v, part.do, part.rate = q[:, users], k[:, shared], v[:, shared], do[:, users], rate[users]
    part.check_fwd(o[:, users], fin[:, users])
    part.check_bwd((grads[0][:, users], grads[1][:, shared], grads[2][:, shared], grads[3][:, users]))


def test_outputs_that_go_past_the_caches():
    """64 MB and more of bf16 rows; two heads of them against the reference."""
    L, S, H = 2048, 16, 17
    c = Case(list(range(0, S * L + 1, L)), H, 64, 64, torch.bfloat16, dense=True, seed=6)
    (o, fin), grads = c.fwd(), c.bwd()
    picked = [3, 16]
    part = Case([0, L, 2 * L], 2, 64, 64, torch.bfloat16, dense=True, states=False)
    of = lambda t: t.reshape(S * L, H, -1)[2 * L:4 * L, picked]  # noqa: E731
    part.q, part.k, part.v, part.do = (of(t) for t in (c.q, c.k, c.v, c.do))
    part.rate, part.h0, part.dhf = c.rate[picked], c.h0[2:4, picked], c.dhf[2:4, picked]
    part.check_fwd(of(o), fin[2:4, picked])
    part.check_bwd((*(of(t) for t in grads[:3]), grads[3][2:4, picked]))


@TYPES
def test_many_sequences(dtype):
    """More sequences than a workgroup has threads: most of them short or empty, one long."""
    g = np.random.default_rng(2)
    n = np.where(g.random(1500) < 0.5, 0, g.integers(0, 6, 1500))
    n[700] = 900
    bounds = [0, *np.cumsum(n).tolist()]
    c = Case(bounds, 1, 8, 8, dtype, T=bounds[-1] + 2)
    c.check_fwd(*c.fwd())
    c.check_bwd(c.bwd())


@TYPES
@pytest.mark.parametrize("pad", [0, 1, 8])
@pytest.mark.parametrize("dense", [False, True])
def test_sequences_in_segments(dense, pad, dtype):
    """Few heads and long sequences are cut; rows at odd addresses, too."""
    b = [0, 1500, 3000] if dense else [0, 1, 2600, 2600, 3000]
    c = Case(b, 1, 40, 64, dtype, dense=dense, pad=pad, rate=[1e-3], seed=pad)
    c.check_fwd(*c.fwd())
    c.check_bwd(c.bwd())


@TYPES
def test_rates_from_none_to_the_largest(dtype):
    rate = [0.0, 1e-38, 1e-4, 0.5, 20.0, 200.0, 3e38]
    c = Case([0, 130, 400], len(rate), 24, 24, dtype, rate=rate)
    c.check_fwd(*c.fwd())
    c.check_bwd(c.bwd())


@TYPES
@pytest.mark.parametrize("bad", [-1e-3, math.inf, math.nan])
def test_a_bad_rate_gives_nan_in_its_head_alone(bad, dtype):
    b = [0, 70, 70, 1400]
    good, c = (Case(b, 2, 32, 32, dtype, rate=[0.1, r]) for r in (0.1, bad))
    for x, y in zip((*good.fwd(), *good.bwd()), (*c.fwd(), *c.bwd())):
        head = 1 if x.dim() in (3, 4) else None
        assert torch.equal(x.select(head, 0), y.select(head, 0))
        other = y.select(head, 1)
        if x.dim() == 4:  # a sequence without rows hands its state on
            assert torch.equal(other[1], x.select(head, 1)[1])
            other = other[[0, 2]]
        assert other.isnan().all()


@TYPES
@pytest.mark.parametrize("value", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("which", ["q", "k", "v"])
def test_no_row_depends_on_a_later_one(which, value, dtype):
    """Rows before an infinity or a NaN are what they are without it, those of other heads and sequences too,
    and what is not finite is so where the formula's result is not."""
    b = [0, 60, 200, 330]
    plain, c = (Case(b, 2, 24, 40, dtype, seed=3) for _ in range(2))
    getattr(c, which)[150, 0, 1] = value
    (o, fin), (p, pfin) = plain.fwd(), c.fwd()
    args = [_np(t) for t in (c.q, c.k, c.v)]
    want, wfin = R.fwd(*args, _np(c.rate), c.scale, b, _np(c.h0))
    ok, fok = np.isfinite(want), np.isfinite(wfin)
    assert np.array_equal(np.isfinite(_np(p)), ok) and np.array_equal(np.isfinite(_np(pfin)), fok)
    assert torch.equal(o[:124], p[:124]) and torch.equal(o[200:], p[200:])  # the chunks before it, the next sequence
    assert torch.equal(o[:, 1], p[:, 1]) and torch.equal(fin[:, 1], pfin[:, 1])
    size, fsize = R.fwd(*[np.nan_to_num(t, posinf=0, neginf=0) for t in args], _np(c.rate), c.scale, b, _np(c.h0), absolute=True)
    tol = c.units(c.Dk) * size + (2.0 ** -8 * (size + np.abs(want)) if dtype == torch.bfloat16 else 0)
    near("o", _np(p)[ok], want[ok], tol[ok])
    near("h_final", _np(pfin)[fok], wfin[fok], (c.state_units() * fsize)[fok])


@TYPES
def test_no_gradient_depends_on_an_earlier_row(dtype):
    """A NaN in q reaches dk and dv of its row and those before it, and dq of none; one in k reaches dq from its row on."""
    b = [0, 200]
    plain, c, d = (Case(b, 1, 32, 32, dtype, seed=4) for _ in range(3))
    c.q[100, 0, 3] = math.nan
    d.k[100, 0, 3] = math.nan
    x, y, z = plain.bwd(), c.bwd(), d.bwd()
    assert torch.equal(x[0], y[0]) and torch.equal(x[1], z[1])
    assert y[1][:101, 0, 3].isnan().all() and y[1][:, 0, :3].isfinite().all() and y[2][:101].isnan().all()
    assert z[0][100:, 0, 3].isnan().all() and z[0][:, 0, :3].isfinite().all() and z[2][100].isnan().all()
    args = [_np(t) for t in (plain.q, plain.k, plain.v, plain.rate, plain.do)]
    kw = dict(scale=plain.scale, bounds=b, h0=_np(plain.h0), dh_final=_np(plain.dhf))
    want, size = R.bwd(*args, **kw), R.bwd(*args, **kw, absolute=True)
    for name, got, rows in (("dk", y[1], slice(101, None)), ("dv", y[2], slice(101, None)), ("dq", z[0], slice(0, 100)),
                            ("dv", z[2], slice(0, 100)), ("dv", z[2], slice(101, None))):
        w, m = want[name][rows], size[name][rows]
        near(name, _np(got)[rows], w, plain.units(33) * m + (2.0 ** -8 * (m + np.abs(w)) if dtype == torch.bfloat16 else 0))


@TYPES
def test_states_that_are_not_finite(dtype):
    c = Case([0, 100, 150], 2, 16, 16, dtype)
    c.h0[0, 0, 3, 5] = math.inf
    o, fin = c.fwd()
    want, wfin = R.fwd(_np(c.q), _np(c.k), _np(c.v), _np(c.rate), c.scale, c.bounds, _np(c.h0))
    assert np.array_equal(np.isfinite(_np(o)), np.isfinite(want)) and np.array_equal(np.isfinite(_np(fin)), np.isfinite(wfin))


@TYPES
def test_strides(dtype):
    """Head-major rows, rows that are alike (stride 0) and rows that stand apart."""
    g = torch.Generator().manual_seed(5)
    L, H, D = 150, 3, 32
    base = Case([0, L], H, D, D, dtype, dense=True, states=False)
    q = torch.randn(1, H, L, D, generator=g).to(dtype).to(DEV).transpose(1, 2)
    k = torch.randn(1, L, 1, D, generator=g).to(dtype).to(DEV).expand(1, L, H, D)
    v = torch.randn(1, L, H, 3, D, generator=g).to(dtype).to(DEV)[:, :, :, 1]
    got = pdssm.decay_attn_fwd(q, k, v, base.rate)
    want = pdssm.decay_attn_fwd(q.contiguous(), k.contiguous(), v.contiguous(), base.rate)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    do = torch.randn(1, H, L, D, generator=g).to(dtype).to(DEV).transpose(1, 2)
    got = pdssm.decay_attn_bwd(q, k, v, base.rate, do)
    want = pdssm.decay_attn_bwd(q.contiguous(), k.contiguous(), v.contiguous(), base.rate, do.contiguous())
    assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("T,L", [(0, 0), (0, None)])
def test_calls_without_rows(T, L):
    h = torch.randn(3, 2, 8, 16, device=DEV)
    rate = torch.full((2,), 0.1, device=DEV)
    cu = torch.zeros(4, dtype=torch.int32, device=DEV) if L is None else None
    lead = (0,) if L is None else (3, 0)
    q, v = torch.zeros(*lead, 2, 8, device=DEV), torch.zeros(*lead, 2, 16, device=DEV)
    for state, want in ((h, h), (None, torch.zeros_like(h))):
        o, fin = pdssm.decay_attn_fwd(q, q, v, rate, cu=cu, h0=state)
        assert o.shape == v.shape and torch.equal(fin, want)
        assert torch.equal(pdssm.decay_attn_bwd(q, q, v, rate, v, cu=cu, dh_final=state)[3], want)


@pytest.mark.parametrize("cu", [[1, 5, 9], [0, 7, 3], [0, 5, 11], [0, -4, 9]], ids=str)
def test_a_bad_cu_is_reported(cu):
    q = torch.randn(10, 2, 16, device=DEV)
    rate = torch.full((2,), 0.1, device=DEV)
    cu = torch.tensor(cu, dtype=torch.int32, device=DEV)
    for f in (lambda: pdssm.decay_attn_fwd(q, q, q, rate, cu=cu), lambda: pdssm.decay_attn_bwd(q, q, q, rate, q, cu=cu)):
        with pytest.raises(pdssm.PdssmError) as e:
            f()
        assert e.value.status == pdssm.ERR_INDEX


@TYPES
@pytest.mark.parametrize("D", [(1, 1), (37, 72), (64, 64), (128, 130), (256, 256)], ids=str)
@pytest.mark.parametrize("heads", [(4, 4, 4), (4, 2, 2), (2, 1, 4)], ids=str)
def test_one_token(heads, D, dtype):
    B, pool, H = 5, 9, 4
    c = Case([0, B], H, *D, dtype, heads=heads, states=False, pad=1)
    h = torch.randn(pool, H, *D, device=DEV)
    slots = torch.tensor([7, -1, 0, 8, 3], dtype=torch.int32, device=DEV)
    o = torch.full((B, H, D[1]), 9.0, device=DEV).to(dtype)
    out = torch.full_like(h, 5.0)
    new, o2 = pdssm.decay_attn_step(c.q, c.k, c.v, c.rate, h, scale=0.3, slots=slots, out=out, o=o)
    assert new is out and o2 is o
    want_h, want_o = np.full(h.shape, 5.0), np.full(o.shape, 9.0)
    size_h, size_o = np.zeros(h.shape), np.zeros(o.shape)
    for b, s in enumerate(slots.tolist()):
        if s >= 0:
            args = [_np(t[b:b + 1]) for t in (c.q, c.k, c.v)] + [_np(c.rate), 0.3, [0, 1], _np(h[s:s + 1])]
            (want_o[b],), (want_h[s],) = R.fwd(*args)
            (size_o[b],), (size_h[s],) = R.fwd(*args, absolute=True)
    near("h", _np(out), want_h, 8 * U * size_h)
    near("o", _np(o), want_o, (D[0] + 16) * U * size_o + (2.0 ** -8 * np.abs(want_o) if dtype == torch.bfloat16 else 0))
    same, o3 = pdssm.decay_attn_step(c.q, c.k, c.v, c.rate, h, scale=0.3, slots=slots)  # in place
    keep = torch.tensor([s for s in slots.tolist() if s >= 0], device=DEV)
    assert same is h and torch.equal(h[keep], out[keep]) and torch.equal(o3[[0, 2, 3, 4]], o[[0, 2, 3, 4]])


def test_one_token_bad_slots():
    q = torch.randn(4, 2, 16, device=DEV)
    rate = torch.full((2,), 0.1, device=DEV)
    for slots in ([0, 1, 3, 0], [2, 2, 1, 0]):
        h = torch.randn(3, 2, 16, 16, device=DEV)
        was, o = h.clone(), torch.full((4, 2, 16), 7.0, device=DEV)
        with pytest.raises(pdssm.PdssmError) as e:
            pdssm.decay_attn_step(q, q, q, rate, h, slots=torch.tensor(slots, dtype=torch.int32, device=DEV), o=o)
        assert e.value.status == pdssm.ERR_INDEX
        row = 2 if slots[2] == 3 else 1  # past the pool, or the second to name its state
        assert (o[row] == 7).all()
        first = {s: b for b, s in reversed(list(enumerate(slots)))}
        for s in range(3):
            if s in first:
                want = torch.exp(-rate)[:, None, None] * was[s] + q[first[s]][:, :, None] * q[first[s]][:, None, :]
                torch.testing.assert_close(h[s], want, rtol=1e-5, atol=1e-5)
            else:
                assert torch.equal(h[s], was[s])


@TYPES
def test_prompt_then_tokens_then_gradients(dtype):
    """A layer as it is used: a prompt, tokens after it, and a training pass over all of them; heads gated and normed."""
    L, more, H, D = 70, 5, 4, 32
    c = Case([0, L + more, 2 * (L + more)], H, D, D, dtype, heads=(4, 2, 2), dense=True, seed=8)
    q, k, v, do = (c.rows(t) for t in (c.q, c.k, c.v, c.do))
    whole, fin = c.fwd()
    first, state = pdssm.decay_attn_fwd(q[:1, :L], k[:1, :L], v[:1, :L], c.rate, h0=c.h0[:1])
    outs = [first]
    for t in range(L, L + more):
        state, o = pdssm.decay_attn_step(q[0, t:t + 1], k[0, t:t + 1], v[0, t:t + 1], c.rate, state)
        outs.append(o[:, None])
    c.check_fwd(torch.stack([torch.cat(outs, 1)[0], whole[1]]), torch.cat([state, fin[1:]]))
    g = torch.Generator().manual_seed(1)
    rows = whole.flatten(2)
    w, b = (torch.randn(H * D, generator=g).to(DEV) for _ in range(2))
    gate, dy = (torch.randn(2, L + more, H * D, generator=g).to(dtype).to(DEV) for _ in range(2))
    y = pdssm.group_norm(rows, H, w, b, gate=gate, act="silu")
    dx, dw, db, dgate = pdssm.group_norm_bwd(rows, dy, H, w, b, gate=gate, act="silu")
    dq, dk, dv, _ = pdssm.decay_attn_bwd(q, k, v, c.rate, dx.unflatten(2, (H, D)), h0=c.h0)
    # the same layer in 64 bits, from the rows that the kernels' passes hand on
    n = (rows.shape[0] * rows.shape[1], H * D)
    want = R.norm_bwd(_np(rows).reshape(n), _np(dy).reshape(n), H, _np(w), _np(b), _np(gate).reshape(n), "silu")
    c.do = dx.reshape(c.T, H, D)
    c.dhf = None
    eps = 2.0 ** -8 if dtype == torch.bfloat16 else 0.0
    near("dx", _np(dx).reshape(n), want["dx"], eps * np.abs(want["dx"]) + 200 * U * want["dx_size"])
    near("dw", _np(dw), want["dw"], 400 * U * want["dw_size"])
    assert y.shape == rows.shape and dgate.shape == rows.shape and db.shape == b.shape
    args = [_np(t) for t in (c.q, c.k, c.v, c.rate, c.do)]
    kw = dict(scale=c.scale, bounds=c.bounds, h0=_np(c.h0))
    want, size = R.bwd(*args, **kw), R.bwd(*args, **kw, absolute=True)
    for name, t in (("dq", dq), ("dk", dk), ("dv", dv)):
        c.near(name, t.flatten(0, 1), want[name], size[name], D + H)


def test_the_same_call_twice_gives_the_same_bits():
    c = Case([0, 1000, 1003, 2900], 3, 96, 80, torch.bfloat16, heads=(3, 1, 1))
    a, b = (*c.fwd(), *c.bwd()), (*c.fwd(), *c.bwd())
    assert all(torch.equal(x, y) for x, y in zip(a, b))


def test_rows_past_32_bits():
    """Offsets of rows and heads beyond 2^32 bytes and 2^31 entries."""
    T, ld = 300, 1 << 23
    buf = torch.zeros(T * ld, dtype=torch.bfloat16, device=DEV)
    c = Case([0, 100, T], 2, 32, 32, torch.bfloat16, seed=2)
    q, k, v = (torch.as_strided(buf, (T, 2, 32), (ld, 4096, 1), i * 64) for i in range(3))
    for t, s in ((q, c.q), (k, c.k), (v, c.v)):
        t.copy_(s)
    got = pdssm.decay_attn_fwd(q, k, v, c.rate, cu=c.cu, h0=c.h0)
    want = c.fwd()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_large_pool_past_32_bits():
    pool, H, D = 1100, 32, 256  # 2^31 entries and more of states
    h = torch.zeros(pool, H, D, D, device=DEV)
    q = torch.randn(2, H, D, device=DEV)
    h[-1] = 1.0
    rate = torch.zeros(H, device=DEV)
    _, o = pdssm.decay_attn_step(q, q, q, rate, h, slots=torch.tensor([pool - 1, 0], dtype=torch.int32, device=DEV))
    want = 1 + q[0][:, :, None].double() * q[0][:, None, :].double()
    # one product and one sum
    torch.testing.assert_close(h[-1].double(), want, rtol=2 * U, atol=U)
    assert torch.isfinite(o).all() and not h[1:-1].any()


def test_another_stream():
    c = Case([0, 500, 1400], 2, 64, 64, torch.bfloat16)
    want = (*c.fwd(), *c.bwd())
    s = torch.cuda.Stream()
    got = (*c.fwd(stream=s), *c.bwd(stream=s))
    torch.cuda.current_stream().wait_stream(s)
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_graphs_side_by_side():
    """Two captured sets of calls, replayed with new inputs and eager work in between."""
    cases = [Case([0, 700, 1500], 2, 64, 48, torch.bfloat16, heads=(2, 1, 1), seed=s) for s in range(2)]
    graphs, outs, streams = [], [], [torch.cuda.Stream() for _ in cases]
    for c, s in zip(cases, streams):
        with torch.cuda.stream(s):
            c.fwd(check=False), c.bwd(check=False)
        s.synchronize()
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            outs.append((*c.fwd(check=False), *c.bwd(check=False)))
    for k in range(3):
        for c in cases:
            c.v.copy_(torch.randn(c.v.shape, device=DEV))
            c.do.copy_(torch.randn(c.do.shape, device=DEV))
        torch.cuda.synchronize()
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
        torch.cuda.synchronize()
        for c, got in zip(cases, outs):
            want = (*c.fwd(), *c.bwd())
            assert all(torch.equal(a, b) for a, b in zip(got, want)), k
