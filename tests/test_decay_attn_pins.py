"""The float64 reference of linear attention and of the group norm (no GPU):
against sums written out, against differences and against torch's autograd."""
import numpy as np
import pytest
import torch

from oracle import decay_attn as R


def _inputs(H=4, heads=(4, 2, 1), Dk=5, Dv=3, bounds=(0, 0, 1, 6, 6, 13), extra=2, seed=0):
    g = np.random.default_rng(seed)
    T, S = bounds[-1] + extra, len(bounds) - 1
    q, k, v = (g.standard_normal((T, n, D)) for n, D in zip(heads, (Dk, Dk, Dv)))
    return dict(q=q, k=k, v=v, rate=np.array([0.0, 0.1, 0.7, 3.0])[:H], scale=0.4, bounds=bounds,
                h0=g.standard_normal((S, H, Dk, Dv))), g.standard_normal((T, H, Dv)), g.standard_normal((S, H, Dk, Dv))


def test_forward_is_the_sum_over_earlier_rows():
    c, _, _ = _inputs()
    o, fin = R.fwd(**c)
    q, k, v = (R.wide(c[n], 4) for n in "qkv")
    for s in range(5):
        b, e = c["bounds"][s], c["bounds"][s + 1]
        for h in range(4):
            a = np.exp(-c["rate"][h])
            for t in range(b, e):
                want = c["scale"] * (a ** (t - b + 1) * q[t, h] @ c["h0"][s, h] + sum(a ** (t - j) * (q[t, h] @ k[j, h]) * v[j, h]
                                                                                  for j in range(b, t + 1)))
                np.testing.assert_allclose(o[t, h], want, rtol=1e-12, atol=1e-12)
            want = a ** (e - b) * c["h0"][s, h] + sum((a ** (e - 1 - j) * np.outer(k[j, h], v[j, h]) for j in range(b, e)), np.zeros((5, 3)))
            np.testing.assert_allclose(fin[s, h], want, rtol=1e-12, atol=1e-12)
    assert not o[13:].any()


@pytest.mark.parametrize("heads", [(4, 4, 4), (4, 2, 2), (1, 1, 4), (2, 4, 1)], ids=str)
def test_gradients_against_differences(heads):
    c, do, dhf = _inputs(heads=heads)
    g = R.bwd(do=do, dh_final=dhf, **c)

    def loss(**kw):
        o, fin = R.fwd(**{**c, **kw})
        return (o * do).sum() + (fin * dhf).sum()

    rng, step = np.random.default_rng(1), 1e-5
    for name, grad in (("q", "dq"), ("k", "dk"), ("v", "dv"), ("h0", "dh0")):
        d = rng.standard_normal(c[name].shape)
        num = (loss(**{name: c[name] + step * d}) - loss(**{name: c[name] - step * d})) / (2 * step)
        # the loss is a polynomial of degree 3 at most: the difference is off by step^2 and by rounding over step
        assert abs(num - (g[grad] * d).sum()) < 1e-7 * max(1.0, abs(num))


@pytest.mark.parametrize("act", ["none", "silu"])
@pytest.mark.parametrize("gated", [False, True])
def test_norm_against_autograd(gated, act):
    g = torch.Generator().manual_seed(3)
    x, gate, dy = (torch.randn(7, 12, generator=g, dtype=torch.float64, requires_grad=k < 2) for k in range(3))
    w, b = (torch.randn(12, generator=g, dtype=torch.float64, requires_grad=True) for _ in range(2))
    u = torch.nn.functional.group_norm(x, 3, w, b, 1e-5)
    f = torch.nn.functional.silu if act == "silu" else (lambda z: z)
    y = u * f(gate) if gated else f(u)
    (y * dy.detach()).sum().backward()
    args = [t.detach().numpy() for t in (x, w, b, gate, dy)]
    kw = dict(weight=args[1], bias=args[2], gate=args[3] if gated else None, act=act)
    np.testing.assert_allclose(R.norm(args[0], 3, **kw), y.detach().numpy(), rtol=1e-10, atol=1e-12)
    got = R.norm_bwd(args[0], args[4], 3, **kw)
    for name, t in (("dx", x), ("dw", w), ("db", b)) + ((("dgate", gate),) if gated else ()):
        np.testing.assert_allclose(got[name], t.grad.numpy(), rtol=1e-9, atol=1e-11)
