"""The float64 reference of the gated recurrence, its gradients and the 8-bit
form, held to what they are defined by (CPU)."""
import numpy as np
import pytest
import torch

from oracle import gated as G


def _case(T=23, C=3, seed=0):
    r = np.random.default_rng(seed)
    x, ga, gi, dy = (r.normal(size=(T, C)) for _ in range(4))
    rate = np.exp(r.uniform(np.log(0.01), np.log(2.0), C))
    bounds = [0, 5, 5, 6, T - 2]
    h0, dhf = r.normal(size=(4, C)), r.normal(size=(4, C))
    ga[7] = -np.inf
    ga[8, 0] = -64.0
    x[7] = 3.0
    return x, ga, gi, dy, rate, bounds, h0, dhf


def _loss(x, ga, gi, rate, h0, bounds, dy, dhf):
    h, fin = G.gated_fwd(x, ga, gi, rate, bounds, h0)
    end = bounds[-1]
    return (h[:end] * dy[:end]).sum() + (fin * dhf).sum()


def test_gradients_against_differences():
    x, ga, gi, dy, rate, bounds, h0, dhf = _case()
    h, _ = G.gated_fwd(x, ga, gi, rate, bounds, h0)
    got = G.gated_bwd(x, ga, gi, rate, bounds, G.states_before(h, bounds, h0), dy, dhf)
    args = dict(x=x, ga=ga, gi=gi, rate=rate, h0=h0)
    end = bounds[-1]
    for name, key in (("x", "dx"), ("ga", "dga"), ("gi", "dgi"), ("rate", "drate"), ("h0", "dh0")):
        flat = args[name].reshape(-1)
        for k in range(flat.size):
            if name in ("x", "ga", "gi") and k // x.shape[1] >= end:
                continue
            old = flat[k]
            if not np.isfinite(old) or (name == "ga" and old <= -64):
                assert got[key].reshape(-1)[k] == 0
                continue
            eps = 1e-5 * max(1.0, abs(old))
            flat[k] = old + eps
            up = _loss(**args, bounds=bounds, dy=dy, dhf=dhf)
            flat[k] = old - eps
            down = _loss(**args, bounds=bounds, dy=dy, dhf=dhf)
            flat[k] = old
            # central differences: eps^2 of the third derivative, and the loss's own rounding over eps
            assert abs(got[key].reshape(-1)[k] - (up - down) / (2 * eps)) < 2e-7, (name, k)


def test_gradients_against_autograd():
    x, ga, gi, dy, rate, bounds, h0, dhf = _case(seed=3)
    ga[7], ga[8, 0] = -60.0, 1.0  # autograd of the unguarded formula
    t = [torch.tensor(v, requires_grad=True) for v in (x, ga, gi, rate, h0)]
    r, i = torch.sigmoid(t[1]), torch.sigmoid(t[2])
    s = t[3] * r
    a, beta = torch.exp(-s), torch.sqrt(-torch.expm1(-2 * s))
    loss = 0.0
    for k in range(4):
        h = t[4][k]
        for n in range(bounds[k], bounds[k + 1]):
            h = a[n] * h + beta[n] * i[n] * t[0][n]
            loss = loss + (h * torch.tensor(dy[n])).sum()
        loss = loss + (h * torch.tensor(dhf[k])).sum()
    want = torch.autograd.grad(loss, t)
    h, _ = G.gated_fwd(x, ga, gi, rate, bounds, h0)
    got = G.gated_bwd(x, ga, gi, rate, bounds, G.states_before(h, bounds, h0), dy, dhf)
    for key, w in zip(("dx", "dga", "dgi", "drate", "dh0"), want):
        n = bounds[-1] if key in ("dx", "dga", "dgi") else None
        np.testing.assert_allclose(got[key][:n], w.numpy()[:n], rtol=1e-11, atol=1e-13)


def test_held_rows_and_empty_sequences():
    x, ga, gi, dy, rate, bounds, h0, dhf = _case()
    x[7], gi[7] = np.nan, np.inf
    h, fin = G.gated_fwd(x, ga, gi, rate, bounds, h0)
    assert np.array_equal(h[7], h[6]) and np.isfinite(h[:bounds[-1]]).all()
    assert np.array_equal(fin[1], h0[1])
    b = G.gated_bwd(x, ga, gi, rate, bounds, G.states_before(h, bounds, h0), dy, dhf)
    assert np.array_equal(b["dh0"][1], dhf[1])
    assert (b["dx"][7] == 0).all() and (b["dga"][7] == 0).all() and (b["dgi"][7] == 0).all()


def test_constant_gates_give_powers():
    """Constant gates: h_t = a^(t+1) h0 + b (1 - a^(t+1)) / (1 - a)."""
    T, rate = 40, np.array([0.7])
    one = np.ones((T, 1))
    h, _ = G.gated_fwd(2 * one, 0.5 * one, -1.0 * one, rate, [0, T], np.array([[3.0]]))
    a = np.exp(-0.7 / (1 + np.exp(-0.5)))
    b = np.sqrt(1 - a * a) * 2 / (1 + np.exp(1.0))
    p = a ** np.arange(1, T + 1)
    np.testing.assert_allclose(h[:, 0], p * 3 + b * (1 - p) / (1 - a), rtol=1e-12)


def test_states_from_chunks_equal_the_run():
    r = np.random.default_rng(5)
    T, C = 300, 2
    x, ga, gi = (r.normal(size=(T, C)) for _ in range(3))
    bounds, h0 = [0, 120, 300], r.normal(size=(2, C))
    rate = np.array([0.02, 0.5])
    h, _ = G.gated_fwd(x, ga, gi, rate, bounds, h0)
    np.testing.assert_allclose(G.states_before(h, bounds, h0, anew=h, x=x, ga=ga, gi=gi, rate=rate),
                               G.states_before(h, bounds, h0), rtol=1e-12)


@pytest.mark.parametrize("T", [1, 31, 32, 33, 100])
def test_eight_bit_form(T):
    r = np.random.default_rng(T)
    u = r.normal(size=(T, 4)) * np.array([1.0, 1e-3, 127.0, 0.0])
    u[0, 2] = 127.0
    q, e = G.pack8(u)
    v = G.unpack8(q, e)
    step = np.repeat(2.0 ** e.astype(float), 32, 0)[:T]
    assert (np.abs(v - u) <= step / 2).all() and (np.abs(q.astype(int)) <= 127).all()
    assert (q[:, 3] == 0).all()
    top = np.stack([np.abs(u[k:k + 32]).max(0) for k in range(0, T, 32)])
    assert (127 * 2.0 ** e >= top).all() and ((127 * 2.0 ** (e - 1.0) < top) | (e == -126)).all()
    # exact in bf16, and a second pass changes nothing
    assert np.array_equal(torch.tensor(v).to(torch.bfloat16).double().numpy(), v)
    assert np.array_equal(G.unpack8(*G.pack8(v)), v)


def test_eight_bit_form_of_what_is_not_finite():
    u = np.ones((40, 3))
    u[3, 0], u[35, 1] = np.nan, -np.inf
    q, e = G.pack8(u)
    assert e[0, 0] == -128 and e[1, 1] == -128 and (e[:, 2] == -6).all() and e[1, 0] == e[0, 1] == -6
    v = G.unpack8(q, e)
    assert np.isnan(v[:32, 0]).all() and (v[32:, 0] == 1).all() and np.isnan(v[32:, 1]).all()
