"""What the bounds on bf16 attention results see (no GPU): the chunked form in
64 bits with its operands held in one, two or three bf16 numbers, and with
mistakes in it, against the recurrence."""
import numpy as np
import pytest

from oracle import decay_attn as R

CHUNK = 64


def _terms(x, n):
    """x as the sum of n bf16 numbers, or as it is."""
    if n is None:
        return x
    y = np.zeros_like(x)
    for _ in range(n):
        y = y + R.to_bf16(x - y)
    return y


def _chunked(q, k, v, rate, scale, state=2, score=2, row=3, wrong=1.0, drop=False):
    """One sequence of one head each: (o, final state) by chunks.  wrong: a factor on the rate; drop: the first row of
    each chunk does not reach the state."""
    T, H, Dk = q.shape
    o, fin = np.zeros((T, H, v.shape[2])), np.zeros((1, H, Dk, v.shape[2]))
    for h in range(H):
        r = rate[h] * wrong
        S = fin[0, h]
        for b in range(0, T, CHUNK):
            Q, K, V = (x[b:b + CHUNK, h] for x in (q, k, v))
            n = len(Q)
            i = np.arange(n)
            near = np.where(i[:, None] >= i, np.exp(-r * np.abs(i[:, None] - i)), 0.0)
            o[b:b + n, h] = scale * (_terms((Q @ K.T) * near, score) @ V + np.exp(-r * (i + 1))[:, None] * (Q @ _terms(S, state)))
            left = np.exp(-r * (n - 1 - i))
            left[0] = 0.0 if drop else left[0]
            S = np.exp(-r * n) * S + K.T @ _terms(left[:, None] * V, row)
        fin[0, h] = S
    return o, fin


def _case(T=700, H=3, Dk=64, Dv=64, centre=0.0, seed=0):
    g = np.random.default_rng(seed)
    q, k, v = (R.to_bf16(g.standard_normal((T, H, D))) for D in (Dk, Dk, Dv))
    k = R.to_bf16(k + centre * g.standard_normal((1, H, Dk)))
    q = R.to_bf16(q - q.mean(2, keepdims=True))
    rate = np.exp(-np.linspace(2, 7, H) * np.log(2.0))
    return (q, k, v, rate, Dk ** -0.5), R.fwd(q, k, v, rate, Dk ** -0.5, [0, T])


def _off(got, want):
    return R.rows_off(R.to_bf16(got[0]), want[0]), R.states_off(got[1], want[1])


@pytest.mark.parametrize("T,D", [(70, (64, 64)), (384, (128, 128)), (700, (64, 64)), (1500, (40, 64))], ids=str)
def test_the_chunked_form_is_within_the_bounds(T, D):
    args, want = _case(T, 3, *D)
    rows, states = _off(_chunked(*args), want)
    assert (rows < R.ROWS_OFF).all() and (states < R.STATES_OFF).all()


@pytest.mark.parametrize("change", [dict(state=1), dict(score=1), dict(state=1, score=1), dict(wrong=1.05), dict(wrong=1.01),
                                    dict(drop=True)], ids=str)
@pytest.mark.parametrize("T,D", [(384, (128, 128)), (700, (64, 64)), (1500, (40, 64))], ids=str)
def test_rows_out_of_the_bound(T, D, change):
    """A mistake shows in one of the heads at least: in short memories the scores count, in long ones the states."""
    args, want = _case(T, 3, *D)
    rows, _ = _off(_chunked(*args, **change), want)
    assert rows.max() > R.ROWS_OFF


@pytest.mark.parametrize("change", [dict(row=2), dict(row=1), dict(wrong=1.01), dict(drop=True)], ids=str)
@pytest.mark.parametrize("T,D", [(70, (64, 64)), (384, (128, 128)), (1500, (40, 64))], ids=str)
def test_states_out_of_the_bound(T, D, change):
    args, want = _case(T, 3, *D)
    _, states = _off(_chunked(*args, **change), want)
    assert states.max() > R.STATES_OFF


@pytest.mark.parametrize("centre", [1.0, 4.0, 10.0])
def test_rows_that_cancel(centre):
    """Keys off centre and queries without a constant part, as a norm's gradient is: terms much larger than their sum."""
    args, want = _case(1024, 3, 128, 128, centre=0.0)
    q, k, v, rate, scale = args
    k = R.to_bf16(k + centre)
    args, want = (q, k, v, rate, scale), R.fwd(q, k, v, rate, scale, [0, 1024])
    rows, _ = _off(_chunked(*args), want)
    assert (rows < R.ROWS_OFF).all()
    rows, _ = _off(_chunked(*args, state=1), want)
    assert rows.max() > (1.3 if centre == 1 else 3.0)
