"""Float64 reference of linear attention with a decay for each head and of the
group norm of rows, written from their formulas (numpy, row by row).  Test
infrastructure only: it shares no code with the HIP library.

Sequences are given by their bounds [S+1]; rows behind the last bound come back
as zeros.
"""
import numpy as np


def wide(x, H):
    """The rows of every state's head: head h of H reads head h // (H / heads)."""
    x = np.asarray(x, np.float64)
    return x[:, np.arange(H) // (H // x.shape[1])]


def fwd(q, k, v, rate, scale, bounds, h0=None, absolute=False):
    """(o [T,H,Dv], h_final [S,H,Dk,Dv]); absolute: of the magnitudes, the size of the terms that an entry is the sum of."""
    H = len(rate)
    q, k, v = wide(q, H), wide(k, H), wide(v, H)
    S, T, Dk, Dv = len(bounds) - 1, q.shape[0], q.shape[2], v.shape[2]
    fin = np.zeros((S, H, Dk, Dv)) if h0 is None else np.array(h0, np.float64)
    if absolute:
        q, k, v, fin, scale = np.abs(q), np.abs(k), np.abs(v), np.abs(fin), abs(scale)
    a = np.exp(-np.asarray(rate, np.float64))[:, None, None]
    o = np.zeros((T, H, Dv))
    with np.errstate(invalid="ignore", over="ignore"):
        for s in range(S):
            for t in range(bounds[s], bounds[s + 1]):
                fin[s] = a * fin[s] + k[t][:, :, None] * v[t][:, None, :]
                o[t] = scale * (q[t][:, :, None] * fin[s]).sum(1)
    return o, fin


def bwd(q, k, v, rate, do, scale, bounds, h0=None, dh_final=None, absolute=False):
    """dict of dq, dk, dv (summed over the users of a shared head) and dh0."""
    H = len(rate)
    heads = [x.shape[1] for x in (q, k, v)]
    q, k, v, do = wide(q, H), wide(k, H), wide(v, H), np.asarray(do, np.float64)
    S, T, Dk, Dv = len(bounds) - 1, q.shape[0], q.shape[2], v.shape[2]
    state = np.zeros((S, H, Dk, Dv)) if h0 is None else np.array(h0, np.float64)
    after = np.zeros((S, H, Dk, Dv)) if dh_final is None else np.array(dh_final, np.float64)
    if absolute:
        q, k, v, do, state, after, scale = (np.abs(x) for x in (q, k, v, do, state, after, scale))
    a = np.exp(-np.asarray(rate, np.float64))[:, None, None]
    dq, dk, dv = np.zeros((T, H, Dk)), np.zeros((T, H, Dk)), np.zeros((T, H, Dv))
    for s in range(S):
        rows = range(bounds[s], bounds[s + 1])
        for t in rows:
            state[s] = a * state[s] + k[t][:, :, None] * v[t][:, None, :]
            dq[t] = scale * (state[s] @ do[t][:, :, None])[..., 0]
        for t in reversed(rows):
            after[s] += scale * q[t][:, :, None] * do[t][:, None, :]
            dk[t] = (after[s] @ v[t][:, :, None])[..., 0]
            dv[t] = (k[t][:, None, :] @ after[s])[:, 0]
            after[s] = a * after[s]

    def together(x, n):
        return x.reshape(T, n, H // n, -1).sum(2)

    return dict(dq=together(dq, heads[0]), dk=together(dk, heads[1]), dv=together(dv, heads[2]), dh0=after)


def to_bf16(x):
    """float64 rounded to bf16, to nearest even (numbers in the range of normal ones)."""
    x = np.asarray(x, np.float64)
    m, e = np.frexp(x)
    return np.ldexp(np.round(m * 256), e - 8)


# How far bf16 results may be off as a whole; entry by entry there is only the size of the terms, which is
# tens of times an entry where a thousand of them add up.
#
# A row output is rounded once.  That alone is off by the rms of to_bf16(want) - want.  Scores, states and weighted rows
# are sums of two or three bf16 numbers, off by 2^-16 of themselves at most and each for itself, so what they bring in
# is 2^-16 of the root of the sum of an output's terms squared: 0.4 of the rounding up to terms a hundred
# times an output.  Squares add: 1 + 0.16 + what fp32 sums bring.
ROWS_OFF = 1.1
# A state's weighted rows are sums of three bf16 numbers (2^-24 of themselves); weights are rounded to fp32 and
# so are products, and each chunk rounds a weight, a product and two sums of 32 rows by three numbers:
# 16 roundings of 2^-24 that are not independent.  Of two bf16 numbers the rows are off by 2^-16 at most and 2.5e-6 in the mean.
STATES_OFF = 16 * 2.0 ** -24


def rows_off(got, want):
    """For each head of rows [T, heads, D], the rms error in units of what one rounding to bf16 makes."""
    got, want = np.asarray(got, np.float64), np.asarray(want, np.float64)
    return np.sqrt(((got - want) ** 2).sum((0, 2)) / ((to_bf16(want) - want) ** 2).sum((0, 2)))


def states_off(got, want):
    """For each state of [S, H, Dk, Dv], the rms error relative to its rms."""
    got, want = np.asarray(got, np.float64), np.asarray(want, np.float64)
    return np.sqrt(((got - want) ** 2).sum((2, 3)) / (want ** 2).sum((2, 3)))


def _sigmoid(z):
    with np.errstate(over="ignore"):
        return 1 / (1 + np.exp(-z))


def _act(z, act):
    """(f(z), f'(z))"""
    if act == "none":
        return z, np.ones_like(z)
    p = _sigmoid(z)
    with np.errstate(invalid="ignore"):
        return np.where(z < -700, 0.0, z * p), np.where(z < -700, 0.0, p + np.where(z > 700, 0.0, z * p * (1 - p)))


def _normal(x, G, eps):
    T, C = x.shape
    g = x.reshape(T, G, C // G)
    d = g - g.mean(2, keepdims=True)
    r = 1 / np.sqrt((d * d).mean(2, keepdims=True) + eps)
    return (d * r).reshape(T, C), np.broadcast_to(r, g.shape).reshape(T, C)


def norm(x, G, weight=None, bias=None, gate=None, act="none", eps=1e-5):
    x = np.asarray(x, np.float64)
    n, _ = _normal(x, G, eps)
    u = n * (1 if weight is None else weight) + (0 if bias is None else bias)
    return _act(u, act)[0] if gate is None else u * _act(np.asarray(gate, np.float64), act)[0]


def norm_bwd(x, dy, G, weight=None, bias=None, gate=None, act="none", eps=1e-5):
    """dict of dx, dw, db, dgate and of the magnitudes that they are sums of (dx_size, dw_size, db_size)."""
    x, dy = np.asarray(x, np.float64), np.asarray(dy, np.float64)
    T, C = x.shape
    w = np.ones(C) if weight is None else np.asarray(weight, np.float64)
    b = np.zeros(C) if bias is None else np.asarray(bias, np.float64)
    n, r = _normal(x, G, eps)
    u = n * w + b
    out = {}
    if gate is None:
        du = dy * _act(u, act)[1]
    else:
        f, df = _act(np.asarray(gate, np.float64), act)
        du = dy * f
        out["dgate"] = dy * u * df

    def mean(v):
        return np.repeat(v.reshape(T, G, C // G).mean(2), C // G, axis=1)

    dn = du * w
    out["dx"] = r * (dn - mean(dn) - n * mean(dn * n))
    out["dx_size"] = r * (np.abs(dn) + mean(np.abs(dn)) + np.abs(n) * mean(np.abs(dn * n)))
    out["dw"], out["db"] = (du * n).sum(0), du.sum(0)
    out["dw_size"], out["db_size"] = np.abs(du * n).sum(0), np.abs(du).sum(0)
    out["n"], out["u"], out["r"], out["du"] = n, u, r, du
    return out
