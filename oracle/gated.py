"""Float64 reference of the gated recurrent operators, written from their
formulas (numpy, row by row).  Test infrastructure only: it shares no code
with the HIP library.

Sequences are given by their bounds [S+1]; rows behind the last bound come
back as NaN, a mark no comparison of used rows meets.
"""
import numpy as np

HOLD, CHUNK, BLOCK = -64.0, 128, 32


def gates(x, ga, gi, rate):
    """(a, beta, r, i, x, s, held) of every row; x and i are 0 in held rows."""
    x, ga, gi = (np.asarray(v, np.float64) for v in (x, ga, gi))
    held = ga <= HOLD
    with np.errstate(over="ignore", invalid="ignore"):
        r = np.where(held, 0.0, 1 / (1 + np.exp(-ga)))
        i = np.where(held, 0.0, 1 / (1 + np.exp(-gi)))
    x = np.where(held, 0.0, x)
    s = np.asarray(rate, np.float64) * r
    return np.exp(-s), np.sqrt(-np.expm1(-2 * s)), r, i, x, s, held


def gated_fwd(x, ga, gi, rate, bounds, h0=None, absolute=False):
    """(h [T,C], h_final [S,C]); absolute: of the magnitudes |x| and |h0|, the
    size of the terms that a state is the sum of."""
    a, beta, _, i, x, _, _ = gates(x, ga, gi, rate)
    b = beta * i * x
    if absolute:
        b = np.abs(b)
    S, C = len(bounds) - 1, a.shape[1]
    fin = np.zeros((S, C)) if h0 is None else np.array(h0, np.float64)
    if absolute:
        fin = np.abs(fin)
    out = np.full(a.shape, np.nan)
    for s in range(S):
        for t in range(bounds[s], bounds[s + 1]):
            fin[s] = a[t] * fin[s] + b[t]
            out[t] = fin[s]
    return out, fin


def states_before(h, bounds, h0=None, anew=None, x=None, ga=None, gi=None, rate=None):
    """The state before every row.  anew: states of an exact run; the rows'
    own values then count only within a chunk of CHUNK rows, which begins
    from anew."""
    S, C = len(bounds) - 1, h.shape[1]
    out = np.full(h.shape, np.nan)
    if anew is not None:
        a, beta, _, i, x, _, _ = gates(x, ga, gi, rate)
    for s in range(S):
        cur = np.zeros(C) if h0 is None else np.array(h0[s], np.float64)
        for t in range(bounds[s], bounds[s + 1]):
            if anew is not None and t > bounds[s] and t % CHUNK == 0:
                cur = anew[t - 1]
            out[t] = cur
            cur = h[t] if anew is None else a[t] * cur + beta[t] * i[t] * x[t]
    return out


def gated_bwd(x, ga, gi, rate, bounds, before, dy, dh_final=None, absolute=False):
    """dict of dx, dga, dgi [T,C], drate [C], dh0 [S,C] from the states before
    every row; absolute: the sums of the magnitudes of their terms."""
    a, beta, r, i, x, s, held = gates(x, ga, gi, rate)
    if absolute:
        x, before, dy = np.abs(x), np.abs(before), np.abs(np.asarray(dy, np.float64))
    S, C = len(bounds) - 1, a.shape[1]
    g = np.full(a.shape, np.nan)
    dh0 = np.zeros((S, C)) if dh_final is None else np.array(dh_final, np.float64)
    if absolute:
        dh0 = np.abs(dh0)
    for k in range(S):
        for t in range(bounds[k + 1] - 1, bounds[k] - 1, -1):
            g[t] = np.asarray(dy[t], np.float64) + dh0[k]
            dh0[k] = a[t] * g[t]
    with np.errstate(divide="ignore", invalid="ignore"):
        w = i * x * s * a * a / beta
    w = np.where(held, 0.0, w)
    move = np.where(held, 0.0, s * a * before)
    w = g * (w + move if absolute else w - move)
    used = ~np.isnan(g)
    return dict(dx=np.where(held, 0.0, g * beta * i), dga=w * (1 - r),
                dgi=np.where(held, 0.0, g * beta * i * x * (1 - i)),
                drate=np.where(used, w, 0.0).sum(0) / np.asarray(rate, np.float64), dh0=dh0)


def pack8(u):
    """(q, e) of rows u: the smallest e >= -126 with 127 * 2^e at least the
    largest magnitude of BLOCK rows, q the nearest whole number (ties to
    even; at e = 122 at most 63, as 64 would stand for 2^128); a block with a NaN or an infinity has e = -128."""
    u = np.asarray(u, np.float64)
    T, C = u.shape
    n = -(-T // BLOCK)
    q, e = np.zeros((T, C), np.int8), np.zeros((n, C), np.int8)
    for k in range(n):
        v = u[k * BLOCK:(k + 1) * BLOCK]
        for c in range(C):
            top = np.abs(v[:, c]).max()
            if not np.isfinite(top):
                e[k, c] = -128
                continue
            p = -126
            while 127 * 2.0 ** p < top:
                p += 1
            e[k, c] = p
            q[k * BLOCK:k * BLOCK + v.shape[0], c] = np.clip(np.rint(v[:, c] / 2.0 ** p), *((-63, 63) if p == 122 else (-127, 127)))
    return q, e


def unpack8(q, e):
    scale = np.where(e == -128, np.nan, 2.0 ** np.asarray(e, np.float64))
    v = np.asarray(q, np.float64) * np.repeat(scale, BLOCK, 0)[:q.shape[0]]
    return np.where(q == -128, -np.inf, v)


OPEN, SHUT = 31.75, -89.0  # in 32 bits the sigmoid is 1 from OPEN up and 0 from SHUT down


def kept(x, ga, gi, end):
    """The values of x, ga, gi that the forward's 8-bit form stands for: rows up
    to `end`, held rows kept as 0, held, 0; logits past OPEN as the largest code
    of a block that reaches OPEN; gi from SHUT down as -inf where its code is past
    -127; rows behind as 0."""
    held = np.asarray(ga[:end], np.float64) <= HOLD
    out = []
    for k, v in enumerate((x, ga, gi)):
        v = np.where(held, 0.0, np.asarray(v[:end], np.float64))
        low = held if k == 1 else v <= SHUT if k == 2 else np.zeros_like(held)
        w = np.where(low, 0.0, v if k == 0 else np.where(v > OPEN, OPEN, v))
        q, e = pack8(w)
        step = np.repeat(2.0 ** e.astype(np.float64), BLOCK, 0)[:end]
        if k > 0:
            q = np.where(v > OPEN, np.minimum(np.rint(np.minimum(v, 1e9) / step), 127), q)
        if k == 2:
            q = np.where(low, np.maximum(np.rint(np.maximum(v, -1e9) / step), -128), q)
        w = unpack8(q, e)
        w = np.where(held, -np.inf if k == 1 else 0.0, w)
        full = np.zeros(x.shape)
        full[:end] = w
        out.append(full)
    return out
