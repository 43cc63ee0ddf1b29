"""Expert networks, the layer for a few tokens and gradient clipping in fp64, from
their formulas (step 4 of Algorithm 1 of the paper and its gradient).

Every value comes with a bound on how far a computation of it may be off that
forms each sum in fp32 and rounds where the header says: `u` is the unit roundoff of
fp32, `r` that of the element type (0 where the type is fp32).  A sum of n products
with magnitude M (the sum of the absolute products) is off by at most (n + 1) u M
plus what its factors are off.
"""

import numpy as np

U32 = 2.0 ** -24
U_BF16 = 2.0 ** -8  # half a step of bf16, relative to the value
RELU, GELU, SILU = 0, 1, 2
_A, _B = np.sqrt(2.0 / np.pi), 0.044715


def _sigmoid(x):
    with np.errstate(over="ignore"):
        return 1.0 / (1.0 + np.exp(-x))


def act(kind, a):
    """The activation and its derivative."""
    if kind == RELU:
        return np.maximum(a, 0.0), (a > 0).astype(np.float64)
    if kind == SILU:
        p = _sigmoid(a)
        return a * p, p + a * p * (1.0 - p)
    t = np.tanh(_A * (a + _B * a ** 3))
    f = 0.5 * a * (1.0 + t)
    return f, 0.5 * (1.0 + t) + 0.5 * a * (1.0 - t * t) * _A * (1.0 + 3.0 * _B * a * a)


def act_error(kind, a, a_err):
    """Bounds of the activation and of its derivative computed in fp32 from an `a` that is off
    by at most a_err.  |act'| <= 1.13 and |act''| <= 1 (gelu and silu); the sigmoid's
    exponential is off by its argument's rounding, 2 (|z| + 2) u, and a few units of its own."""
    if kind == RELU:
        # the derivative jumps at 0: where a may lie on either side it is off by 1
        return a_err, (np.abs(a) <= a_err).astype(np.float64) * (a_err > 0)
    z = np.abs(a) if kind == SILU else 2.0 * _A * np.abs(a + _B * a ** 3)
    p = _sigmoid(a if kind == SILU else 2.0 * _A * (a + _B * a ** 3))
    p_err = p * (1.0 - p) * (4.0 * z + 4.0) * U32 + 6.0 * U32 * p + 1e-37
    slope = 1.0 + np.abs(a) * (1.0 if kind == SILU else 2.0 * _A * (1.0 + 3.0 * _B * a * a))
    return 1.13 * a_err + np.abs(a) * p_err + 4.0 * U32 * np.abs(a) * p, \
        1.0 * a_err + 3.0 * slope * p_err + 12.0 * U32 * (p + slope * p * (1.0 - p))


def _product(a, b, a_err, b_err, n=None):
    """a @ b and its bound."""
    n = a.shape[-1] if n is None else n
    v = a @ b
    aa, bb = np.abs(a), np.abs(b)
    err = (n + 2) * U32 * (aa @ bb)
    if a_err is not None:
        err = err + a_err @ (bb if b_err is None else bb + b_err)
    if b_err is not None:
        err = err + aa @ b_err
    return v, err


def _bias(v, err, b):
    if b is None:
        return v, err
    return v + b, err + U32 * (np.abs(v) + np.abs(b) + err)


def network(x, w1, b1, w2, b2, kind, gated, r, terms=1):
    """One expert on rows x: dict of (value, bound) for pre, hidden, y; the stored ones
    (pre and hidden) include their rounding, y its own.  With two terms hidden is the sum
    of its rounding and the rounding of what that leaves, off by r^2, and the second
    product has twice the terms."""
    h = w2.shape[0]
    pre, pe = _bias(*_product(x, w1, None, None), b1)
    if gated:
        f = act(kind, pre[:, :h])[0]
        fe = act_error(kind, pre[:, :h], pe[:, :h])[0]
        u, ue = pre[:, h:], pe[:, h:]
        hid = f * u
        he = fe * np.abs(u) + (np.abs(f) + fe) * ue + U32 * np.abs(hid)
    else:
        hid = act(kind, pre)[0]
        he = act_error(kind, pre, pe)[0]
    he = he + r ** terms * (np.abs(hid) + he)
    y, ye = _bias(*_product(hid, w2, he, None, terms * h), b2)
    return dict(pre=(pre, pe + r * (np.abs(pre) + pe)), hidden=(hid, he), y=(y, ye + r * (np.abs(y) + ye)),
                y_unrounded=(y, ye))


def _rows(counts, E, C):
    return [C] * E if counts is None else [int(min(max(c, 0), C)) for c in counts]


def experts(xe, w1, b1, w2, b2, counts, kind, gated, r):
    """fp64 arrays [E, C, .]; returns dict of (value, bound) with zero rows behind counts."""
    E, C, d = xe.shape
    h, h1 = w2.shape[1], w1.shape[2]
    out = {key: (np.zeros((E, C, n)), np.zeros((E, C, n))) for key, n in (("pre", h1), ("hidden", h), ("ye", d))}
    for e, n in enumerate(_rows(counts, E, C)):
        o = network(xe[e, :n], w1[e], None if b1 is None else b1[e], w2[e], None if b2 is None else b2[e], kind, gated, r)
        for key, src in (("pre", "pre"), ("hidden", "hidden"), ("ye", "y")):
            out[key][0][e, :n], out[key][1][e, :n] = o[src]
    return out


def experts_bwd(dye, xe, w1, w2, counts, pre, hidden, kind, gated, r):
    """Gradients from given pre and hidden (exact inputs)."""
    E, C, d = dye.shape
    h, h1 = w2.shape[1], w1.shape[2]
    shapes = dict(dxe=(E, C, d), dw1=(E, d, h1), db1=(E, h1), dw2=(E, h, d), db2=(E, d))
    out = {key: (np.zeros(s), np.zeros(s)) for key, s in shapes.items()}
    for e, n in enumerate(_rows(counts, E, C)):
        dy, x, p, hid = dye[e, :n], xe[e, :n], pre[e, :n], hidden[e, :n]
        dh, dhe = _product(dy, w2[e].T, None, None)
        a = p[:, :h] if gated else p
        f, df = act(kind, a)
        fe, dfe = act_error(kind, a, np.zeros_like(a))
        if gated:
            u = p[:, h:]
            parts = [(dh * u * df, np.abs(u) * (dhe * (np.abs(df) + dfe) + np.abs(dh) * dfe) + 2 * U32 * np.abs(dh * u * df)),
                     (dh * f, dhe * (np.abs(f) + fe) + np.abs(dh) * fe + U32 * np.abs(dh * f))]
            dpre, dpe = (np.concatenate(q, axis=1) for q in zip(*parts))
        else:
            dpre, dpe = dh * df, dhe * (np.abs(df) + dfe) + np.abs(dh) * dfe + U32 * np.abs(dh * df)
        stored = dpe + r * (np.abs(dpre) + dpe)  # what the products read
        ones = np.ones((1, n))
        vals = dict(dxe=_product(dpre, w1[e].T, stored, None), dw1=_product(x.T, dpre, None, stored),
                    dw2=_product(hid.T, dy, None, None))
        for key, (v, err) in vals.items():
            err = err + r * (np.abs(v) + err)
            if key == "dxe":
                out[key][0][e, :n], out[key][1][e, :n] = v, err
            else:
                out[key][0][e], out[key][1][e] = v, err
        for key, (v, err) in (("db1", _product(ones, dpre, None, dpe)), ("db2", _product(ones, dy, None, None))):
            out[key][0][e], out[key][1][e] = v[0], err[0]
    return out


def token_layer(x, ids, weights, w1, b1, w2, b2, kind, gated, r):
    """y and its bound from given ids and weights [S, k]; an id outside [0, E) adds nothing."""
    S, d = x.shape
    E = w1.shape[0]
    y, err, mag = np.zeros((S, d)), np.zeros((S, d)), np.zeros((S, d))
    for s in range(S):
        for e, w in zip(ids[s], weights[s]):
            if 0 <= e < E:
                v, ve = network(x[s:s + 1], w1[e], None if b1 is None else b1[e], w2[e],
                                None if b2 is None else b2[e], kind, gated, r, 2 if r else 1)["y_unrounded"]
                y[s] += w * v[0]
                err[s] += abs(w) * ve[0]
                mag[s] += np.abs(w * v[0])
    err = err + (ids.shape[1] + 2) * U32 * (mag + err)
    return y, err + r * (np.abs(y) + err)
