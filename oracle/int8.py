"""Quantization to 8-bit integers and the expert networks on them, in fp64.

Integer sums are exact.  Hidden rows are quantized from what the networks store, whose
bound (`oracle.experts`) may span a border between two stored values or two integers:
where it does, and only there, the bound of y holds the difference.
"""

import numpy as np

from . import experts as ox
from .bf16 import bf16_to_f64, f64_to_bf16

U32 = ox.U32


def quantize(x):
    """Rows (last axis) of fp64 values: integers next to 127 x / max|x| (ties to even) and
    scales max|x| / 127, rounded once to fp32.  Rows that are not finite: NaN and zeros."""
    with np.errstate(invalid="ignore"):
        a = np.abs(x).max(axis=-1, keepdims=True) if x.shape[-1] else np.zeros(x.shape[:-1] + (1,))
        finite = np.isfinite(x).all(axis=-1, keepdims=True)
        q = np.rint(127.0 * np.where(finite, x, 0.0) / np.where(finite & (a > 0), a, 1.0))
        scale = np.where(finite, a / 127.0, np.nan).astype(np.float32)
    return q, scale[..., 0].astype(np.float64)


def quantize_weights(w):
    """[E, K, N] -> integers [E, N, K], scales [E, N]."""
    return quantize(np.swapaxes(w, 1, 2))


def _stored(v, r):
    return bf16_to_f64(f64_to_bf16(v)) if r else v.astype(np.float32).astype(np.float64)


def network(x, q1, s1, b1, q2, s2, b2, kind, gated, r):
    """One expert on rows x [n, d]: (y, bound) before y's own rounding."""
    h = q2.shape[1]
    q, sx = quantize(x)
    pre = (q @ q1.T) * sx[:, None] * s1
    pe = 4 * U32 * np.abs(pre)  # the sum in fp32, two products, or one and a joint one with the bias
    if b1 is not None:
        pre = pre + b1
        pe = pe + U32 * (np.abs(pre) + pe)
    hid, he = ox.act(kind, pre[:, :h])[0], ox.act_error(kind, pre[:, :h], pe[:, :h])[0]
    if gated:
        u, ue = pre[:, h:], pe[:, h:]
        he = he * np.abs(u) + (np.abs(hid) + he) * ue + U32 * np.abs(hid * u)
        hid = hid * u
    # what may be stored, lowest and highest, and with it the row's largest value
    lo, mid, hi = _stored(hid - he, r), _stored(hid, r), _stored(hid + he, r)
    most = np.maximum(np.abs(lo), np.abs(hi)).max(axis=1, keepdims=True)
    least = np.where((lo > 0) | (hi < 0), np.minimum(np.abs(lo), np.abs(hi)), 0.0).max(axis=1, keepdims=True)
    qm, sm = quantize(mid)
    value = qm * sm[:, None]
    off = np.zeros_like(value)
    for v in (lo, mid, hi):
        for a in (least, most):
            other = np.rint(127.0 * v / np.where(a > 0, a, 1.0)).clip(-127, 127) * (a / 127.0)
            off = np.maximum(off, np.abs(other - value))
    off = off + 2 * U32 * np.abs(value)
    w2 = q2 * s2[:, None]
    y = value @ w2.T
    ye = off @ np.abs(w2).T + 4 * U32 * np.abs(y)
    if b2 is not None:
        y = y + b2
        ye = ye + U32 * (np.abs(y) + ye)
    return y, ye


def experts(xe, q1, s1, b1, q2, s2, b2, counts, kind, gated, r):
    """(ye, bound) [E, C, d], zero rows behind counts."""
    E, C, d = xe.shape
    y, err = np.zeros((E, C, d)), np.zeros((E, C, d))
    for e, n in enumerate(ox._rows(counts, E, C)):
        if n:
            v, ve = network(xe[e, :n], q1[e], s1[e], None if b1 is None else b1[e], q2[e], s2[e],
                            None if b2 is None else b2[e], kind, gated, r)
            y[e, :n], err[e, :n] = v, ve + r * (np.abs(v) + ve)
    return y, err


def token_layer(x, ids, weights, q1, s1, b1, q2, s2, b2, kind, gated, r):
    """(y, bound) from given ids and weights [S, k]; an id outside [0, E) adds nothing."""
    S, d = x.shape
    y, err, mag = np.zeros((S, d)), np.zeros((S, d)), np.zeros((S, d))
    for s in range(S):
        for e, w in zip(ids[s], weights[s]):
            if 0 <= e < q1.shape[0]:
                v, ve = network(x[s:s + 1], q1[e], s1[e], None if b1 is None else b1[e], q2[e], s2[e],
                                None if b2 is None else b2[e], kind, gated, r)
                y[s] += w * v[0]
                err[s] += abs(w) * ve[0]
                mag[s] += np.abs(w * v[0])
    err = err + (ids.shape[1] + 2) * U32 * (mag + err)
    return y, err + r * (np.abs(y) + err)
