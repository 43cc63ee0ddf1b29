"""Dropout in fp64, alone and inside the expert networks.

The random words are Philox4x32-10 (Salmon, Moraes, Dror, Shaw, "Parallel random
numbers: as easy as 1, 2, 3", SC 2011), in 64-bit integers; the paper's known answers
pin it.  Bounds are those of `oracle.experts`: `r` is the unit roundoff of the element
type (0 for fp32).
"""

import numpy as np

from . import experts as ox

_M = np.uint64(0xFFFFFFFF)


def philox4x32(counter, key, rounds=10):
    """counter [..., 4], key [..., 2] of 32-bit values -> [..., 4]."""
    c = [np.asarray(counter[..., i], dtype=np.uint64) for i in range(4)]
    k = [np.asarray(key[..., i], dtype=np.uint64) for i in range(2)]
    for _ in range(rounds):
        a, b = np.uint64(0xD2511F53) * c[0], np.uint64(0xCD9E8D57) * c[2]
        c = [(b >> np.uint64(32)) ^ c[1] ^ k[0], b & _M, (a >> np.uint64(32)) ^ c[3] ^ k[1], a & _M]
        k = [(k[0] + np.uint64(0x9E3779B9)) & _M, (k[1] + np.uint64(0xBB67AE85)) & _M]
    return np.stack(c, axis=-1)


def words(first, n, seed, call):
    """The 16-bit words of elements first .. first + n - 1."""
    i = np.arange(first, first + n, dtype=np.uint64)
    block = i >> np.uint64(3)
    blocks, back = np.unique(block, return_inverse=True)
    one = np.ones_like(blocks)
    call, seed = int(call) % 2 ** 64, int(seed) % 2 ** 64
    counter = np.stack([blocks & _M, blocks >> np.uint64(32), one * np.uint64(call & 0xFFFFFFFF), one * np.uint64(call >> 32)], -1)
    key = np.stack([one * np.uint64(seed & 0xFFFFFFFF), one * np.uint64(seed >> 32)], -1)
    w = philox4x32(counter, key)[back, (i % np.uint64(8) // np.uint64(2)).astype(np.int64)]
    return (w >> (np.uint64(16) * (i & np.uint64(1)))) & np.uint64(0xFFFF)


def factors(first, n, p, seed, call):
    """What each element is multiplied by: 0, or 2^16 / (2^16 - t)."""
    t = int(np.rint(float(np.float32(p)) * 65536.0))
    keep = words(first, n, seed, call) >= t
    return np.where(keep, 65536.0 / (65536 - t) if t < 65536 else 0.0, 0.0)


def dropout(x, f, residual, r):
    """(value, bound) of residual + f x; a dropped x counts as 0 whatever it holds."""
    v = np.where(f > 0, x, 0.0) * f
    y = v if residual is None else residual + v
    err = 2 * ox.U32 * np.abs(v) + ox.U32 * np.abs(y)
    return y, err + r * (np.abs(y) + err)


def experts(xe, w1, b1, w2, b2, counts, kind, gated, r, f):
    """oracle.experts.experts with hidden multiplied by f [E, C, h] before its rounding."""
    E, C, d = xe.shape
    h, h1 = w2.shape[1], w1.shape[2]
    out = {key: (np.zeros((E, C, n)), np.zeros((E, C, n))) for key, n in (("pre", h1), ("hidden", h), ("ye", d))}
    for e, n in enumerate(ox._rows(counts, E, C)):
        pre, pe = ox._bias(*ox._product(xe[e, :n], w1[e], None, None), None if b1 is None else b1[e])
        hid, he = ox.act(kind, pre[:, :h])[0], ox.act_error(kind, pre[:, :h], pe[:, :h])[0]
        if gated:
            u, ue = pre[:, h:], pe[:, h:]
            he = he * np.abs(u) + (np.abs(hid) + he) * ue + ox.U32 * np.abs(hid * u)
            hid = hid * u
        g = f[e, :n]
        he = he * g + 2 * ox.U32 * np.abs(hid) * g
        hid = hid * g
        he = he + r * (np.abs(hid) + he)
        y, ye = ox._bias(*ox._product(hid, w2[e], he, None), None if b2 is None else b2[e])
        for key, (v, err) in dict(pre=(pre, pe + r * (np.abs(pre) + pe)), hidden=(hid, he), ye=(y, ye + r * (np.abs(y) + ye))).items():
            out[key][0][e, :n], out[key][1][e, :n] = v, err
    return out


def experts_bwd(dye, xe, w1, w2, counts, pre, hidden, kind, gated, r, f):
    """oracle.experts.experts_bwd with dhidden multiplied by f; a dropped element's dpre is 0."""
    E, C, d = dye.shape
    h, h1 = w2.shape[1], w1.shape[2]
    shapes = dict(dxe=(E, C, d), dw1=(E, d, h1), db1=(E, h1), dw2=(E, h, d), db2=(E, d))
    out = {key: (np.zeros(s), np.zeros(s)) for key, s in shapes.items()}
    for e, n in enumerate(ox._rows(counts, E, C)):
        dy, x, hid, g = dye[e, :n], xe[e, :n], hidden[e, :n], f[e, :n]
        g2 = np.concatenate([g, g], axis=1) if gated else g
        p = np.where(g2 > 0, pre[e, :n], 0.0)
        dh, dhe = ox._product(dy, w2[e].T, None, None)
        dhe = dhe * g + 2 * ox.U32 * np.abs(dh) * g
        dh = dh * g
        a = p[:, :h]
        act, df = ox.act(kind, a)
        fe, dfe = ox.act_error(kind, a, np.zeros_like(a))
        if gated:
            u = p[:, h:]
            parts = [(dh * u * df, np.abs(u) * (dhe * (np.abs(df) + dfe) + np.abs(dh) * dfe) + 2 * ox.U32 * np.abs(dh * u * df)),
                     (dh * act, dhe * (np.abs(act) + fe) + np.abs(dh) * fe + ox.U32 * np.abs(dh * act))]
            dpre, dpe = (np.concatenate(q, axis=1) for q in zip(*parts))
        else:
            dpre, dpe = dh * df, dhe * (np.abs(df) + dfe) + np.abs(dh) * dfe + ox.U32 * np.abs(dh * df)
        stored = dpe + r * (np.abs(dpre) + dpe)
        ones = np.ones((1, n))
        vals = dict(dxe=ox._product(dpre, w1[e].T, stored, None), dw1=ox._product(x.T, dpre, None, stored),
                    dw2=ox._product(hid.T, dy, None, None))
        for key, (v, err) in vals.items():
            err = err + r * (np.abs(v) + err)
            if key == "dxe":
                out[key][0][e, :n], out[key][1][e, :n] = v, err
            else:
                out[key][0][e], out[key][1][e] = v, err
        for key, (v, err) in (("db1", ox._product(ones, dpre, None, dpe)), ("db2", ox._product(ones, dy, None, None))):
            out[key][0][e], out[key][1][e] = v[0], err[0]
    return out
