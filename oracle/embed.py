"""Embedding rows and their table's gradient in fp64, with bounds as in `oracle.experts`."""

import numpy as np

from .experts import U32


def embed(ids, table, scale, r):
    """(value, bound) of scale * table[ids]; ids outside the table give zero rows."""
    V = table.shape[0]
    inside = (ids >= 0) & (ids < V)
    y = np.where(inside[:, None], table[np.where(inside, ids, 0)] * scale, 0.0)
    err = U32 * np.abs(y)
    return y, err + r * (np.abs(y) + err)


def embed_bwd(dy, ids, V, scale, there, r):
    """(value, bound) of [there +] scale * the sum of dy over the tokens of each row; a row that no
    token names keeps `there` exactly."""
    d = dy.shape[1]
    inside = (ids >= 0) & (ids < V)
    total, mag, count = np.zeros((V, d)), np.zeros((V, d)), np.zeros((V, 1))
    np.add.at(total, ids[inside], dy[inside])
    np.add.at(mag, ids[inside], np.abs(dy[inside]))
    np.add.at(count, ids[inside], 1.0)
    v = scale * total
    err = (count + 1) * U32 * mag * abs(scale) + U32 * np.abs(v)
    if there is not None:
        v = there + v
        err = err + U32 * (np.abs(v) + err)
    err = err + r * (np.abs(v) + err)
    return v, np.where(count > 0, err, 0.0)
