"""Launches of more than 2^20 blocks, whose blocks lie along two dimensions of the grid with the last row
partly filled: the first rows, those around the border, the last ones, and what lies behind them."""

import numpy as np
import pytest
import torch

import paper_2203_14685_amd as hm
from oracle import dropout as od
from oracle import int8 as oi

from _experts import DEV, announce, f64

pytestmark = pytest.mark.gpu

GUARD = 64


@pytest.fixture(autouse=True, scope="module")
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    hm.load()
    yield


def test_quantized_rows():
    rows, n = 2 ** 24 + 17, 16  # 16 rows of 16 per block
    announce(f"quantize rows={rows} n={n}")
    x = torch.randn(rows, n, dtype=torch.bfloat16, device=DEV)
    q = torch.full((rows * n + GUARD,), 99, dtype=torch.int8, device=DEV)
    s = torch.full((rows + GUARD,), -1.0, device=DEV)
    hm.moe_quantize(rows, n, hm.MOE_BF16, x, q, s)
    assert (q[rows * n:] == 99).all() and (s[rows:] == -1).all()
    assert (s[:rows] > 0).all()  # every row was reached
    for lo in (0, 2 ** 24 - 300, rows - 300):
        want_q, want_s = oi.quantize(f64(x[lo:lo + 300]))
        assert np.array_equal(f64(q[lo * n:(lo + 300) * n]).reshape(300, n), want_q), lo
        assert np.array_equal(f64(s[lo:lo + 300]), want_s), lo


def test_embedding_rows():
    T, V, d = 2 ** 29 + 300, 50, 8  # rows of one piece, 512 per block
    announce(f"embed T={T} d={d}")
    table = torch.randn(V, d, dtype=torch.bfloat16, device=DEV)
    ids = (torch.arange(T, device=DEV, dtype=torch.int32) % (V + 1)) - 1  # the first of each 51 is padding
    y = torch.full((T * d + GUARD,), 7.0, dtype=torch.bfloat16, device=DEV)
    hm.moe_embed(hm.embed_params(T, V, d, hm.MOE_BF16), ids, table, y)
    assert (y[T * d:] == 7).all()
    padded = torch.cat([torch.zeros(1, d, dtype=torch.bfloat16, device=DEV), table])
    for lo in list(range(0, T - 2 ** 24, 2 ** 26)) + [2 ** 29 - 300, T - 500]:
        n = min(T - lo, 2 ** 22)
        assert torch.equal(y[lo * d:(lo + n) * d].view(n, d), padded[ids[lo:lo + n].long() + 1]), lo


def test_dropped_elements():
    n = 2 ** 32 + 4096 + 5  # 4096 elements per block
    announce(f"dropout n={n}")
    x = torch.ones(n + GUARD, dtype=torch.bfloat16, device=DEV)
    hm.dropout(x[:n], hm.dropout_mask(0.5, 78, 6), out=x[:n])
    assert (x[n:] == 1).all()
    for first in (0, 2 ** 32 - 3000, n - 3000):
        k = min(6000, n - first)
        assert np.array_equal(f64(x[first:first + k]), od.factors(first, k, 0.5, 78, 6)), first
