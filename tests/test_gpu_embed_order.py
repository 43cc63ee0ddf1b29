"""The order of the sums of the table's gradient, bit for bit: an fp32 emulation of what the kernels state.  Tokens
sorted by id, stably; the sorted tokens in chunks of equal length, a run's part in each added in the tokens' order;
the parts of a run that crosses chunks added by eight waves, every eighth part each, then over the waves."""

import numpy as np
import pytest
import torch

import paper_2203_14685_amd as hm

from _experts import DEV, announce

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True, scope="module")
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    hm.load()
    yield


def _chunk(T, d):
    if T <= 32:
        return 32
    want, n = T * max(4 * d, 128) // 1024 // 4096, 8
    while n < 1024 and n < want:
        n *= 2
    return n


def _added(rows):
    total = np.zeros(rows.shape[1], dtype=np.float32)
    for r in rows:
        total = total + r
    return total


def _emulated(dy, ids, V, chunk):
    order = np.argsort(ids, kind="stable")
    keys = ids[order]
    out = np.zeros((V, dy.shape[1]), dtype=np.float32)
    for v in np.unique(keys):
        lo, hi = np.searchsorted(keys, v), np.searchsorted(keys, v, side="right")
        cuts = [lo] + [c for c in range(lo // chunk * chunk + chunk, hi, chunk)] + [hi]
        parts = np.stack([_added(dy[order[a:b]]) for a, b in zip(cuts, cuts[1:])])
        out[v] = parts[0] if len(parts) == 1 else _added(np.stack([_added(parts[w::8]) for w in range(8)]))
    return out


@pytest.mark.parametrize("T,V,d", [(20, 3, 8), (32, 1, 64), (33, 2, 8), (300, 4, 264), (3000, 4, 8), (5000, 300, 16), (8192, 7, 64),
                                   (8193, 7, 64), (20000, 3, 8), (20000, 500, 1032)])
def test_sums_run_in_the_stated_order(T, V, d):
    announce(f"embed_bwd order T={T} V={V} d={d}")
    rng = np.random.default_rng(T + d)
    # terms of every size, so that another order of a sum of more than a few of them gives another result
    dy = (rng.standard_normal((T, d)) * 2.0 ** rng.integers(-12, 13, (T, d))).astype(np.float32)
    ids = (rng.integers(0, V, T) * rng.integers(0, 2, T)).astype(np.int32)  # half of them 0
    want = _emulated(dy, ids, V, _chunk(T, d))
    got = hm.embed_bwd(torch.from_numpy(dy).to(DEV), torch.from_numpy(ids).to(DEV), V).cpu().numpy()
    assert np.array_equal(got.view(np.int32), want.view(np.int32))
    # the oracle tells orders apart: tokens of equal ids the other way round
    back = _emulated(dy[::-1], ids[::-1], V, _chunk(T, d))
    assert not np.array_equal(back, want)
