"""The 8-bit layer on another gate's choices where tokens name one expert several times: more rows of an
expert than tokens, at lengths where they fill the LDS of a block, in the first product and the second."""

import numpy as np
import pytest
import torch

import paper_2203_14685_amd as hm
from oracle import int8 as oi

from _experts import ACTS, DEV, ROUND, announce, check, normal

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True, scope="module")
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    hm.load()
    yield


def _quantized(rng, E, K, N):
    """Integers [E, N, K] and scales [E, N], on the device and for the oracle."""
    q = rng.integers(-127, 128, (E, N, K), dtype=np.int8)
    s = ((0.5 + rng.random((E, N))) * K ** -0.5 / 73).astype(np.float32)  # integers of 73 in the mean square
    return (torch.from_numpy(q).to(DEV), torch.from_numpy(s).to(DEV)), (q, s.astype(np.float64))


# rows that the first product's blocks hold at a time: one of two, three of eight, two of four, three of
# twelve (blocks by choice and by expert), one of four; and the second's: K in one block, and split
CASES = [(1, 2, 8192, 2, 48), (1, 8, 4096, 8, 32), (2, 2, 6144, 4, 32), (3, 4, 4096, 12, 48), (3, 4, 4096, 2, 48), (1, 4, 8176, 1, 16),
         (1, 8, 2112, 8, 3200), (2, 4, 64, 8, 8192), (1, 8, 48, 64, 8192), (4, 2, 512, 8, 4096)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("S,k,d,E,h", CASES)
def test_one_expert_named_by_all(S, k, d, E, h, dtype):
    rng = np.random.default_rng(S + d)
    x, xv = normal(rng, (S, d), dtype)
    for act, gated in (("gelu", False), ("silu", True)):
        (q1, s1), (q1v, s1v) = _quantized(rng, E, d, 2 * h if gated else h)
        (q2, s2), (q2v, s2v) = _quantized(rng, E, h, d)
        w = rng.random((S, k)).astype(np.float32)
        few = np.arange(S * k).reshape(S, k) % max(1, E // 2)
        few[0, 0] = -1  # padding
        for kind, ids in (("first", np.zeros((S, k))), ("last", np.full((S, k), E - 1)), ("some", few)):
            announce(f"token_layer_int8 {dtype} S={S} k={k} d={d} E={E} h={h} {act} gated={gated} ids={kind}")
            ids = ids.astype(np.int32)
            args = dict(act=ACTS[act], gated=gated, ids=torch.from_numpy(ids).to(DEV), weights=torch.from_numpy(w).to(DEV))
            y = hm.token_layer_int8(x.to(DEV), q1, s1, q2, s2, **args)["y"]
            ref = oi.token_layer(xv, ids, w.astype(np.float64), q1v, s1v, None, q2v, s2v, None, ACTS[act], gated, ROUND[dtype])
            check(y, ref, f"y, {kind}")
            assert torch.equal(y, hm.token_layer_int8(x.to(DEV), q1, s1, q2, s2, **args)["y"])
