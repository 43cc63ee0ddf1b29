"""The layer for few tokens where the second product's K is split over blocks, whose parts the
combine adds: narrow and wide strips, blocks per choice and per expert, passes side by side."""

import numpy as np
import pytest
import torch

import paper_2203_14685_amd as hm
from oracle import experts as ox

from _experts import ACTS, DEV, ROUND, announce, check, f64, normal, weights

# S, d, E, k, h, parts of K in both types: narrow strips (up to 16 tokens) by choice, more than four parts, by expert;
# wide ones by expert, by choice, with two and three tiles of rows, passes side by side
SPLIT = [(1, 64, 8, 2, 8200, 4), (1, 64, 8, 2, 12296, 6), (9, 72, 4, 2, 12296, 6), (40, 72, 4, 2, 2600, 5),
         (17, 40, 40, 2, 1544, 3), (20, 72, 6, 2, 2056, 4), (100, 136, 2, 2, 4104, 8), (200, 72, 2, 1, 2600, 5),
         (256, 72, 1, 1, 1032, 2)]


def _align(n):
    return (n + 255) // 256 * 256


def _params(S, d, E, k, h, dtype, act="silu", gated=False):
    return hm.token_layer_params(S, d, E, k, h, act=ACTS[act], gated=gated, routed=True,
                                 dtype=hm.MOE_BF16 if dtype == "bf16" else hm.MOE_F32)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("S,d,E,k,h,parts", SPLIT)
def test_workspace_holds_the_parts(S, d, E, k, h, parts, dtype):
    """With given routing: hidden in 4 bytes a value, and `parts` sums of each choice's row."""
    size = hm.moe_token_layer_workspace_size(_params(S, d, E, k, h, dtype))
    assert size == _align(S * k * h * 4) + _align(parts * S * k * d * 4)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("S,d,E,k,h,parts", SPLIT)
def test_split_sums(S, d, E, k, h, parts, dtype):
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    for act, gated, case in (("gelu", False, "even"), ("silu", True, "mixed"), ("relu", False, "one")):
        announce(f"token_layer split {dtype} S={S} d={d} E={E} k={k} h={h} {act} gated={gated} {case}")
        rng = np.random.default_rng(S + h)
        x, xv = normal(rng, (S, d), dtype)
        (w1, w1v), (b1, b1v), (w2, w2v), (b2, b2v) = weights(rng, E, d, h, gated, dtype)
        ids = rng.integers(0, E, (S, k)).astype(np.int32)
        if case == "mixed":  # padding among them
            ids = np.where(rng.random((S, k)) < 0.3, -1, ids).astype(np.int32)
        if case == "one":    # one expert has all rows
            ids[:] = E - 1
        w, wv = normal(rng, (S, k), "f32")
        p = _params(S, d, E, k, h, dtype, act, gated)
        ws = torch.full((hm.moe_token_layer_workspace_size(p),), 255, dtype=torch.uint8, device=DEV)  # NaN
        y = torch.full((S, d), -7.0, dtype=x.dtype, device=DEV)
        hm.moe_token_layer(p, x.to(DEV), None, None, None, None, None, w1, b1, w2, b2, torch.from_numpy(ids).to(DEV),
                           w.to(DEV), y, ws)
        torch.cuda.synchronize()
        ref = ox.token_layer(xv, ids, wv, w1v, b1v, w2v, b2v, ACTS[act], gated, ROUND[dtype])
        check(y, ref, f"y {act} gated={gated} {case}")


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("S,E,k,h", [(1, 8, 2, 136), (40, 4, 2, 264), (3, 8, 1, 8200)])
def test_infinite_second_weight(S, E, k, h, dtype):
    """w2[e, j, c] = inf with hidden[j] > 0 makes y[:, c] of the rows that chose e infinite, of their
    weight's sign, whichever way hidden rounds, and changes no other value."""
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    announce(f"token_layer infinite w2 {dtype} S={S} E={E} k={k} h={h}")
    rng = np.random.default_rng(S)
    d = 64
    x = normal(rng, (S, d), dtype)[0].to(DEV)
    (w1, _), (b1, _), (w2, _), (b2, _) = weights(rng, E, d, h, False, dtype)
    ids = torch.from_numpy(np.stack([rng.permutation(E)[:k] for _ in range(S)]).astype(np.int32)).to(DEV)
    w = normal(rng, (S, k), "f32")[0].to(DEV)
    kw = dict(b1=b1, b2=b2, act=hm.MOE_ACT_RELU, ids=ids, weights=w)
    b1[:] = b1.abs() + 12.0  # every hidden value positive: a row of x times a column of w1 is some 1 +- 1
    w1.clamp_(-0.5, 0.5)
    base = hm.token_layer(x, w1, w2, **kw)["y"]
    e = int(ids[0, 0])
    hit = (ids == e)
    for j in range(0, h, max(1, h // 24)):  # hidden values of many roundings
        v = w2.clone()
        v[e, j, 5] = float("inf")
        y = hm.token_layer(x, w1, v, **kw)["y"]
        torch.cuda.synchronize()
        sign = (w.sign() * hit).sum(dim=1)
        rows = hit.any(dim=1)
        assert (y[rows, 5].float() == sign[rows] * float("inf")).all(), (j, y[rows, 5])
        same = torch.ones_like(y, dtype=torch.bool)
        same[rows, 5] = False
        assert torch.equal(y[same], base[same]), j
