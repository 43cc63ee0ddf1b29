"""Weights that hold infinities or NaN, and pre-activations of the largest magnitudes: what
is not finite shows in the sums it enters over the rows in use, and nowhere else."""

import numpy as np
import pytest
import torch

import paper_2203_14685_amd as hm

from _experts import ACTS, DEV, TORCH, announce, normal, weights

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True, scope="module")
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    hm.load()
    yield


# tiles of 64, 128 and 256 rows in bf16, of 64 and 32 in fp32; the counts end inside a tile
SHAPES = [(3, 70, 64, 136), (32, 100, 16, 1032), (70, 260, 16, 400), (4, 200, 520, 72)]


def _same_but(a, b, hit, what):
    """a equals b bit for bit where `hit` (broadcast to them) does not hold."""
    hit = hit.expand_as(a)
    assert torch.equal(a[~hit], b[~hit]), what


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("E,C,d,h", SHAPES)
@pytest.mark.parametrize("act,gated", [("relu", False), ("silu", True), ("gelu", False)])
def test_infinite_second_weight_in_the_gradients(E, C, d, h, act, gated, dtype):
    """w2[e, j, c] = inf makes dhidden[:, j] of the rows in use infinite, all of one sign where
    dye[:, c] is positive, and with positive pre-activations dpre too: db1[e, j] is inf.  Rows
    behind the count add nothing, and no other column changes."""
    announce(f"experts_bwd infinite w2 {dtype} E={E} C={C} d={d} h={h} {act} gated={gated}")
    rng = np.random.default_rng(E + C)
    (w1, _), _, (w2, _), _ = weights(rng, E, d, h, gated, dtype, False)
    h1 = w1.shape[2]
    counts = rng.integers(1, C, E).astype(np.int32)
    counts[0] = 1
    xe, dye = (normal(rng, (E, C, d), dtype)[0] for _ in range(2))
    pre = (normal(rng, (E, C, h1), "f32")[0].abs() + 0.25).to(TORCH[dtype])
    hidden = normal(rng, (E, C, h), dtype)[0]
    c, j = d // 2, h - 3
    dye[:, :, c] = dye[:, :, c].abs() + 0.5
    for e in range(E):
        for t in (xe, dye, pre, hidden):
            t[e, counts[e]:] = float("nan")
    xe, dye, pre, hidden = (t.to(DEV) for t in (xe, dye, pre, hidden))
    cd = torch.from_numpy(counts).to(DEV)
    kw = dict(counts=cd, act=ACTS[act], gated=gated)
    base = hm.experts_bwd(dye, xe, w1, w2, pre, hidden, **kw)
    bad = torch.arange(E, device=DEV) % 3 != 1  # experts that get the infinity
    w2[bad, j, c] = float("inf")
    o = hm.experts_bwd(dye, xe, w1, w2, pre, hidden, **kw)
    torch.cuda.synchronize()
    col = torch.zeros(h1, dtype=torch.bool, device=DEV)
    col[[j, h + j] if gated else [j]] = True
    hit = bad[:, None] & col[None, :]
    assert all(torch.isfinite(base[key]).all() for key in base)
    assert (o["db1"][hit] == float("inf")).all(), o["db1"][hit][:4]
    _same_but(o["db1"], base["db1"], hit, "db1")
    _same_but(o["dw1"], base["dw1"], hit[:, None, :], "dw1")
    assert torch.equal(o["db2"], base["db2"]) and torch.equal(o["dw2"], base["dw2"])
    _same_but(o["dxe"], base["dxe"], bad[:, None, None], "dxe")
    used = torch.arange(C, device=DEV)[None, :] < cd[:, None]
    assert (o["dxe"][~used] == 0).all() and not torch.isfinite(o["dxe"][used & bad[:, None]]).any()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("E,C,d,h", SHAPES)
@pytest.mark.parametrize("bad", [float("inf"), float("nan")])
def test_weights_that_are_not_finite_in_the_forward_pass(E, C, d, h, bad, dtype):
    """A bad element of w1 spoils its column of pre and hidden, one of w2 its column of ye, in
    the rows in use of its expert; rows behind the count are zeros."""
    announce(f"experts weights {bad} {dtype} E={E} C={C} d={d} h={h}")
    rng = np.random.default_rng(E + C)
    (w1, _), (b1, _), (w2, _), (b2, _) = weights(rng, E, d, h, False, dtype)
    counts = rng.integers(0, C, E).astype(np.int32)
    cd = torch.from_numpy(counts).to(DEV)
    xe = normal(rng, (E, C, d), dtype)[0].to(DEV)
    used = torch.arange(C, device=DEV)[None, :] < cd[:, None]
    xe[~used] = float("nan")
    kw = dict(b1=b1, b2=b2, counts=cd, act=hm.MOE_ACT_SILU, want_pre=True)
    base = hm.experts(xe, w1, w2, **kw)
    e, j, c = E - 1, h // 2, d - 1
    v1, v2 = w1.clone(), w2.clone()
    v1[e, 3, j], v2[e, j, c] = bad, bad
    first, second = hm.experts(xe, v1, w2, **kw), hm.experts(xe, w1, v2, **kw)
    torch.cuda.synchronize()
    here = torch.zeros(E, dtype=torch.bool, device=DEV)
    here[e] = True

    def hit(n, i):
        m = used[:, :, None] & here[:, None, None] & torch.ones(n, dtype=torch.bool, device=DEV)
        if i is not None:
            m = m & (torch.arange(n, device=DEV) == i)
        return m

    for o, where in ((first, dict(pre=hit(h, j), hidden=hit(h, j), ye=hit(d, None))),
                     (second, dict(pre=hit(h, j) & False, hidden=hit(h, j) & False, ye=hit(d, c)))):
        for key, m in where.items():
            _same_but(o[key], base[key], m, key)
            assert (o[key][~used] == 0).all(), key
    assert not torch.isfinite(second["ye"][hit(d, c)]).any()
    if bad != bad:
        assert torch.isnan(first["pre"][hit(h, j)]).all() and torch.isnan(first["ye"][hit(d, None)]).all()


# beyond 1.8e19 a square leaves fp32, beyond 7e12 a cube
LARGE = [1e6, 7e12, 1e15, 1.7e19, 2e19, 6e19, 1e25, 3e38]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("act", sorted(ACTS))
@pytest.mark.parametrize("gated", [False, True])
def test_derivatives_of_large_pre_activations(act, gated, dtype):
    """One row with dhidden = 1, so db1 is the activation's derivative: 1 to the right, 0 to the left
    (gated, the other half's are the activation itself)."""
    announce(f"experts_bwd large pre {dtype} {act} gated={gated}")
    a = torch.tensor([[LARGE + [-v for v in LARGE]]]).to(TORCH[dtype])
    h, d = 16, 8
    pre = torch.cat([a, torch.ones_like(a)], dim=2) if gated else a
    w1 = torch.zeros((1, d, pre.shape[2]), dtype=a.dtype, device=DEV)
    w2 = torch.zeros((1, h, d), dtype=a.dtype, device=DEV)
    w2[:, :, 0] = 1
    dye = torch.zeros((1, 1, d), dtype=a.dtype, device=DEV)
    dye[0, 0, 0] = 1
    hid = torch.zeros((1, 1, h), dtype=a.dtype, device=DEV)
    o = hm.experts_bwd(dye, torch.ones_like(dye), w1, w2, pre.to(DEV), hid, act=ACTS[act], gated=gated)
    torch.cuda.synchronize()
    # the sigmoid of such arguments is exactly 1 or 0
    av = a.to(DEV).float()[0]
    assert torch.equal(o["db1"][:, :h], (av > 0).float()), o["db1"]
    if gated:
        assert torch.equal(o["db1"][:, h:], av.clamp(min=0)), o["db1"]
