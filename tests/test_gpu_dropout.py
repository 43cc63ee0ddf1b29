"""Dropout of rows and inside the expert networks against the fp64 oracle: types, odd
lengths, shares 0 and 1, values that are not finite in dropped places, in place, the step in
device memory under a graph, two streams; and that both forms drop the same elements."""

import numpy as np
import pytest
import torch

import paper_2203_14685_amd as hm
from oracle import dropout as od

from _experts import ACTS, DEV, ROUND, TORCH, announce, check, f64, normal, weights

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True, scope="module")
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    hm.load()
    yield


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", [1, 7, 8, 9, 63, 4096, 8191, 70001])
def test_rows(n, dtype):
    for p, residual, seed, call in ((0.1, True, 3, 0), (0.5, False, 2 ** 63 + 12345, 2 ** 40 + 7), (0.999, True, 0, 2 ** 64 - 1)):
        announce(f"dropout {dtype} n={n} p={p} residual={residual}")
        rng = np.random.default_rng(n)
        x, xv = normal(rng, (n,), dtype)
        r, rv = normal(rng, (n,), dtype)
        y = hm.dropout(x.to(DEV), hm.dropout_mask(p, seed, call), residual=r.to(DEV) if residual else None)
        f = od.factors(0, n, p, seed, call)
        check(y, od.dropout(xv, f, rv if residual else None, ROUND[dtype]), "y")
        if not residual:
            assert np.array_equal(f64(y) == 0, (f == 0) | (xv == 0))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_shares_of_nothing_and_all(dtype):
    x = torch.randn(1000, device=DEV).to(TORCH[dtype])
    r = torch.randn(1000, device=DEV).to(TORCH[dtype])
    assert torch.equal(hm.dropout(x, hm.dropout_mask(0.0, 1)), x)
    assert torch.equal(hm.dropout(x, hm.dropout_mask(1.0, 1), residual=r), r)
    assert not hm.dropout(x, hm.dropout_mask(1.0, 1)).any()
    # a share below half a step of 2^-16 drops nothing
    assert torch.equal(hm.dropout(x, hm.dropout_mask(7e-6, 1)), x)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_dropped_values_may_be_anything(dtype):
    n, p = 5000, 0.4
    f = od.factors(0, n, p, 5, 6)
    x = torch.ones(n, dtype=TORCH[dtype])
    for i, bad in enumerate((float("nan"), float("inf"), float("-inf"))):
        x[torch.from_numpy(np.flatnonzero(f == 0)[i::3])] = bad
    y = f64(hm.dropout(x.to(DEV), hm.dropout_mask(p, 5, 6)))
    assert (y[f == 0] == 0).all() and not np.signbit(y[f == 0]).any()
    assert np.abs(y[f > 0] - f[f > 0]).max() <= (ROUND[dtype] + 2 ** -23) * f.max()
    kept = int(np.flatnonzero(f > 0)[0])
    x = torch.ones(n, dtype=TORCH[dtype])
    x[kept] = float("nan")
    assert np.isnan(f64(hm.dropout(x.to(DEV), hm.dropout_mask(p, 5, 6)))[kept])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_in_place_and_its_neighbours(dtype):
    x = torch.randn(4099 + 64, device=DEV).to(TORCH[dtype])
    r = torch.randn(4099, device=DEV).to(TORCH[dtype])
    m = hm.dropout_mask(0.3, 8)
    want = hm.dropout(x[:4099], m, residual=r)
    a, c = x.clone(), r.clone()
    assert hm.dropout(a[:4099], m, residual=r, out=a[:4099]).data_ptr() == a.data_ptr()
    assert torch.equal(a[:4099], want) and torch.equal(a[4099:], x[4099:])
    hm.dropout(x[:4099], m, residual=c, out=c)
    assert torch.equal(c, want)


def test_far_elements():
    """Past 2^31 elements: the words of the first and the last ones."""
    n = 2 ** 31 + 12345
    announce(f"dropout n={n}")
    x = torch.ones(n, dtype=torch.bfloat16, device=DEV)
    hm.dropout(x, hm.dropout_mask(0.5, 77, 5), out=x)
    for first in (0, 2 ** 31 - 64, n - 1000):
        k = min(1000, n - first)
        assert np.array_equal(f64(x[first:first + k]), od.factors(first, k, 0.5, 77, 5)), first


def test_step_under_a_graph_and_on_another_stream():
    n = 3000
    x = torch.randn(n, device=DEV)
    step = torch.zeros(1, dtype=torch.int64, device=DEV)
    m = hm.dropout_mask(0.5, 9, 2 ** 41, step)
    y = torch.empty_like(x)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        hm.dropout(x, m, out=y)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        hm.dropout(x, m, out=y)
        step.add_(1)
    step.zero_()
    seen = []
    for i in range(4):
        graph.replay()
        torch.cuda.synchronize()
        want = od.factors(0, n, 0.5, 9, 2 ** 41 + i)
        assert np.array_equal(f64(y) != 0, want > 0)
        seen.append(y.clone())
        assert torch.equal(y, hm.dropout(x, hm.dropout_mask(0.5, 9, 2 ** 41 + i)))  # eager work between replays
    assert not torch.equal(seen[0], seen[1])
    # two streams at once
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    big = torch.randn(1 << 22, device=DEV)
    torch.cuda.synchronize()
    a = hm.dropout(big, hm.dropout_mask(0.1, 1), stream=s1)
    b = hm.dropout(big, hm.dropout_mask(0.1, 2), stream=s2)
    torch.cuda.synchronize()
    assert torch.equal(a, hm.dropout(big, hm.dropout_mask(0.1, 1))) and torch.equal(b, hm.dropout(big, hm.dropout_mask(0.1, 2)))


# ---------------------------------------------------------------- inside the experts

SHAPES = [
    # E, C, d, h: one row; tiles cut short; around 64, 128 and 256 rows; rows of hidden that
    # begin inside a block of 8 elements (fp32, h = 4 mod 8)
    (1, 1, 8, 8), (4, 5, 72, 200), (3, 65, 136, 264), (5, 129, 64, 8), (3, 300, 8, 328), (3, 130, 264, 520), (2, 257, 520, 24),
]


def _counts(rng, E, C):
    c = rng.integers(0, C + 1, E)
    for e, v in zip(range(E), (0, min(1, C), C)):
        c[e] = v
    return c.astype(np.int32)


def _case(E, C, d, h, dtype, act, gated, p, seed):
    rng = np.random.default_rng(seed)
    xe, xv = normal(rng, (E, C, d), dtype)
    w = weights(rng, E, d, h, gated, dtype)
    counts = _counts(rng, E, C)
    for e in range(E):
        xe[e, counts[e]:] = float("nan")  # not read
    f = od.factors(0, E * C * h, p, seed, 2 ** 33 + 1).reshape(E, C, h)
    return rng, xe.to(DEV), xv, w, counts, f, hm.dropout_mask(p, seed, 2 ** 33 + 1)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("E,C,d,h", SHAPES + [(3, 33, 20, 52)])
def test_experts(E, C, d, h, dtype):
    if dtype == "bf16" and h % 8:
        d, h = 24, 56
    for i, (act, gated, p) in enumerate([("relu", False, 0.4), ("silu", True, 0.1), ("gelu", False, 0.9)]):
        announce(f"experts dropout {dtype} E={E} C={C} d={d} h={h} {act} gated={gated} p={p}")
        rng, x, xv, ((w1, w1v), (b1, b1v), (w2, w2v), (b2, b2v)), counts, f, m = _case(E, C, d, h, dtype, act, gated, p, 11 + i)
        cd = torch.from_numpy(counts).to(DEV)
        o = hm.experts(x, w1, w2, b1=b1, b2=b2, counts=cd, act=ACTS[act], gated=gated, want_pre=True, dropout=m)
        ref = od.experts(xv, w1v, b1v, w2v, b2v, counts, ACTS[act], gated, ROUND[dtype], f)
        for key in ("pre", "hidden", "ye"):
            check(o[key], ref[key], key)
        # backward, from what the forward pass stored; rows behind the counts are not read
        dye, dyv = normal(rng, (E, C, d), dtype)
        pre, hid = o["pre"].clone(), o["hidden"].clone()
        for e in range(E):
            dye[e, counts[e]:] = float("nan")
            pre[e, counts[e]:] = float("nan")
            hid[e, counts[e]:] = float("nan")
        g = hm.experts_bwd(dye.to(DEV), x, w1, w2, pre, hid, counts=cd, act=ACTS[act], gated=gated, dropout=m)
        gref = od.experts_bwd(dyv, xv, w1v, w2v, counts, f64(o["pre"]), f64(o["hidden"]), ACTS[act], gated, ROUND[dtype], f)
        for key in ("dxe", "dw1", "db1", "dw2", "db2"):
            check(g[key], gref[key], key)


@pytest.mark.parametrize("dtype,gated,big", [("bf16", True, True), ("bf16", False, True), ("f32", False, True), ("f32", True, False)])
def test_experts_drop_what_rows_drop(dtype, gated, big):
    """Tiles of every size: hidden is dropout() of the hidden without dropout, up to its rounding,
    and with nothing dropped every result is that of the plain call, bit for bit."""
    E, C, d, h = (4, 1300, 256, 2048) if big else (2, 70, 64, 72)
    announce(f"experts dropout against rows {dtype} gated={gated} E={E} C={C} d={d} h={h}")
    rng = np.random.default_rng(0)
    xe = normal(rng, (E, C, d), dtype)[0].to(DEV)
    (w1, _), (b1, _), (w2, _), (b2, _) = weights(rng, E, d, h, gated, dtype)
    dye = normal(rng, (E, C, d), dtype)[0].to(DEV)
    kw = dict(act=ACTS["silu"], gated=gated)
    plain = hm.experts(xe, w1, w2, b1=b1, b2=b2, want_pre=True, **kw)
    m = hm.dropout_mask(0.3, 21, 4)
    o = hm.experts(xe, w1, w2, b1=b1, b2=b2, want_pre=True, dropout=m, **kw)
    assert torch.equal(o["pre"], plain["pre"])
    f = od.factors(0, E * C * h, 0.3, 21, 4).reshape(E, C, h)
    got, want = f64(o["hidden"]), f64(plain["hidden"]) * f
    assert (got[f == 0] == 0).all()
    # two roundings of hidden and one product on either side
    assert (np.abs(got - want) <= (2 * ROUND[dtype] + ROUND[dtype] ** 2 + 4 * 2.0 ** -24) * np.abs(want)).all()
    zero = hm.dropout_mask(0.0, 21, 4)
    z = hm.experts(xe, w1, w2, b1=b1, b2=b2, want_pre=True, dropout=hm.dropout_mask(1.0, 21, 4), **kw)
    assert not z["hidden"].any() and torch.equal(z["pre"], plain["pre"])  # all dropped: the bias is what remains
    assert (f64(z["ye"]) == f64(b2.to(TORCH[dtype]))[:, None, :]).all()
    z = hm.experts(xe, w1, w2, b1=b1, b2=b2, want_pre=True, dropout=zero, **kw)
    for key in ("pre", "hidden", "ye"):
        assert torch.equal(z[key], plain[key])
    g0 = hm.experts_bwd(dye, xe, w1, w2, plain["pre"], plain["hidden"], **kw)
    gz = hm.experts_bwd(dye, xe, w1, w2, plain["pre"], plain["hidden"], dropout=zero, **kw)
    g = hm.experts_bwd(dye, xe, w1, w2, o["pre"], o["hidden"], dropout=m, **kw)
    again = hm.experts_bwd(dye, xe, w1, w2, o["pre"], o["hidden"], dropout=m, **kw)
    for key in g0:
        assert torch.equal(g0[key], gz[key]) and torch.equal(g[key], again[key]), key
    assert torch.equal(g["db2"], g0["db2"]) and not torch.equal(g["dxe"], g0["dxe"])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_dropped_places_of_pre_may_be_anything(dtype):
    E, C, d, h = 2, 20, 16, 24
    for act, gated in (("gelu", False), ("silu", True)):
        announce(f"experts dropout, pre that is not finite {dtype} {act} gated={gated}")
        rng, x, xv, ((w1, w1v), (b1, b1v), (w2, w2v), (b2, b2v)), counts, f, m = _case(E, C, d, h, dtype, act, gated, 0.5, 4)
        cd = torch.from_numpy(counts).to(DEV)
        o = hm.experts(x, w1, w2, b1=b1, b2=b2, counts=cd, act=ACTS[act], gated=gated, want_pre=True, dropout=m)
        dye, dyv = normal(rng, (E, C, d), dtype)
        args = dict(counts=cd, act=ACTS[act], gated=gated, dropout=m)
        g = hm.experts_bwd(dye.to(DEV), x, w1, w2, o["pre"], o["hidden"], **args)
        bad = o["pre"].clone()
        gone = torch.from_numpy(np.concatenate([f, f], axis=2) == 0 if gated else f == 0).to(DEV)
        bad[gone] = float("nan")
        b = hm.experts_bwd(dye.to(DEV), x, w1, w2, bad, o["hidden"], **args)
        for key in g:
            assert torch.equal(g[key], b[key]), key
