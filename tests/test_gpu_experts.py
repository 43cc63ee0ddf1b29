"""Expert networks and their gradients against the fp64 oracle: types, activations,
odd widths, capacities around the tile sizes, experts without rows, rows behind the
counts that hold NaN, optional arguments, graphs, streams, and the training step
they complete."""

import numpy as np
import pytest
import torch

import paper_2203_14685_amd as hm
from oracle import experts as ox

from _experts import ACTS, DEV, ROUND, TORCH, announce, check, f64, normal, weights

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True, scope="module")
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    hm.load()
    yield


def _counts(rng, E, C):
    """No rows, one, all, and draws in between."""
    c = rng.integers(0, C + 1, E)
    for e, v in zip(range(E), (0, min(1, C), C)):
        c[e] = v
    return c.astype(np.int32)


SHAPES = [
    # E, C, d, h: one row; tiles of 64 cut short; around 64, 128 and 256 rows; wide and narrow
    (1, 1, 8, 8), (3, 1, 64, 128), (4, 5, 72, 200), (3, 64, 128, 64), (3, 65, 136, 264), (5, 129, 64, 8),
    (2, 257, 520, 24), (3, 300, 8, 328), (60, 7, 40, 72), (3, 130, 264, 520),
]


def _setup(E, C, d, h, dtype, gated, seed, bias=True, garbage=True):
    rng = np.random.default_rng(seed)
    xe, xv = normal(rng, (E, C, d), dtype)
    w = weights(rng, E, d, h, gated, dtype, bias)
    counts = _counts(rng, E, C)
    x = xe.clone()
    if garbage:  # what lies behind the counts may be anything
        for e in range(E):
            x[e, counts[e]:] = float("nan")
    return rng, x.to(DEV), xv, w, counts


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("E,C,d,h", SHAPES)
def test_forward(E, C, d, h, dtype):
    for i, (act, gated) in enumerate([("relu", False), ("gelu", True), ("silu", True), ("gelu", False), ("silu", False)]):
        if i >= 3 and E * C * d * h > 2_000_000:
            continue
        announce(f"experts {dtype} E={E} C={C} d={d} h={h} {act} gated={gated}")
        _, x, xv, ((w1, w1v), (b1, b1v), (w2, w2v), (b2, b2v)), counts = _setup(E, C, d, h, dtype, gated, 7 * i + C)
        o = hm.experts(x, w1, w2, b1=b1, b2=b2, counts=torch.from_numpy(counts).to(DEV), act=ACTS[act], gated=gated,
                       want_pre=True)
        torch.cuda.synchronize()
        ref = ox.experts(xv, w1v, b1v, w2v, b2v, counts, ACTS[act], gated, ROUND[dtype])
        for key in ("pre", "hidden", "ye"):
            check(o[key], ref[key], f"{key} {act} gated={gated}")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("E,C,d,h", SHAPES)
def test_backward(E, C, d, h, dtype):
    for i, (act, gated) in enumerate([("silu", True), ("relu", False), ("gelu", True), ("silu", False), ("relu", True)]):
        if i >= 3 and E * C * d * h > 2_000_000:
            continue
        announce(f"experts_bwd {dtype} E={E} C={C} d={d} h={h} {act} gated={gated}")
        rng, x, xv, ((w1, w1v), _, (w2, w2v), _), counts = _setup(E, C, d, h, dtype, gated, 11 * i + C)
        h1 = w1.shape[2]
        pre, pv = normal(rng, (E, C, h1), dtype)
        hid, hv = normal(rng, (E, C, h), dtype)
        dye, dv = normal(rng, (E, C, d), dtype)
        dev = []
        for t in (pre, hid, dye):
            t = t.clone()
            for e in range(E):
                t[e, counts[e]:] = float("nan")
            dev.append(t.to(DEV))
        o = hm.experts_bwd(dev[2], x, w1, w2, dev[0], dev[1], counts=torch.from_numpy(counts).to(DEV), act=ACTS[act],
                           gated=gated)
        torch.cuda.synchronize()
        ref = ox.experts_bwd(dv, xv, w1v, w2v, counts, pv, hv, ACTS[act], gated, ROUND[dtype])
        for key in ("dxe", "dw1", "db1", "dw2", "db2"):
            check(o[key], ref[key], f"{key} {act} gated={gated}")


@pytest.mark.parametrize("dtype,E,C,d,h,act,gated", [
    ("bf16", 16, 300, 512, 1024, "gelu", False), ("bf16", 8, 520, 256, 2048, "silu", True),
    ("f32", 8, 260, 512, 1024, "relu", False), ("bf16", 70, 33, 1400, 64, "relu", True)])
def test_large_tiles(dtype, E, C, d, h, act, gated):
    """Sizes that take the largest tiles in both directions."""
    announce(f"experts large {dtype} E={E} C={C} d={d} h={h}")
    rng, x, xv, ((w1, w1v), (b1, b1v), (w2, w2v), (b2, b2v)), counts = _setup(E, C, d, h, dtype, gated, 3)
    cd = torch.from_numpy(counts).to(DEV)
    o = hm.experts(x, w1, w2, b1=b1, b2=b2, counts=cd, act=ACTS[act], gated=gated, want_pre=True)
    torch.cuda.synchronize()
    ref = ox.experts(xv, w1v, b1v, w2v, b2v, counts, ACTS[act], gated, ROUND[dtype])
    for key in ("pre", "hidden", "ye"):
        check(o[key], ref[key], key)
    dye, dv = normal(rng, (E, C, d), dtype)
    g = hm.experts_bwd(dye.to(DEV), x, w1, w2, o["pre"], o["hidden"], counts=cd, act=ACTS[act], gated=gated)
    torch.cuda.synchronize()
    ref = ox.experts_bwd(dv, xv, w1v, w2v, counts, f64(o["pre"]), f64(o["hidden"]), ACTS[act], gated, ROUND[dtype])
    for key in ("dxe", "dw1", "db1", "dw2", "db2"):
        check(g[key], ref[key], key)


def _both_ways(dtype, E, C, d, h, act, gated, counts, seed):
    """Forward and backward, rows behind the counts NaN, against the oracle."""
    rng, x, xv, ((w1, w1v), (b1, b1v), (w2, w2v), (b2, b2v)), _ = _setup(E, C, d, h, dtype, gated, seed, garbage=False)
    dye, dv = normal(rng, (E, C, d), dtype)
    dye = dye.to(DEV)
    cd = None
    if counts is not None:
        cd = torch.from_numpy(counts).to(DEV)
        for e in range(E):
            x[e, counts[e]:] = float("nan")
            dye[e, counts[e]:] = float("nan")
    o = hm.experts(x, w1, w2, b1=b1, b2=b2, counts=cd, act=ACTS[act], gated=gated, want_pre=True)
    torch.cuda.synchronize()
    ref = ox.experts(xv, w1v, b1v, w2v, b2v, counts, ACTS[act], gated, ROUND[dtype])
    for key in ("pre", "hidden", "ye"):
        check(o[key], ref[key], key)
    g = hm.experts_bwd(dye, x, w1, w2, o["pre"], o["hidden"], counts=cd, act=ACTS[act], gated=gated)
    torch.cuda.synchronize()
    ref = ox.experts_bwd(dv, xv, w1v, w2v, counts, f64(o["pre"]), f64(o["hidden"]), ACTS[act], gated, ROUND[dtype])
    for key in ("dxe", "dw1", "db1", "dw2", "db2"):
        check(g[key], ref[key], key)


@pytest.mark.parametrize("full,act,gated", [(70, "gelu", False), (35, "silu", True), (30, "relu", False)])
def test_last_round_of_tiles(full, act, gated):
    """bf16 tiles of 256 x 256 in every product, with a last round that fills less than half of 256
    CUs: 280 tiles where all experts are full (of the gated first product: where half of them are),
    120 where 30 are.  The experts' second row of tiles holds 4 rows, its lower half none."""
    E, C, d, h = 70, 260, 400, 400
    counts = np.zeros(E, dtype=np.int32)
    counts[E - full:] = C
    counts[E - full:E - full + 3] = (C - 1, C - 2, C - 3) if full < E else C
    announce(f"experts_last_round bf16 E={E} C={C} d={d} h={h} full={full} {act} gated={gated}")
    _both_ways("bf16", E, C, d, h, act, gated, None if full == E else counts, 51)


@pytest.mark.parametrize("E,C,d,h,act,gated", [(16, 100, 512, 520, "silu", True), (9, 600, 512, 256, "gelu", False),
                                               (2, 600, 40, 72, "relu", True)])
def test_long_sums_in_fp32(E, C, d, h, act, gated):
    """Sums over 512 and more elements in groups of waves, in every product."""
    announce(f"experts_long f32 E={E} C={C} d={d} h={h} {act} gated={gated}")
    _both_ways("f32", E, C, d, h, act, gated, _counts(np.random.default_rng(E), E, C), 53)


@pytest.mark.parametrize("act,gated", [("gelu", False), ("silu", True)])
def test_tiles_of_128_in_fp32(act, gated):
    """512 and more tiles of 128 x 128 over 256 and more, cut at the edges, in every product."""
    E, C, d, h = 64, 256, 500, 508
    announce(f"experts_128 f32 E={E} C={C} d={d} h={h} {act} gated={gated}")
    _both_ways("f32", E, C, d, h, act, gated, _counts(np.random.default_rng(59), E, C), 59)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,h,act,gated", [(264, 520, "relu", True), (24, 264, "silu", False)])
def test_few_rows_of_many_experts(d, h, act, gated, dtype):
    """At most 32 rows per expert (and, with d = 24, of a weight gradient) and more than 256 tiles."""
    E, C = 70, 20
    announce(f"experts_few {dtype} E={E} C={C} d={d} h={h} {act} gated={gated}")
    _both_ways(dtype, E, C, d, h, act, gated, _counts(np.random.default_rng(67), E, C), 67)


def test_many_experts_and_more_tiles_than_a_list_holds():
    """1024 experts of one row, 129 tiles each: more than 256 tiles for each of 512 blocks."""
    E, C, d, h = 1024, 1, 8, 8256
    announce(f"experts_many bf16 E={E} C={C} d={d} h={h}")
    _, x, xv, ((w1, w1v), _, (w2, w2v), _), _ = _setup(E, C, d, h, "bf16", False, 57, bias=False, garbage=False)
    counts = np.ones(E, dtype=np.int32)
    counts[5] = 0
    o = hm.experts(x, w1, w2, counts=torch.from_numpy(counts).to(DEV), want_pre=True)
    torch.cuda.synchronize()
    ref = ox.experts(xv, w1v, None, w2v, None, counts, ox.RELU, False, ROUND["bf16"])
    for key in ("pre", "hidden", "ye"):
        check(o[key], ref[key], key)


def test_two_calls_at_once():
    """Two streams run the same weights on their own rows at the same time, several times."""
    E, C, d, h = 24, 200, 256, 512
    runs = []
    for seed in (61, 63):
        rng, x, _, ((w1, _), (b1, _), (w2, _), (b2, _)), counts = _setup(E, C, d, h, "bf16", True, seed)
        dye = normal(rng, (E, C, d), "bf16")[0].to(DEV)
        runs.append((x, w1, b1, w2, b2, torch.from_numpy(counts).to(DEV), dye, torch.cuda.Stream()))

    def run(x, w1, b1, w2, b2, cd, dye, _):
        o = hm.experts(x, w1, w2, b1=b1, b2=b2, counts=cd, act=hm.MOE_ACT_SILU, gated=True, want_pre=True)
        return {**o, **hm.experts_bwd(dye, x, w1, w2, o["pre"], o["hidden"], counts=cd, act=hm.MOE_ACT_SILU, gated=True)}

    alone = [run(*r) for r in runs]
    torch.cuda.synchronize()
    for _ in range(3):
        out = []
        for r in runs:
            with torch.cuda.stream(r[-1]):
                out.append(run(*r))
        torch.cuda.synchronize()
        for a, b in zip(alone, out):
            for key in a:
                assert torch.equal(a[key], b[key]), key


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_optional_arguments(dtype):
    """No counts, no biases, no pre; each gradient asked for alone equals the one of all."""
    E, C, d, h = 4, 70, 72, 136
    rng, x, xv, ((w1, w1v), _, (w2, w2v), _), _ = _setup(E, C, d, h, dtype, False, 5, bias=False, garbage=False)
    o = hm.experts(x, w1, w2, act=hm.MOE_ACT_GELU)
    assert o["pre"] is None
    ref = ox.experts(xv, w1v, None, w2v, None, None, ox.GELU, False, ROUND[dtype])
    check(o["ye"], ref["ye"], "ye")
    pre, hid, dye = (normal(rng, s, dtype)[0].to(DEV) for s in ((E, C, h), (E, C, h), (E, C, d)))
    full = hm.experts_bwd(dye, x, w1, w2, pre, hid, act=hm.MOE_ACT_SILU)
    dcode = hm.MOE_BF16 if dtype == "bf16" else hm.MOE_F32
    p = hm.experts_params(E, C, d, h, hm.MOE_ACT_SILU, False, dcode)
    ws = torch.empty((hm.moe_experts_bwd_workspace_size(p),), dtype=torch.uint8, device=DEV)
    needs = dict(dxe=("w1", "w2", "pre"), dw1=("xe", "w2", "pre"), db1=("w2", "pre"), dw2=("hidden",), db2=())
    have = dict(xe=x, w1=w1, w2=w2, pre=pre, hidden=hid)
    for key, uses in needs.items():
        out = {k: (torch.full_like(full[k], -7.0) if k == key else None) for k in full}
        a = {k: (v if k in uses else None) for k, v in have.items()}
        hm.moe_experts_bwd(p, dye, a["xe"], a["w1"], a["w2"], None, a["pre"], a["hidden"], out["dxe"], out["dw1"],
                           out["db1"], out["dw2"], out["db2"], ws)
        torch.cuda.synchronize()
        assert torch.equal(out[key], full[key]), key


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_counts_out_of_range_and_no_rows(dtype):
    E, C, d, h = 3, 20, 64, 64
    rng, x, xv, ((w1, w1v), (b1, b1v), (w2, w2v), (b2, b2v)), _ = _setup(E, C, d, h, dtype, False, 9, garbage=False)
    counts = np.array([-5, 2 ** 30, 7], dtype=np.int32)
    o = hm.experts(x, w1, w2, b1=b1, b2=b2, counts=torch.from_numpy(counts).to(DEV), want_pre=True)
    ref = ox.experts(xv, w1v, b1v, w2v, b2v, counts, ox.RELU, False, ROUND[dtype])
    for key in ("pre", "hidden", "ye"):
        check(o[key], ref[key], key)
    # no slots at all: nothing to do forward, zero gradients of the weights
    empty = torch.empty((E, 0, d), dtype=TORCH[dtype], device=DEV)
    assert hm.experts(empty, w1, w2)["ye"].shape == (E, 0, d)
    g = hm.experts_bwd(empty, empty, w1, w2, torch.empty((E, 0, h), dtype=TORCH[dtype], device=DEV),
                       torch.empty((E, 0, h), dtype=TORCH[dtype], device=DEV))
    torch.cuda.synchronize()
    assert all((g[key] == 0).all() for key in ("dw1", "db1", "dw2", "db2"))


def test_infinities_and_nans_stay_in_their_rows():
    """A row that holds an infinity or a NaN spoils itself and the weight gradients it enters,
    nothing else."""
    E, C, d, h = 2, 40, 64, 128
    rng, x, xv, ((w1, w1v), (b1, b1v), (w2, w2v), (b2, b2v)), _ = _setup(E, C, d, h, "bf16", True, 13, garbage=False)
    base = hm.experts(x, w1, w2, b1=b1, b2=b2, act=hm.MOE_ACT_SILU, gated=True, want_pre=True)
    y = x.clone()
    y[0, 3, 5] = float("inf")
    y[1, 39, 0] = float("nan")
    o = hm.experts(y, w1, w2, b1=b1, b2=b2, act=hm.MOE_ACT_SILU, gated=True, want_pre=True)
    torch.cuda.synchronize()
    keep = torch.ones((E, C), dtype=torch.bool, device=DEV)
    keep[0, 3] = keep[1, 39] = False
    for key in ("pre", "hidden", "ye"):
        assert torch.equal(o[key][keep], base[key][keep]), key
    assert not torch.isfinite(o["ye"][0, 3]).any() and torch.isnan(o["ye"][1, 39]).all()


def test_gradients_against_differences():
    """d(sum ye * dye) by central differences of the fp32 forward in directions of every input."""
    E, C, d, h = 3, 40, 64, 96
    for act, gated in (("gelu", False), ("silu", True)):
        rng, x, xv, ((w1, w1v), (b1, b1v), (w2, w2v), (b2, b2v)), counts = _setup(E, C, d, h, "f32", gated, 21, garbage=False)
        dye, dv = normal(rng, (E, C, d), "f32")
        cd = torch.from_numpy(counts).to(DEV)
        o = hm.experts(x, w1, w2, b1=b1, b2=b2, counts=cd, act=ACTS[act], gated=gated, want_pre=True)
        g = hm.experts_bwd(dye.to(DEV), x, w1, w2, o["pre"], o["hidden"], counts=cd, act=ACTS[act], gated=gated)
        args = dict(xe=xv, w1=w1v, b1=b1v, w2=w2v, b2=b2v)

        def loss(**kw):
            a = {**args, **kw}
            return (ox.experts(a["xe"], a["w1"], a["b1"], a["w2"], a["b2"], counts, ACTS[act], gated, 0.0)["ye"][0] * dv).sum()

        for key, grad in (("xe", "dxe"), ("w1", "dw1"), ("b1", "db1"), ("w2", "dw2"), ("b2", "db2")):
            v = rng.standard_normal(args[key].shape)
            step = 1e-4
            num = (loss(**{key: args[key] + step * v}) - loss(**{key: args[key] - step * v})) / (2 * step)
            terms = f64(g[grad]) * v
            # the differences are off by the third derivative times step^2 (the loss is smooth, of
            # third derivative below 100 times its gradient here) and the fp64 cancellation; the
            # gradient by its fp32 sums of at most 2 * 96 + 40 terms each
            tol = (100 * step ** 2 + 400 * ox.U32) * np.abs(terms).sum()
            assert abs(terms.sum() - num) <= tol, (act, gated, key, terms.sum(), num, tol)


def test_graph_and_streams():
    """Captured forward and backward on a side stream, replayed with eager work between, equal the
    eager results bit for bit, also after the inputs were refilled."""
    E, C, d, h = 6, 150, 256, 384
    rng, x, _, ((w1, _), (b1, _), (w2, _), (b2, _)), counts = _setup(E, C, d, h, "bf16", True, 31)
    cd = torch.from_numpy(counts).to(DEV)
    dye = normal(rng, (E, C, d), "bf16")[0].to(DEV)
    p = hm.experts_params(E, C, d, h, hm.MOE_ACT_SILU, True, hm.MOE_BF16)
    new = lambda *s, dt=torch.bfloat16: torch.empty(s, dtype=dt, device=DEV)  # noqa: E731
    b = dict(pre=new(E, C, 2 * h), hidden=new(E, C, h), ye=new(E, C, d), dxe=new(E, C, d), dw1=new(E, d, 2 * h),
             db1=new(E, 2 * h, dt=torch.float32), dw2=new(E, h, d), db2=new(E, d, dt=torch.float32))
    ws = torch.empty((hm.moe_experts_bwd_workspace_size(p),), dtype=torch.uint8, device=DEV)

    def step(st):
        hm.moe_experts(p, x, w1, b1, w2, b2, cd, b["pre"], b["hidden"], b["ye"], st)
        hm.moe_experts_bwd(p, dye, x, w1, w2, cd, b["pre"], b["hidden"], b["dxe"], b["dw1"], b["db1"], b["dw2"], b["db2"],
                           ws, st)

    def eager():
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        step(side)
        torch.cuda.current_stream().wait_stream(side)
        torch.cuda.synchronize()
        return {k: v.clone() for k, v in b.items()}

    ref = eager()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(torch.cuda.current_stream())
    for rep in range(5):
        if rep == 3:
            x.copy_(torch.randn_like(x))
            ref2 = eager()
            assert not torch.equal(ref2["ye"], ref["ye"])
            ref = ref2
        for v in b.values():
            v.fill_(-3)
        ws.fill_(255)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for k, v in b.items():
            assert torch.equal(v, ref[k]), (rep, k)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_training_step_of_a_layer(dtype):
    """gate, dispatch, experts, combine and every gradient back to x, then clipping: the layer's
    output and gradients equal the oracle's on the gate's own routing."""
    S, d, E, k, h, C = 150, 64, 6, 2, 96, 60
    rng = np.random.default_rng(41)
    x, xv = normal(rng, (S, d), dtype)
    wg, _ = normal(rng, (d, E), dtype, d ** -0.5)
    (w1, w1v), (b1, b1v), (w2, w2v), (b2, b2v) = weights(rng, E, d, h, True, dtype)
    dy, dyv = normal(rng, (S, d), dtype)
    x, wg, dy = x.to(DEV), wg.to(DEV), dy.to(DEV)
    r = ROUND[dtype]
    gt = hm.gate(hm.MOE_GATE_TOPK, k, E, C, x=x, wg=wg, normalize=1, want_logits=True)
    xe = hm.dispatch(x, gt["ids"], gt["slots"], gt["slot_src"])
    o = hm.experts(xe, w1, w2, b1=b1, b2=b2, counts=gt["counts"], act=hm.MOE_ACT_SILU, gated=True, want_pre=True)
    y = hm.combine(o["ye"], gt["ids"], gt["slots"], gt["weights"])
    dye, dw = hm.combine_bwd(dy, gt["ids"], gt["slots"], gt["slot_src"], gt["weights"], ye=o["ye"])
    g = hm.experts_bwd(dye, xe, w1, w2, o["pre"], o["hidden"], counts=gt["counts"], act=hm.MOE_ACT_SILU, gated=True)
    dx = hm.dispatch_bwd(g["dxe"], gt["ids"], gt["slots"])
    gb = hm.gate_bwd(hm.MOE_GATE_TOPK, gt["logits"], gt["ids"], dw, x=x, wg=wg, normalize=1, dx=dx, accumulate_dx=True)
    grads = [g["dw1"], g["db1"], g["dw2"], g["db2"], gb["dwg"], gb["dbias"]]
    before = [f64(t) for t in grads]
    norm = hm.clip_grads(grads, 0.5)
    torch.cuda.synchronize()
    ids, slots, w = gt["ids"].cpu().numpy(), gt["slots"].cpu().numpy(), f64(gt["weights"])
    counts = gt["counts"].cpu().numpy()
    assert (slots >= 0).any() and counts.max() <= C
    ref = ox.experts(f64(xe), w1v, b1v, w2v, b2v, counts, ox.SILU, True, r)
    check(o["ye"], ref["ye"], "ye")
    yv, ye = np.zeros((S, d)), np.zeros((S, d))
    for s in range(S):
        for q in range(k):
            if slots[s, q] >= 0:
                v, b = ref["ye"][0][ids[s, q], slots[s, q]], ref["ye"][1][ids[s, q], slots[s, q]]
                yv[s] += w[s, q] * v
                ye[s] += w[s, q] * b + 4 * ox.U32 * np.abs(w[s, q] * v)
    check(y, (yv, ye + r * (np.abs(yv) + ye)), "y")
    ref = ox.experts_bwd(f64(dye), f64(xe), w1v, w2v, counts, f64(o["pre"]), f64(o["hidden"]), ox.SILU, True, r)
    for key, v in (("dw1", before[0]), ("db1", before[1]), ("dw2", before[2]), ("db2", before[3])):
        check(torch.from_numpy(v), ref[key], key)
    total = np.sqrt(sum((v ** 2).sum() for v in before))
    assert abs(float(norm) - total) <= 2 * ox.U32 * total
    assert total > 0.5
    for t, v in zip(grads, before):
        scale = 0.5 / total
        half = (ox.U_BF16 if t.dtype == torch.bfloat16 else ox.U32) + 3 * ox.U32
        check(t, (v * scale, np.abs(v * scale) * half + 1e-40), "clipped")


def test_workspaces_of_a_call_on_another_stream():
    """What a call with stream= allocates for itself is not handed out again before it ran."""
    E, C, d, h = 4, 150, 64, 128
    rng, x, _, ((w1, _), (b1, _), (w2, _), (b2, _)), counts = _setup(E, C, d, h, "bf16", False, 71)
    cd = torch.from_numpy(counts).to(DEV)
    pre, hid, dye = (normal(rng, s, "bf16")[0].to(DEV) for s in ((E, C, h), (E, C, h), (E, C, d)))
    ref = hm.experts_bwd(dye, x, w1, w2, pre, hid, counts=cd)
    grads = [ref["db1"], ref["db2"]]
    total, _ = hm.grad_norm(grads)
    side = torch.cuda.Stream()
    size = hm.moe_experts_bwd_workspace_size(hm.experts_params(E, C, d, h, 0, False, hm.MOE_BF16))
    for stream in (side, side.cuda_stream):
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            torch.cuda._sleep(20_000_000)  # the calls below are still waiting when they return
        out = hm.experts_bwd(dye, x, w1, w2, pre, hid, counts=cd, stream=stream)
        norm, sumsq = hm.grad_norm(grads, stream=stream)
        junk = [torch.full((n,), 255, dtype=torch.uint8, device=DEV) for n in (size, size, 8, 16, 512, 4096)]
        torch.cuda.synchronize()
        for key in ref:
            assert torch.equal(out[key], ref[key]), key
        assert torch.equal(norm, total) and len(junk) == 6


def test_bias_gradient_of_more_row_ranges_than_a_grid_dimension():
    """65537 ranges of 256 rows; the sums of a few rows of small whole numbers are exact."""
    C = 65536 * 256 + 100
    dye = torch.zeros((1, C, 8), dtype=torch.bfloat16, device=DEV)
    for i, row in enumerate((0, 255, 70_000, 65536 * 256 - 1, 65536 * 256, C - 1)):
        dye[0, row] = 2.0 ** i
    p = hm.experts_params(1, C, 8, 8, hm.MOE_ACT_RELU, False, hm.MOE_BF16)
    ws = torch.empty((hm.moe_experts_bwd_workspace_size(p),), dtype=torch.uint8, device=DEV)
    db2 = torch.full((1, 8), -1.0, device=DEV)
    hm.moe_experts_bwd(p, dye, None, None, None, None, None, None, None, None, None, None, db2, ws)
    torch.cuda.synchronize()
    assert torch.equal(db2, torch.full_like(db2, 63.0))
