"""Embedding rows and their gradient against the fp64 oracle: types, widths, padding, ids of
every spread, both ways of sorting, runs that cross chunks, accumulation, and repeats."""

import numpy as np
import pytest
import torch

import paper_2203_14685_amd as hm
from oracle import embed as oe

from _experts import DEV, ROUND, TORCH, announce, check, f64, normal

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True, scope="module")
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    hm.load()
    yield


def _ids(rng, T, V, kind):
    if kind == "one":
        return np.full(T, V - 1, dtype=np.int32)
    if kind == "even":
        return rng.integers(0, V, T).astype(np.int32)
    if kind == "order":  # runs of equal ids, descending
        return np.sort(rng.integers(0, V, T))[::-1].astype(np.int32).copy()
    p = np.arange(1, V + 1, dtype=np.float64) ** -1.2
    ids = rng.choice(V, T, p=p / p.sum()).astype(np.int32)
    pad = rng.random(T) < 0.1
    ids[pad] = rng.choice(np.array([-1, V, V + 5, 2 ** 31 - 1, -2 ** 31], dtype=np.int64), int(pad.sum())).astype(np.int32)
    return ids


SIZES = [(1, 1, 8), (1, 300, 64), (3, 2, 72), (63, 500, 264), (64, 7, 128), (257, 1000, 8), (1000, 40, 520), (2049, 3, 136),
         (700, 5000, 1032)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,V,d", SIZES + [(9000, 100, 24), (4100, 30, 4096)])
def test_rows(T, V, d, dtype):
    announce(f"embed {dtype} T={T} V={V} d={d}")
    rng = np.random.default_rng(T + V)
    table, tv = normal(rng, (V, d), dtype)
    ids = _ids(rng, T, V, "zipf")
    for scale in (1.0, d ** 0.5):
        y = hm.embed(torch.from_numpy(ids).to(DEV), table.to(DEV), scale)
        check(y, oe.embed(ids, tv, float(np.float32(scale)), ROUND[dtype]), "y")
    inside = (ids >= 0) & (ids < V)
    y = hm.embed(torch.from_numpy(ids).to(DEV), table.to(DEV))
    assert np.array_equal(f64(y)[inside], tv[ids[inside]])  # a copy
    assert not torch.signbit(hm.embed(torch.from_numpy(ids).to(DEV), table.to(DEV), -1.0)).cpu()[torch.from_numpy(~inside)].any()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,V,d", SIZES)
def test_gradient(T, V, d, dtype):
    for kind in ("zipf", "even", "one", "order"):
        for accumulate in (False, True):
            announce(f"embed_bwd {dtype} T={T} V={V} d={d} {kind} accumulate={accumulate}")
            rng = np.random.default_rng(T + V)
            dy, dv = normal(rng, (T, d), dtype)
            there, hv = normal(rng, (V, d), dtype)
            ids = _ids(rng, T, V, kind)
            out = torch.cat([there.to(DEV).reshape(-1), torch.full((64,), 7.0, dtype=TORCH[dtype], device=DEV)])
            if not accumulate:
                out[:V * d] = float("nan")
            grad = out[:V * d].view(V, d)
            idt = torch.from_numpy(ids).to(DEV)
            hm.embed_bwd(dy.to(DEV), idt, V, scale=1.5, dtable=grad, accumulate=accumulate)
            check(grad, oe.embed_bwd(dv, ids, V, 1.5, hv if accumulate else None, ROUND[dtype]), "dtable")
            assert (out[V * d:] == 7).all()
            if not accumulate:
                assert torch.equal(hm.embed_bwd(dy.to(DEV), idt, V, scale=1.5), grad)  # repeats bit for bit


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,V,d", [(8192, 50, 8), (8193, 200, 16), (20000, 70000, 8), (33000, 1 << 17, 72), (12345, 17000000, 8),
                                   (50000, 255, 1032), (70000, 256, 40)])
def test_gradient_of_many_tokens(T, V, d, dtype):
    """On either side of the length where sorting changes; one, two, three and four digits."""
    for kind in ("zipf", "one") if V < 10 ** 6 else ("even",):
        announce(f"embed_bwd {dtype} T={T} V={V} d={d} {kind}")
        rng = np.random.default_rng(T)
        dy, dv = normal(rng, (T, d), dtype)
        ids = _ids(rng, T, V, kind)
        grad = hm.embed_bwd(dy.to(DEV), torch.from_numpy(ids).to(DEV), V)
        if V < 10 ** 6:
            check(grad, oe.embed_bwd(dv, ids, V, 1.0, None, ROUND[dtype]), "dtable")
        else:
            rows, back = np.unique(ids, return_inverse=True)
            value, bound = oe.embed_bwd(dv, back.astype(np.int64), len(rows), 1.0, None, ROUND[dtype])
            check(grad[torch.from_numpy(rows.astype(np.int64)).to(DEV)], (value, bound), "rows in use")
            grad[torch.from_numpy(rows.astype(np.int64)).to(DEV)] = 0
            assert not grad.any()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_order_of_a_sum_is_the_tokens(dtype):
    """A large value, ones, and its negative: every other order of 3000 equal ids gives another sum."""
    T, d = 3000, 8
    dy = torch.ones(T, d)
    dy[0], dy[-1] = 2.0 ** 30, -2.0 ** 30
    ids = torch.zeros(T, dtype=torch.int32)
    runs = [hm.embed_bwd(dy.to(TORCH[dtype]).to(DEV), ids.to(DEV), 4) for _ in range(3)]
    assert torch.equal(runs[0], runs[1]) and torch.equal(runs[0], runs[2])
    # the same tokens among others: the same chunks, or not, but never beyond the bound
    value, bound = oe.embed_bwd(dy.double().numpy(), ids.numpy(), 4, 1.0, None, ROUND[dtype])
    check(runs[0], (value, bound), "dtable")


def test_padding_rows_are_not_read():
    T, V, d = 500, 20, 64
    for ids in (np.full(T, -1, dtype=np.int32), np.where(np.arange(T) % 3 == 0, V, np.arange(T) % V).astype(np.int32)):
        dy = torch.randn(T, d, device=DEV)
        dy[torch.from_numpy((ids < 0) | (ids >= V)).to(DEV)] = float("nan")
        grad = hm.embed_bwd(dy, torch.from_numpy(ids).to(DEV), V)
        assert torch.isfinite(grad).all()
        there = torch.full((V, d), 3.0, device=DEV)
        hm.embed_bwd(dy, torch.from_numpy(ids).to(DEV), V, dtable=there, accumulate=True)
        assert torch.isfinite(there).all()


def test_no_tokens():
    y = hm.embed(torch.empty(0, dtype=torch.int32, device=DEV), torch.ones(5, 8, device=DEV))
    assert y.shape == (0, 8)
    dy, ids = torch.empty(0, 8, device=DEV), torch.empty(0, dtype=torch.int32, device=DEV)
    assert not hm.embed_bwd(dy, ids, 5).any()
    there = torch.ones(5, 8, device=DEV)
    assert (hm.embed_bwd(dy, ids, 5, dtable=there, accumulate=True) == 1).all()


@pytest.mark.parametrize("T", [300, 10000])
def test_graph_and_streams(T):
    V, d = 400, 72
    rng = np.random.default_rng(T)
    dy = normal(rng, (T, d), "bf16")[0].to(DEV)
    ids = torch.from_numpy(_ids(rng, T, V, "zipf")).to(DEV)
    want = hm.embed_bwd(dy, ids, V)
    params = hm.embed_params(T, V, d, hm.MOE_BF16)
    ws = torch.empty(hm.moe_embed_bwd_workspace_size(params), dtype=torch.uint8, device=DEV)
    out = torch.empty_like(want)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        hm.moe_embed_bwd(params, dy, ids, out, ws)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        hm.moe_embed_bwd(params, dy, ids, out, ws)
    keep_dy, keep_ids = dy.clone(), ids.clone()
    for i in range(4):
        out.fill_(float("nan"))
        ws.fill_(0xff)
        dy.copy_(keep_dy if i % 2 == 0 else keep_dy.flip(0))
        ids.copy_(keep_ids if i % 2 == 0 else keep_ids.flip(0))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want if i % 2 == 0 else hm.embed_bwd(dy, ids, V)), i
    dy.copy_(keep_dy)
    ids.copy_(keep_ids)
    torch.cuda.synchronize()
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    a, b = hm.embed_bwd(dy, ids, V, stream=s1), hm.embed_bwd(dy, ids, V, stream=s2)
    torch.cuda.synchronize()
    assert torch.equal(a, want) and torch.equal(b, want)
