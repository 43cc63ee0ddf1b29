"""The layer for few tokens against the fp64 oracle on the routing it returns, and that
routing against the gate's: types, activations, every gate, one token to the most,
more choices than experts and fewer, one expert taken by all, given routing with
padding, graphs and streams."""

import numpy as np
import pytest
import torch

import paper_2203_14685_amd as hm
from oracle import experts as ox

from _experts import ACTS, DEV, ROUND, announce, check, f64, normal, weights

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True, scope="module")
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    hm.load()
    yield


def _layer(S, d, E, k, h, act, gated, dtype, seed, experts_bias=True, **gate):
    rng = np.random.default_rng(seed)
    x, xv = normal(rng, (S, d), dtype)
    w = weights(rng, E, d, h, gated, dtype, experts_bias)
    (w1, w1v), (b1, b1v), (w2, w2v), (b2, b2v) = w
    o = hm.token_layer(x.to(DEV), w1, w2, b1=b1, b2=b2, act=ACTS[act], gated=gated, k=k, **gate)
    torch.cuda.synchronize()
    ref = ox.token_layer(xv, o["ids"].cpu().numpy(), f64(o["weights"]), w1v, b1v, w2v, b2v, ACTS[act], gated, ROUND[dtype])
    check(o["y"], ref, f"y {act} gated={gated}")
    return x.to(DEV), o


def _same_choice(o, g, x, wg, noise=None, temperature=0.0):
    """ids and weights against the gate's on the same inputs.  Each side's fp32 logits are off by
    at most delta = (d + 4) u sum |x| |wg| (and two more roundings with noise and temperature), so
    where the experts chosen differ their logits lie within 2 delta, and a weight, whose
    logarithm has slope at most 2 in the logits, is off by 4 delta relative, plus the
    exponentials' 1e-5."""
    xv, wv = f64(x), f64(wg)
    logits, mag = xv @ wv, np.abs(xv) @ np.abs(wv)
    if temperature:
        n = 0 if noise is None else f64(noise)
        logits, mag = (logits + n) / temperature, (mag + np.abs(n)) / temperature
    delta = (x.shape[1] + 6) * ox.U32 * mag.max(axis=1, keepdims=True)
    a, b = o["ids"].cpu().numpy(), g["ids"].cpu().numpy()
    la, lb = np.take_along_axis(logits, a, 1), np.take_along_axis(logits, b, 1)
    assert ((a == b) | (np.abs(la - lb) <= 2 * delta)).all()
    wa, wb = f64(o["weights"]), f64(g["weights"])
    assert (np.abs(wa - wb) <= wb * (4 * delta + 1e-5)).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("S,d,E,k,h", [
    (1, 64, 8, 2, 128), (1, 8, 1, 1, 8), (2, 72, 64, 8, 40), (3, 264, 5, 3, 1048), (16, 128, 4, 1, 72),
    (17, 136, 6, 2, 264), (33, 64, 3, 3, 136), (100, 200, 16, 4, 72), (256, 40, 7, 2, 64), (7, 1032, 300, 4, 24),
    (19, 264, 200, 8, 40), (5, 72, 256, 5, 40), (40, 4096, 136, 2, 8), (64, 64, 64, 1, 64)])
def test_learned_gates(S, d, E, k, h, dtype):
    for i, (act, gated) in enumerate([("silu", True), ("gelu", False), ("relu", True)]):
        announce(f"token_layer {dtype} S={S} d={d} E={E} k={k} h={h} {act} gated={gated}")
        rng = np.random.default_rng(i)
        wg = normal(rng, (d, E), dtype, d ** -0.5)[0].to(DEV)
        x, o = _layer(S, d, E, k, h, act, gated, dtype, 5 * i + S, experts_bias=i != 1, wg=wg, normalize=i % 2)
        _same_choice(o, hm.gate(hm.MOE_GATE_TOPK, k, E, S, x=x, wg=wg, normalize=i % 2), x, wg)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_other_gates(dtype):
    for E in (12, 24, 96):
        _other_gates(dtype, E)


def _other_gates(dtype, E):
    S, d, h = 20, 128, 64
    rng = np.random.default_rng(3)
    wg = normal(rng, (d, E), dtype, d ** -0.5)[0].to(DEV)
    noise = normal(rng, (S, E), "f32")[0].to(DEV)
    tok = torch.from_numpy(rng.integers(0, 1000, S).astype(np.int32)).to(DEV)
    table = torch.from_numpy(rng.integers(0, E, 1000).astype(np.int32)).to(DEV)
    for k, kw in [(3, dict(kind=hm.MOE_GATE_KTOP1, wg=wg)), (2, dict(kind=hm.MOE_GATE_HTOPK, wg=wg, groups=3, normalize=1)),
                  (2, dict(kind=hm.MOE_GATE_TOPK, wg=wg, noise=noise, temperature=0.5)),
                  (1, dict(kind=hm.MOE_GATE_HASH, token_ids=tok, hash_seed=9)),
                  (1, dict(kind=hm.MOE_GATE_HASH, token_ids=tok, hash_table=table))]:
        announce(f"token_layer {dtype} gate {kw['kind']}")
        x, o = _layer(S, d, E, k, h, "silu", False, dtype, 7, **kw)
        kind = kw.pop("kind")
        g = hm.gate(kind, k, E, S, x=None if kind == hm.MOE_GATE_HASH else x, **kw)
        if kind == hm.MOE_GATE_HASH:
            assert torch.equal(o["ids"], g["ids"]) and torch.equal(o["weights"], g["weights"])
        else:
            _same_choice(o, g, x, wg, kw.get("noise"), kw.get("temperature", 0.0))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("S,E,k", [(5, 64, 2), (70, 8, 4), (256, 2, 2), (1, 4, 1)])
def test_given_routing_with_padding(S, E, k, dtype):
    """Ids outside the experts add nothing; a row without any gives zeros; one expert may come
    twice in a row, and all rows may choose one."""
    d, h = 72, 200
    rng = np.random.default_rng(S)
    w = normal(rng, (S, k), "f32")[0].to(DEV)
    for case in ("mixed", "one", "none"):
        announce(f"token_layer routed {dtype} S={S} E={E} k={k} {case}")
        ids = rng.integers(-1, E + 1, (S, k)).astype(np.int32)
        if case == "one":
            ids[:] = E - 1
        if case == "none":
            ids[:] = -1
            ids[:, -1] = 2 ** 31 - 1
        ids_d = torch.from_numpy(ids).to(DEV)
        _, o = _layer(S, d, E, k, h, "gelu", True, dtype, S + k, ids=ids_d, weights=w)
        assert torch.equal(o["ids"].cpu(), torch.from_numpy(ids))
        if case == "none":
            assert (o["y"] == 0).all()


def test_padding_row_ignores_its_values():
    """A padded token's row may hold anything."""
    S, d, E, k, h = 9, 64, 4, 2, 64
    rng = np.random.default_rng(1)
    (w1, _), _, (w2, _), _ = weights(rng, E, d, h, False, "bf16", False)
    x = normal(rng, (S, d), "bf16")[0].to(DEV)
    ids = torch.from_numpy(rng.integers(0, E, (S, k)).astype(np.int32)).to(DEV)
    w = torch.ones((S, k), device=DEV)
    ids[4] = -1
    a = hm.token_layer(x, w1, w2, ids=ids, weights=w)["y"]
    x[4] = float("nan")
    w[4] = float("nan")
    b = hm.token_layer(x, w1, w2, ids=ids, weights=w)["y"]
    torch.cuda.synchronize()
    assert torch.equal(a, b) and (b[4] == 0).all()


def test_no_tokens():
    (w1, _), _, (w2, _), _ = weights(np.random.default_rng(1), 4, 64, 64, False, "bf16", False)
    wg = torch.zeros((64, 4), dtype=torch.bfloat16, device=DEV)
    o = hm.token_layer(torch.empty((0, 64), dtype=torch.bfloat16, device=DEV), w1, w2, wg=wg, k=2)
    assert o["y"].shape == (0, 64) and o["ids"].shape == (0, 2)


@pytest.mark.parametrize("S,E,k", [(2, 32, 2), (40, 8, 2)])
def test_graph_and_streams(S, E, k):
    d, h = 256, 512
    rng = np.random.default_rng(S)
    x = normal(rng, (S, d), "bf16")[0].to(DEV)
    wg = normal(rng, (d, E), "bf16", d ** -0.5)[0].to(DEV)
    (w1, _), (b1, _), (w2, _), (b2, _) = weights(rng, E, d, h, True, "bf16")
    p = hm.token_layer_params(S, d, E, k, h, hm.MOE_GATE_TOPK, hm.MOE_ACT_SILU, True, hm.MOE_BF16, 1)
    ids = torch.empty((S, k), dtype=torch.int32, device=DEV)
    w = torch.empty((S, k), device=DEV)
    y = torch.empty_like(x)
    ws = torch.empty((hm.moe_token_layer_workspace_size(p),), dtype=torch.uint8, device=DEV)

    def step(st):
        hm.moe_token_layer(p, x, wg, None, None, None, None, w1, b1, w2, b2, ids, w, y, ws, st)

    def eager():
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        step(side)
        torch.cuda.current_stream().wait_stream(side)
        torch.cuda.synchronize()
        return y.clone(), ids.clone()

    ref = eager()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(torch.cuda.current_stream())
    for rep in range(6):
        if rep == 3:
            x.copy_(torch.randn_like(x))
            ref = eager()
        y.fill_(-3)
        ids.fill_(-3)
        ws.fill_(255)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, ref[0]) and torch.equal(ids, ref[1]), rep
