"""The operators around the layer together, as a model's block uses them: a training step
from token ids to the clipped gradient of the embedding table, and the same layer served
in 8-bit integers through slots and token by token."""

import math

import numpy as np
import pytest
import torch

import paper_2203_14685_amd as hm
from oracle import int8 as oi

from _experts import ACTS, DEV, ROUND, announce, check, f64, normal, weights

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True, scope="module")
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    hm.load()
    yield


def _plain_step(ids, table, wg, w, dy, masks, E, k, C, scale, keep, chosen):
    """The step in fp64 by torch's gradients, the choices and the dropped elements given."""
    leaves = [t.double().requires_grad_(True) for t in (table, wg, *w)]
    tb, g, w1, b1, w2, b2 = leaves
    S = ids.numel()
    inside = (ids >= 0) & (ids < table.shape[0])
    x = torch.where(inside[:, None], tb[ids.clamp(0, table.shape[0] - 1).long()] * scale, 0.0)
    x = x * masks[0]
    at = torch.gather(x @ g, 1, chosen.long())
    weight = torch.softmax(at, dim=1)
    y = torch.zeros_like(x)
    for s in range(S):
        for r in range(k):
            c = int(keep[s, r])
            if c >= 0:
                e = int(chosen[s, r])
                pre = x[s] @ w1[e] + b1[e]
                hid = torch.nn.functional.silu(pre) * masks[1][e, c]
                y[s] = y[s] + weight[s, r] * (hid @ w2[e] + b2[e])
    out = x + y * masks[2]
    (out * dy).sum().backward()
    return out.detach(), [t.grad for t in leaves]


def test_training_step():
    """fp32: every gradient of the step against torch's in 64 bits."""
    rng = np.random.default_rng(4)
    S, V, d, E, k, h, scale, p = 96, 40, 32, 4, 2, 48, math.sqrt(32), 0.25
    C = 40  # some choices are dropped
    announce("training step: embed, dropout, gate, experts with dropout, combine, residual dropout and back")
    ids = rng.integers(0, V, S).astype(np.int32)
    ids[5] = -1
    ids = torch.from_numpy(ids).to(DEV)
    table, _ = normal(rng, (V, d), "f32", d ** -0.5)
    table = table.to(DEV)
    wg = normal(rng, (d, E), "f32", d ** -0.5)[0].to(DEV)
    (w1, _), (b1, _), (w2, _), (b2, _) = weights(rng, E, d, h, False, "f32")
    dy = normal(rng, (S, d), "f32")[0].to(DEV)
    m_in, m_hid, m_out = (hm.dropout_mask(p, 1234, i << 40) for i in range(3))

    def step():
        x = hm.dropout(hm.embed(ids, table, scale), m_in)
        g = hm.gate(hm.MOE_GATE_TOPK, k, E, C, x=x, wg=wg, normalize=1, want_logits=True)
        xe = hm.dispatch(x, g["ids"], g["slots"], g["slot_src"])
        o = hm.experts(xe, w1, w2, b1=b1, b2=b2, counts=g["counts"], act=ACTS["silu"], want_pre=True, dropout=m_hid)
        y = hm.combine(o["ye"], g["ids"], g["slots"], g["weights"])
        out = hm.dropout(y, m_out, residual=x)
        # back
        dc = hm.dropout(dy, m_out)
        dye, dw = hm.combine_bwd(dc, g["ids"], g["slots"], g["slot_src"], g["weights"], ye=o["ye"])
        e = hm.experts_bwd(dye, xe, w1, w2, o["pre"], o["hidden"], counts=g["counts"], act=ACTS["silu"], dropout=m_hid)
        dx = hm.dispatch_bwd(e["dxe"], g["ids"], g["slots"])
        gb = hm.gate_bwd(hm.MOE_GATE_TOPK, g["logits"], g["ids"], dw, x=x, wg=wg, normalize=1, dx=dx, accumulate_dx=True)
        dx = hm.dropout(gb["dx"] + dy, m_in)  # dy: through the residual
        dt = hm.embed_bwd(dx, ids, V, scale)
        return g, out, [dt, gb["dwg"], e["dw1"], e["db1"], e["dw2"], e["db2"]]

    g, out, grads = step()
    ones = torch.ones(S, d, device=DEV)
    masks = [hm.dropout(ones, m_in).double().cpu(), hm.dropout(torch.ones(E, C, h, device=DEV), m_hid).double().cpu(),
             hm.dropout(ones, m_out).double().cpu()]
    want, wgrads = _plain_step(ids.cpu(), table.cpu(), wg.cpu(), [t.cpu() for t in (w1, b1, w2, b2)], dy.double().cpu(), masks, E, k,
                               C, scale, g["slots"].cpu(), g["ids"].cpu())
    assert (g["slots"] < 0).any() and (g["slots"] >= 0).any()
    # eight products of at most 96 terms behind each other in fp32, errors of about 2^-24 sqrt(96) each
    # on the average, 2^-24 * 96 * 8 at most, relative to the sizes of their terms
    tol = 2.0 ** -24 * 96 * 8
    assert np.linalg.norm(f64(out) - f64(want)) <= tol * np.linalg.norm(f64(want))
    for name, a, b in zip(("dtable", "dwg", "dw1", "db1", "dw2", "db2"), grads, wgrads):
        assert np.linalg.norm(f64(a) - f64(b)) <= tol * np.linalg.norm(f64(b)), name
    total = math.sqrt(sum(float(t.double().square().sum()) for t in wgrads))
    norm = hm.clip_grads(grads, 0.5 * total)
    assert abs(float(norm) - total) <= 1e-4 * total
    again = step()[2]
    hm.clip_grads(again, 0.5 * total)
    for a, b in zip(again, grads):
        assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_serving_through_slots_and_token_by_token(dtype):
    rng = np.random.default_rng(8)
    S, V, d, E, k, h = 50, 300, 64, 6, 2, 96
    announce(f"serving in 8 bits {dtype}")
    ids = torch.from_numpy(rng.integers(0, V, S).astype(np.int32)).to(DEV)
    table = normal(rng, (V, d), dtype)[0].to(DEV)
    wg = normal(rng, (d, E), dtype, d ** -0.5)[0].to(DEV)
    (w1, _), (b1, _), (w2, _), (b2, _) = weights(rng, E, d, h, True, dtype)
    q1, s1 = hm.quantize_weights(w1)
    q2, s2 = hm.quantize_weights(w2)
    x = hm.embed(ids, table)
    g = hm.gate(hm.MOE_GATE_TOPK, k, E, S, x=x, wg=wg, normalize=1)
    kw = dict(b1=b1, b2=b2, act=ACTS["silu"], gated=True)
    ye = hm.experts_int8(hm.dispatch(x, g["ids"], g["slots"], g["slot_src"]), q1, s1, q2, s2, counts=g["counts"], **kw)
    y = hm.combine(ye, g["ids"], g["slots"], g["weights"])
    t = hm.token_layer_int8(x, q1, s1, q2, s2, ids=g["ids"], weights=g["weights"], **kw)["y"]
    vals = [f64(v) for v in (q1, s1, b1, q2, s2, b2)]
    value, bound = oi.token_layer(f64(x), g["ids"].cpu().numpy(), f64(g["weights"]), *vals, ACTS["silu"], True, ROUND[dtype])
    check(t, (value, bound), "y token by token")
    # through slots every expert's result is rounded too
    r = ROUND[dtype]
    mag = sum(np.abs(f64(g["weights"])[:, i:i + 1] * f64(ye)[g["ids"].cpu().numpy()[:, i], g["slots"].cpu().numpy()[:, i]]) for i in range(k))
    check(y, (value, bound + (r + 2.0 ** -22) * mag * (1 + r)), "y through slots")
