"""Rows, weights and gradients whose offsets pass 2^31 elements and 2^32 bytes.  A few rows at the
ends of each expert hold values, all others zeros, which add nothing: the oracle sees those rows alone."""

import math

import numpy as np
import pytest
import torch

import paper_2203_14685_amd as hm
from oracle import experts as ox

from _experts import DEV, ROUND, TORCH, announce, check, f64, normal, weights

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True, scope="module")
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    hm.load()
    yield
    torch.cuda.empty_cache()


@pytest.mark.parametrize("dtype,C,d,h", [("bf16", 540_000, 2048, 2056), ("f32", 270_000, 2052, 2048)])
def test_rows(dtype, C, d, h):
    announce(f"experts long rows {dtype} C={C} d={d} h={h}")
    E, elt = 2, 2 if dtype == "bf16" else 4
    assert E * C * min(d, h) * elt > 2 ** 32 and (dtype == "f32" or E * C * d > 2 ** 31)
    rng = np.random.default_rng(5)
    at = torch.tensor([0, 1, 63, 64, C // 2 + 1, C - 300, C - 65, C - 3, C - 2])
    counts = np.array([C, C - 2], dtype=np.int32)  # the last row of the second expert lies behind its count
    small = np.array([len(at), len(at) - 1], dtype=np.int32)
    (w1, w1v), _, (w2, w2v), _ = weights(rng, E, d, h, False, dtype, False)
    few = {key: normal(rng, (E, len(at), d), dtype) for key in ("xe", "dye")}
    rows = {}
    for key, (t, _) in few.items():
        rows[key] = torch.zeros((E, C, d), dtype=TORCH[dtype], device=DEV)
        rows[key][:, at.to(DEV)] = t.to(DEV)
        rows[key][1, counts[1]:] = float("nan")
    cd = torch.from_numpy(counts).to(DEV)
    o = hm.experts(rows["xe"], w1, w2, counts=cd, act=hm.MOE_ACT_SILU, want_pre=True)
    torch.cuda.synchronize()
    ref = ox.experts(few["xe"][1], w1v, None, w2v, None, small, ox.SILU, False, ROUND[dtype])
    got = {key: v[:, at.to(DEV)] for key, v in o.items()}
    for key in ("pre", "hidden", "ye"):
        check(got[key], ref[key], key)
        total = o[key].ne(0).sum(dim=(1, 2)).cpu()  # no other row has values
        assert torch.equal(total, got[key].ne(0).sum(dim=(1, 2)).cpu()), key
    g = hm.experts_bwd(rows["dye"], rows["xe"], w1, w2, o["pre"], o["hidden"], counts=cd, act=hm.MOE_ACT_SILU)
    torch.cuda.synchronize()
    ref = ox.experts_bwd(few["dye"][1], few["xe"][1], w1v, w2v, small, f64(got["pre"]), f64(got["hidden"]), ox.SILU, False,
                         ROUND[dtype])
    check(g["dxe"][:, at.to(DEV)], ref["dxe"], "dxe")
    assert torch.equal(g["dxe"].ne(0).sum(dim=(1, 2)), g["dxe"][:, at.to(DEV)].ne(0).sum(dim=(1, 2)))
    for key in ("dw1", "db1", "dw2", "db2"):
        check(g[key], ref[key], key)


@pytest.mark.parametrize("dtype,E,d,h", [("bf16", 270, 2048, 4096), ("f32", 140, 2048, 4096)])
def test_weights_of_the_layer_for_few_tokens(dtype, E, d, h):
    announce(f"token_layer long weights {dtype} E={E} d={d} h={h}")
    S, k = 5, 2
    assert (E - 1) * d * h * (2 if dtype == "bf16" else 4) > 2 ** 32 and (dtype == "f32" or (E - 1) * d * h > 2 ** 31)
    rng = np.random.default_rng(7)
    chosen = [0, 1, E // 2, E - 2, E - 1]
    (w1s, w1v), _, (w2s, w2v), _ = weights(rng, len(chosen), d, h, False, dtype, False)
    w1 = torch.zeros((E, d, h), dtype=TORCH[dtype], device=DEV)
    w2 = torch.zeros((E, h, d), dtype=TORCH[dtype], device=DEV)
    for i, e in enumerate(chosen):
        w1[e], w2[e] = w1s[i], w2s[i]
    x, xv = normal(rng, (S, d), dtype)
    pick = rng.integers(0, len(chosen), (S, k))
    pick[:, 0] = np.arange(S)
    ids = torch.from_numpy(np.array(chosen, dtype=np.int32)[pick]).to(DEV)
    w, wv = normal(rng, (S, k), "f32")
    o = hm.token_layer(x.to(DEV), w1, w2, act=hm.MOE_ACT_GELU, ids=ids, weights=w.to(DEV))
    torch.cuda.synchronize()
    check(o["y"], ox.token_layer(xv, pick, wv, w1v, None, w2v, None, ox.GELU, False, ROUND[dtype]), "y")


def test_gradients():
    n = 2 ** 31 + 70_001
    announce(f"clip of {n} values")
    g = torch.zeros((n,), dtype=torch.bfloat16, device=DEV)
    at = torch.tensor([0, 1, 8191, 8192, 2 ** 31 - 1, 2 ** 31, n - 2, n - 1], device=DEV)
    g[at] = torch.tensor([3.0, -1, 2, 4, -5, 6, 7, -8], device=DEV, dtype=torch.bfloat16)
    norm, sumsq = hm.grad_norm([g])
    assert float(sumsq) == 204.0 and abs(float(norm) - math.sqrt(204.0)) <= 2 ** -23 * 15
    before = g[at].double()
    hm.clip_grads([g], 1.0)
    torch.cuda.synchronize()
    v = before / math.sqrt(204.0)
    assert ((g[at].double() - v).abs() <= (2.0 ** -8 + 3 * 2.0 ** -24) * v.abs()).all()
    assert int(g.ne(0).sum()) == len(at)


def _product(a, b, a_err=None):
    """a @ b in 64 bits and how far fp32 sums of it may be off (the oracle's bound)."""
    a_abs, b_abs = a.abs(), b.abs()
    err = (a.shape[-1] + 2) * ox.U32 * (a_abs @ b_abs)
    return a @ b, err if a_err is None else err + a_err @ b_abs


def _near(got, value, err, r, what):
    bad = ~((got.double() - value).abs() <= err + r * (value.abs() + err))
    assert not bad.any(), (what, int(bad.sum()), torch.nonzero(bad)[0].tolist())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,h", [(8, 2 ** 20), (2 ** 20, 8)])
def test_widest_rows(d, h, dtype):
    """Widths of 2^20, gated relu, 258 of 260 rows in use: tiles of the most rows on the longest ones."""
    C, n, r = 260, 258, ROUND[dtype]
    announce(f"experts widest rows {dtype} d={d} h={h}")
    gen = torch.Generator(device=DEV)
    gen.manual_seed(9)

    def new(*shape, scale=1.0):
        return (torch.randn(shape, generator=gen, device=DEV) * scale).to(TORCH[dtype])

    w1, w2 = new(1, d, 2 * h, scale=d ** -0.5), new(1, h, d, scale=h ** -0.5)
    xe, dye = new(1, C, d), new(1, C, d)
    xe[0, n:] = dye[0, n:] = float("nan")
    cd = torch.tensor([n], dtype=torch.int32, device=DEV)
    o = hm.experts(xe, w1, w2, counts=cd, gated=True, want_pre=True)
    g = hm.experts_bwd(dye, xe, w1, w2, o["pre"], o["hidden"], counts=cd, gated=True)
    torch.cuda.synchronize()
    for t in (o["pre"], o["hidden"], o["ye"], g["dxe"]):
        assert (t[0, n:] == 0).all()
    x, dy, v1, v2 = xe[0, :n].double(), dye[0, :n].double(), w1[0].double(), w2[0].double()
    pre, pe = _product(x, v1)
    _near(o["pre"][0, :n], pre, pe, r, "pre")
    a, u, ae, ue = pre[:, :h].clamp(min=0), pre[:, h:], pe[:, :h], pe[:, h:]
    hid, he = a * u, ae * u.abs() + (a + ae) * ue + ox.U32 * (a * u).abs()
    _near(o["hidden"][0, :n], hid, he, r, "hidden")
    hid, pre = o["hidden"][0, :n].double(), o["pre"][0, :n].double()  # as the other products read them
    _near(o["ye"][0, :n], *_product(hid, v2), r, "ye")
    a, u, on = pre[:, :h].clamp(min=0), pre[:, h:], (pre[:, :h] > 0).double()
    dh, dhe = _product(dy, v2.t())
    dpre = torch.cat([dh * u * on, dh * a], dim=1)
    dpe = torch.cat([dhe * u.abs() * on, dhe * a], dim=1) + 2 * ox.U32 * dpre.abs()
    stored = dpe + r * (dpre.abs() + dpe)
    _near(g["dxe"][0, :n], *_product(dpre, v1.t(), stored), r, "dxe")
    err = (n + 2) * ox.U32 * (x.t().abs() @ dpre.abs()) + x.t().abs() @ stored
    _near(g["dw1"][0], x.t() @ dpre, err, r, "dw1")
    _near(g["db1"][0], dpre.sum(dim=0), dpe.sum(dim=0) + (n + 2) * ox.U32 * dpre.abs().sum(dim=0), 0.0, "db1")
    _near(g["dw2"][0], *_product(hid.t(), dy), r, "dw2")
    _near(g["db2"][0], dy.sum(dim=0), (n + 2) * ox.U32 * dy.abs().sum(dim=0), 0.0, "db2")
