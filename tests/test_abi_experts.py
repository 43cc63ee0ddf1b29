"""CPU checks of the expert-network, token-layer and gradient-norm entry points: struct
layouts, workspace sizes, and that bad arguments are refused before any HIP call
(the stand-in addresses are never dereferenced); and the oracle against plain sums."""

import ctypes
import os
import re

import numpy as np
import pytest
import torch

import paper_2203_14685_amd as hm
from oracle import experts as ox
from paper_2203_14685_amd import binding as b

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
A = 1 << 20  # an aligned stand-in address


@pytest.fixture(scope="module")
def lib():
    return hm.load()


def test_struct_layouts(lib):
    assert ctypes.sizeof(b.ExpertsParams) == 28
    assert ctypes.sizeof(b.TokenLayerParams) == 72 and b.TokenLayerParams.h.offset == 56
    assert ctypes.sizeof(b.GradTensor) == 32 and b.GradTensor.n.offset == 16 and b.GradTensor.dtype.offset == 24


EX = dict(E=4, capacity=10, d=64, h=128, act=0, gated=0, dtype=1)
BAD_EX = [(dict(E=0), 1), (dict(E=1025), 1), (dict(capacity=-1), 1), (dict(E=1024, capacity=1 << 21), 1), (dict(d=0), 1),
          (dict(h=0), 1), (dict(act=3), 1), (dict(act=-1), 1), (dict(gated=2), 1), (dict(dtype=2), 1), (dict(d=60), 2),
          (dict(h=4), 2), (dict(d=2, dtype=0), 2), (dict(d=(1 << 20) + 8), 2), (dict(h=(1 << 20) + 8), 2),
          (dict(E=1024, d=1 << 20, h=1 << 20), 2)]


def _experts(lib, p, **kw):
    a = dict(xe=A, w1=A, b1=None, w2=A, b2=None, counts=None, pre=None, hidden=A, ye=A)
    a.update(kw)
    return lib.moe_experts(ctypes.byref(p), a["xe"], a["w1"], a["b1"], a["w2"], a["b2"], a["counts"], a["pre"], a["hidden"],
                           a["ye"], None)


def _experts_bwd(lib, p, ws=A, bytes_=1 << 40, **kw):
    a = dict(dye=A, xe=A, w1=A, w2=A, counts=None, pre=A, hidden=A, dxe=A, dw1=A, db1=A, dw2=A, db2=A)
    a.update(kw)
    return lib.moe_experts_bwd(ctypes.byref(p), *[a[k] for k in ("dye", "xe", "w1", "w2", "counts", "pre", "hidden", "dxe",
                                                                "dw1", "db1", "dw2", "db2")], ws, bytes_, None)


@pytest.mark.parametrize("bad,status", BAD_EX)
def test_bad_experts_params(lib, bad, status):
    p = b.ExpertsParams(**{**EX, **bad})
    n = ctypes.c_size_t(0)
    assert _experts(lib, p) == status and lib.moe_last_error()
    assert _experts_bwd(lib, p) == status
    assert lib.moe_experts_bwd_workspace_size(ctypes.byref(p), ctypes.byref(n)) == status


def test_bad_experts_pointers(lib):
    p = b.ExpertsParams(**EX)
    for key in ("xe", "w1", "w2", "hidden", "ye"):
        assert _experts(lib, p, **{key: None}) == b.MOE_ERR_INVALID_ARG, key
        assert _experts(lib, p, **{key: A + 8}) == b.MOE_ERR_UNSUPPORTED, key
    assert _experts(lib, p, pre=A + 2) == b.MOE_ERR_UNSUPPORTED
    for key in ("b1", "b2", "counts"):
        assert _experts(lib, p, **{key: A + 2}) == b.MOE_ERR_INVALID_ARG, key
    for key in ("dye", "xe", "w1", "w2", "pre", "hidden"):
        assert _experts_bwd(lib, p, **{key: None}) == b.MOE_ERR_INVALID_ARG, key
    for key in ("dxe", "dw1", "dw2"):
        assert _experts_bwd(lib, p, **{key: A + 4}) == b.MOE_ERR_UNSUPPORTED, key
    for key in ("db1", "db2", "counts"):
        assert _experts_bwd(lib, p, **{key: A + 2}) == b.MOE_ERR_INVALID_ARG, key
    assert lib.moe_experts(None, *([None] * 10)) == b.MOE_ERR_INVALID_ARG
    n = hm.moe_experts_bwd_workspace_size(p)
    assert n >= 4 * 10 * 128 * 2
    assert _experts_bwd(lib, p, bytes_=n - 1) == b.MOE_ERR_WORKSPACE
    assert _experts_bwd(lib, p, ws=None) == b.MOE_ERR_WORKSPACE
    assert _experts_bwd(lib, p, ws=A + 8) == b.MOE_ERR_WORKSPACE


def test_nothing_to_do_needs_no_buffers(lib):
    p = b.ExpertsParams(**{**EX, "capacity": 0})
    assert _experts(lib, p, xe=None, w1=None, w2=None, hidden=None, ye=None) == 0


LAYER = dict(S=4, d=64, E=8, k=2, h=128, kind=0, act=0, gated=False, dtype=1, normalize=0, routed=False, groups=0,
             hash_seed=0, temperature=0.0, hash_vocab=0)
BAD_LAYER = [(dict(S=-1), 1), (dict(E=0), 1), (dict(k=9, E=16), 1), (dict(kind=4), 1), (dict(kind=3), 1), (dict(act=3), 1),
             (dict(dtype=2), 1), (dict(S=257), 2), (dict(S=257, routed=True), 2), (dict(k=0, routed=True), 1),
             (dict(d=60), 2), (dict(h=4), 2), (dict(d=1 << 18, h=1 << 13), 2), (dict(S=256, k=8, h=1 << 20), 2),
             (dict(temperature=-1.0), 1)]


def _layer(lib, p, ws=A, bytes_=1 << 40, **kw):
    a = dict(x=A, wg=A, bias=None, token_ids=None, noise=None, hash_table=None, w1=A, b1=None, w2=A, b2=None, ids=A,
             weights=A, y=A)
    a.update(kw)
    return lib.moe_token_layer(ctypes.byref(p), *a.values(), ws, bytes_, None)


@pytest.mark.parametrize("bad,status", BAD_LAYER)
def test_bad_layer_params(lib, bad, status):
    p = hm.token_layer_params(**{**LAYER, **bad})
    n = ctypes.c_size_t(0)
    assert _layer(lib, p) == status and lib.moe_last_error()
    assert lib.moe_token_layer_workspace_size(ctypes.byref(p), ctypes.byref(n)) == status


def test_bad_layer_arguments(lib):
    p = hm.token_layer_params(**LAYER)
    for key in ("x", "w1", "w2", "y"):
        assert _layer(lib, p, **{key: None}) == b.MOE_ERR_INVALID_ARG, key
        assert _layer(lib, p, **{key: A + 8}) == b.MOE_ERR_UNSUPPORTED, key
    for key in ("wg", "ids", "weights"):
        assert _layer(lib, p, **{key: None}) == b.MOE_ERR_INVALID_ARG, key
    for key in ("token_ids", "noise", "hash_table"):  # not for this gate
        assert _layer(lib, p, **{key: A}) == b.MOE_ERR_INVALID_ARG, key
    n = hm.moe_token_layer_workspace_size(p)
    assert _layer(lib, p, bytes_=n - 1) == b.MOE_ERR_WORKSPACE
    assert _layer(lib, p, ws=A + 4) == b.MOE_ERR_WORKSPACE
    routed = hm.token_layer_params(**{**LAYER, "routed": True})
    assert _layer(lib, routed) == b.MOE_ERR_INVALID_ARG  # wg with given routing
    p.gate.capacity = 3
    assert _layer(lib, p) == b.MOE_ERR_INVALID_ARG
    p.gate.capacity, p.gate.logits_in = 0, 1
    assert _layer(lib, p) == b.MOE_ERR_INVALID_ARG
    hashed = hm.token_layer_params(**{**LAYER, "kind": 2, "k": 1})
    assert _layer(lib, hashed, token_ids=A) == b.MOE_ERR_INVALID_ARG  # wg with a hash gate
    assert _layer(lib, hashed, wg=None) == b.MOE_ERR_INVALID_ARG      # no token ids


def _grad(*specs):
    return (b.GradTensor * len(specs))(*[b.GradTensor(s, d, n, t, 0) for s, d, n, t in specs])


def test_bad_gradients(lib):
    good = _grad((A, A, 100, 0), (2 * A, 2 * A, 50, 1))
    n = ctypes.c_size_t(0)
    assert lib.moe_grad_norm_workspace_size(good, 2, ctypes.byref(n)) == 0 and n.value > 0
    assert lib.moe_grad_norm_workspace_size(None, 0, ctypes.byref(n)) == 0 and n.value == 0
    assert lib.moe_grad_norm_workspace_size(good, 2, None) == b.MOE_ERR_INVALID_ARG
    for bad, count, status in [(good, -1, 1), (None, 1, 1), (_grad((None, A, 1, 0)), 1, 1), (_grad((A + 1, A, 1, 0)), 1, 1),
                               (_grad((A, A, -1, 0)), 1, 1), (_grad((A, A, 1, 2)), 1, 1),
                               (_grad((A, A, (1 << 44) + 1, 0)), 1, 2), (_grad(*[(A, A, 1 << 43, 0)] * 5), 5, 2)]:
        assert lib.moe_grad_norm(bad, count, None, None, A, 1 << 40, None) == status
        assert lib.moe_grad_clip(bad, count, A, 1.0, None, None) == status
    assert lib.moe_grad_norm(good, 2, None, None, A, 0, None) == b.MOE_ERR_WORKSPACE
    assert lib.moe_grad_norm(good, 2, A + 4, None, A, 1 << 20, None) == b.MOE_ERR_INVALID_ARG
    for mx in (-1.0, float("nan"), float("inf")):
        assert lib.moe_grad_clip(good, 2, A, mx, None, None) == b.MOE_ERR_INVALID_ARG
    assert lib.moe_grad_clip(good, 2, None, 1.0, None, None) == b.MOE_ERR_INVALID_ARG
    # overlaps: twice the same, an output over another's input, nested ranges; neighbours are fine
    for bad in [((A, A, 100, 0), (A, A, 100, 0)), ((A, 2 * A, 100, 0), (2 * A + 396, 3 * A, 10, 0)),
                ((A, 2 * A, 100, 0), (3 * A, 2 * A + 40, 4, 0)), ((A, A + 4, 100, 0),)]:
        assert lib.moe_grad_clip(_grad(*bad), len(bad), A, 1.0, None, None) == b.MOE_ERR_INVALID_ARG, bad
        assert b"overlaps" in lib.moe_last_error()


def test_binding_refuses_wrong_tensors():
    x = torch.zeros((2, 4, 8))
    with pytest.raises(ValueError, match="weights"):
        hm.experts(x, torch.zeros((2, 8, 16)), torch.zeros((2, 8, 8)))
    with pytest.raises(ValueError, match="weights"):
        hm.experts(x, torch.zeros((2, 8, 8)), torch.zeros((2, 8, 8)), gated=True)
    with pytest.raises(ValueError, match="experts"):
        hm.experts(x, torch.zeros((3, 8, 8)), torch.zeros((3, 8, 8)))
    with pytest.raises(ValueError, match="on the GPU"):
        hm.experts(x, torch.zeros((2, 8, 8)), torch.zeros((2, 8, 8)))
    with pytest.raises(ValueError, match="together"):
        hm.token_layer(x[0], torch.zeros((2, 8, 8)), torch.zeros((2, 8, 8)), ids=torch.zeros((4, 1), dtype=torch.int32))
    with pytest.raises(ValueError, match="outputs"):
        hm.grad_tensors([x], [])


def _forward_plain(xe, w1, b1, w2, b2, counts, kind, gated):
    """Element by element, no matrix product."""
    E, C, d = xe.shape
    h = w2.shape[1]
    y = np.zeros((E, C, d))
    for e in range(E):
        for c in range(counts[e]):
            pre = [sum(xe[e, c, i] * w1[e, i, j] for i in range(d)) + b1[e, j] for j in range(w1.shape[2])]
            f = {0: lambda a: max(a, 0.0), 2: lambda a: a / (1 + np.exp(-a)),
                 1: lambda a: 0.5 * a * (1 + np.tanh(np.sqrt(2 / np.pi) * (a + 0.044715 * a ** 3)))}[kind]
            hid = [f(pre[j]) * (pre[h + j] if gated else 1.0) for j in range(h)]
            for i in range(d):
                y[e, c, i] = sum(hid[j] * w2[e, j, i] for j in range(h)) + b2[e, i]
    return y


@pytest.mark.parametrize("kind", [0, 1, 2])
@pytest.mark.parametrize("gated", [False, True])
def test_oracle_forward_and_gradients(kind, gated):
    """The oracle's forward against plain sums, its gradients against central differences (the step's
    square times the third derivative, and cancellation: 1e-6 relative with steps of 1e-4)."""
    rng = np.random.default_rng(kind)
    E, C, d, h = 2, 3, 4, 5
    h1 = 2 * h if gated else h
    a = dict(xe=rng.standard_normal((E, C, d)), w1=rng.standard_normal((E, d, h1)), b1=rng.standard_normal((E, h1)),
             w2=rng.standard_normal((E, h, d)), b2=rng.standard_normal((E, d)))
    counts = [2, 3]
    dye = rng.standard_normal((E, C, d))
    o = ox.experts(a["xe"], a["w1"], a["b1"], a["w2"], a["b2"], counts, kind, gated, 0.0)
    assert np.allclose(o["ye"][0], _forward_plain(a["xe"], a["w1"], a["b1"], a["w2"], a["b2"], counts, kind, gated), rtol=1e-12)
    g = ox.experts_bwd(dye, a["xe"], a["w1"], a["w2"], counts, o["pre"][0], o["hidden"][0], kind, gated, 0.0)
    for key, grad in (("xe", "dxe"), ("w1", "dw1"), ("b1", "db1"), ("w2", "dw2"), ("b2", "db2")):
        v = rng.standard_normal(a[key].shape)
        loss = []
        for s in (1e-4, -1e-4):
            q = {**a, key: a[key] + s * v}
            loss.append((ox.experts(q["xe"], q["w1"], q["b1"], q["w2"], q["b2"], counts, kind, gated, 0.0)["ye"][0] * dye).sum())
        num = (loss[0] - loss[1]) / 2e-4
        assert abs((g[grad][0] * v).sum() - num) <= 1e-6 * np.abs(g[grad][0] * v).sum() + 1e-6, key


def test_exported_symbols_are_the_declared_ones(lib):
    text = open(os.path.join(ROOT, "include", "hetumoe.h")).read()
    for name in set(re.findall(r"\bmoe_(?:experts|token_layer|grad)\w*\s*\(", text)):
        assert hasattr(lib, name.rstrip(" ("))
