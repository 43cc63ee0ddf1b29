"""CPU checks of the embedding, dropout and 8-bit entry points: struct layouts, workspace
sizes, and that bad arguments are refused before any HIP call (the stand-in addresses
are never dereferenced)."""

import ctypes

import pytest
import torch

import paper_2203_14685_amd as hm
from paper_2203_14685_amd import binding as b

A = 1 << 20  # an aligned stand-in address
INVALID, UNSUPPORTED, WORKSPACE = b.MOE_ERR_INVALID_ARG, b.MOE_ERR_UNSUPPORTED, b.MOE_ERR_WORKSPACE


@pytest.fixture(scope="module")
def lib():
    return hm.load()


def test_struct_layouts(lib):
    assert ctypes.sizeof(b.EmbedParams) == 24 and b.EmbedParams.scale.offset == 16
    assert ctypes.sizeof(b.DropoutMask) == 32
    assert b.DropoutMask.step.offset == 16 and b.DropoutMask.p.offset == 24


EMBED = dict(T=100, V=50, d=64, dtype=1, scale=1.0, accumulate=0)
BAD_EMBED = [(dict(T=-1), INVALID), (dict(V=0), INVALID), (dict(d=0), INVALID), (dict(dtype=2), INVALID),
             (dict(scale=float("inf")), INVALID), (dict(scale=float("nan")), INVALID), (dict(accumulate=2), INVALID),
             (dict(d=60), UNSUPPORTED), (dict(d=2, dtype=0), UNSUPPORTED), (dict(d=(1 << 20) + 8), UNSUPPORTED)]


@pytest.mark.parametrize("bad,status", BAD_EMBED)
def test_bad_embed_params(lib, bad, status):
    p = b.EmbedParams(**{**EMBED, **bad})
    n = ctypes.c_size_t(0)
    assert lib.moe_embed(ctypes.byref(p), A, A, A, None) == status and lib.moe_last_error()
    assert lib.moe_embed_bwd(ctypes.byref(p), A, A, A, A, 1 << 40, None) == status
    assert lib.moe_embed_bwd_workspace_size(ctypes.byref(p), ctypes.byref(n)) == status


def test_bad_embed_calls(lib):
    p = b.EmbedParams(**EMBED)
    ref = ctypes.byref(p)
    assert lib.moe_embed(None, A, A, A, None) == INVALID
    assert lib.moe_embed(ref, None, A, A, None) == INVALID and lib.moe_embed(ref, A, None, A, None) == INVALID
    assert lib.moe_embed(ref, A, A, None, None) == INVALID and lib.moe_embed(ref, A + 2, A, A, None) == INVALID
    assert lib.moe_embed(ref, A, A + 8, A, None) == UNSUPPORTED and lib.moe_embed(ref, A, A, A + 8, None) == UNSUPPORTED
    n = hm.moe_embed_bwd_workspace_size(p)
    assert lib.moe_embed_bwd(ref, None, A, A, A, n, None) == INVALID
    assert lib.moe_embed_bwd(ref, A, A, None, A, n, None) == INVALID
    assert lib.moe_embed_bwd(ref, A + 4, A, A, A, n, None) == UNSUPPORTED
    assert lib.moe_embed_bwd(ref, A, A, A, A, n - 1, None) == WORKSPACE
    assert lib.moe_embed_bwd(ref, A, A, A, None, n, None) == WORKSPACE
    assert lib.moe_embed_bwd(ref, A, A, A, A + 8, n, None) == WORKSPACE
    p.accumulate = 1  # for the gradient alone
    assert lib.moe_embed(ref, A, A, A, None) == INVALID
    p = b.EmbedParams(**{**EMBED, "T": (1 << 30) + 1})
    assert lib.moe_embed_bwd(ctypes.byref(p), A, A, A, A, 1 << 50, None) == UNSUPPORTED
    assert lib.moe_embed_bwd_workspace_size(ref, None) == INVALID
    p = b.EmbedParams(**{**EMBED, "T": 0})
    assert lib.moe_embed(ctypes.byref(p), None, None, None, None) == b.MOE_OK


@pytest.mark.parametrize("T", [0, 1, 8192, 8193, 1 << 20])
def test_embed_workspace_holds_its_lists(lib, T):
    n = hm.moe_embed_bwd_workspace_size(hm.embed_params(T, 1000, 64, hm.MOE_BF16))
    assert n >= 8 * T * (2 if T > 8192 else 1)


def _mask(**kw):
    return b.DropoutMask(**{**dict(seed=1, call=2, step=None, p=0.1, pad=0), **kw})


@pytest.mark.parametrize("p", [-0.01, 1.01, float("nan"), float("inf")])
def test_bad_dropout_share(lib, p):
    m, e = _mask(p=p), b.ExpertsParams(E=4, capacity=10, d=64, h=128, act=0, gated=0, dtype=1)
    assert lib.moe_dropout(ctypes.byref(m), 8, 1, A, None, A, None) == INVALID
    assert lib.moe_experts_dropout(ctypes.byref(e), ctypes.byref(m), A, A, None, A, None, None, None, A, A, None) == INVALID
    assert lib.moe_experts_dropout_bwd(ctypes.byref(e), ctypes.byref(m), *[A] * 12, A, 1 << 40, None) == INVALID


def test_bad_dropout_calls(lib):
    m = ctypes.byref(_mask())
    assert lib.moe_dropout(None, 8, 1, A, None, A, None) == INVALID
    assert lib.moe_dropout(m, -1, 1, A, None, A, None) == INVALID
    assert lib.moe_dropout(m, (1 << 44) + 1, 1, A, None, A, None) == UNSUPPORTED
    assert lib.moe_dropout(m, 8, 2, A, None, A, None) == INVALID
    assert lib.moe_dropout(m, 8, 1, None, None, A, None) == INVALID
    assert lib.moe_dropout(m, 8, 1, A, None, None, None) == INVALID
    for i in range(3):
        args = [A, A, A]
        args[i] = A + 4
        assert lib.moe_dropout(m, 8, 1, *args, None) == UNSUPPORTED
    assert lib.moe_dropout(ctypes.byref(_mask(step=A + 4)), 8, 1, A, None, A, None) == INVALID
    assert lib.moe_dropout(m, 0, 1, None, None, None, None) == b.MOE_OK
    e = b.ExpertsParams(E=4, capacity=10, d=64, h=128, act=0, gated=0, dtype=1)
    assert lib.moe_experts_dropout(ctypes.byref(e), None, A, A, None, A, None, None, None, A, A, None) == INVALID
    assert lib.moe_experts_dropout(ctypes.byref(e), m, A, A, None, A, None, None, None, None, A, None) == INVALID
    n = hm.moe_experts_bwd_workspace_size(e)
    assert lib.moe_experts_dropout_bwd(ctypes.byref(e), m, *[A] * 12, A, n - 1, None) == WORKSPACE
    e.h = 4
    assert lib.moe_experts_dropout(ctypes.byref(e), m, A, A, None, A, None, None, None, A, A, None) == UNSUPPORTED


def test_bad_quantize_calls(lib):
    q = lib.moe_quantize
    assert q(-1, 16, 1, A, A, A, None) == INVALID and q(4, 0, 1, A, A, A, None) == INVALID
    assert q(4, 24, 1, A, A, A, None) == UNSUPPORTED and q(4, 16, 3, A, A, A, None) == INVALID
    assert q(4, 16, 1, None, A, A, None) == INVALID and q(4, 16, 1, A, None, A, None) == INVALID
    assert q(4, 16, 1, A, A, None, None) == INVALID and q(4, 16, 1, A + 8, A, A, None) == UNSUPPORTED
    assert q(4, 16, 1, A, A + 8, A, None) == UNSUPPORTED and q(4, 16, 1, A, A, A + 2, None) == INVALID
    assert q((1 << 32) + 1, 16, 1, A, A, A, None) == UNSUPPORTED
    assert q(0, 16, 1, None, None, None, None) == b.MOE_OK
    w = lib.moe_quantize_weights
    assert w(0, 16, 16, 1, A, A, A, None) == INVALID and w(1025, 16, 16, 1, A, A, A, None) == INVALID
    assert w(1, 0, 16, 1, A, A, A, None) == INVALID and w(1, 16, 0, 1, A, A, A, None) == INVALID
    assert w(1, 24, 16, 1, A, A, A, None) == UNSUPPORTED and w(1, 16, 24, 1, A, A, A, None) == UNSUPPORTED
    assert w(1, (1 << 17) + 16, 16, 1, A, A, A, None) == UNSUPPORTED
    assert w(1, 16, (1 << 18) + 16, 1, A, A, A, None) == UNSUPPORTED
    assert w(1, 16, 16, 1, None, A, A, None) == INVALID and w(1, 16, 16, 1, A, A + 8, A, None) == UNSUPPORTED


EX = dict(E=4, capacity=10, d=64, h=128, act=0, gated=0, dtype=1)
BAD_INT8 = [(dict(E=0), INVALID), (dict(act=3), INVALID), (dict(dtype=2), INVALID), (dict(d=72), UNSUPPORTED),
            (dict(h=40), UNSUPPORTED), (dict(d=(1 << 17) + 16), UNSUPPORTED), (dict(h=(1 << 17) + 16), UNSUPPORTED)]


def _int8(lib, p, ws=A, bytes_=1 << 40, **kw):
    a = dict(xe=A, q1=A, s1=A, b1=None, q2=A, s2=A, b2=None, counts=None, ye=A)
    a.update(kw)
    return lib.moe_experts_int8(ctypes.byref(p), *[a[k] for k in ("xe", "q1", "s1", "b1", "q2", "s2", "b2", "counts", "ye")],
                                ws, bytes_, None)


def test_bad_experts_int8(lib):
    for bad, status in BAD_INT8:
        p, n = b.ExpertsParams(**{**EX, **bad}), ctypes.c_size_t(0)
        assert _int8(lib, p) == status, bad
        assert lib.moe_experts_int8_workspace_size(ctypes.byref(p), ctypes.byref(n)) == status
    p = b.ExpertsParams(**EX)
    for key in ("xe", "q1", "q2", "ye"):
        assert _int8(lib, p, **{key: None}) == INVALID and _int8(lib, p, **{key: A + 8}) == UNSUPPORTED, key
    for key in ("s1", "s2"):
        assert _int8(lib, p, **{key: None}) == INVALID and _int8(lib, p, **{key: A + 2}) == INVALID, key
    for key in ("b1", "b2", "counts"):
        assert _int8(lib, p, **{key: A + 2}) == INVALID, key
    n = hm.moe_experts_int8_workspace_size(p)
    assert n >= 40 * (128 + 4 + 2 * 128)
    assert _int8(lib, p, bytes_=n - 1) == WORKSPACE and _int8(lib, p, ws=None) == WORKSPACE
    p.capacity = 0
    assert lib.moe_experts_int8(ctypes.byref(p), *[None] * 9, None, 0, None) == b.MOE_OK


LAYER = dict(S=5, d=64, E=8, k=2, h=32)


def _layer(lib, p, ws=A, bytes_=1 << 40, **kw):
    a = dict(x=A, wg=A, bias=None, token_ids=None, noise=None, hash_table=None, q1=A, s1=A, b1=None, q2=A, s2=A, b2=None,
             ids=A, weights=A, y=A)
    a.update(kw)
    return lib.moe_token_layer_int8(ctypes.byref(p), *a.values(), ws, bytes_, None)


def test_bad_token_layer_int8(lib):
    for bad, status in [(dict(d=72), UNSUPPORTED), (dict(h=40), UNSUPPORTED), (dict(S=257), UNSUPPORTED),
                        (dict(k=9), INVALID), (dict(act=5), INVALID), (dict(h=(1 << 17) + 16), UNSUPPORTED)]:
        p, n = hm.token_layer_params(**{**LAYER, **bad}, dtype=hm.MOE_BF16), ctypes.c_size_t(0)
        assert _layer(lib, p) == status, bad
        assert lib.moe_token_layer_int8_workspace_size(ctypes.byref(p), ctypes.byref(n)) == status
    p = hm.token_layer_params(**LAYER, dtype=hm.MOE_BF16)
    for key in ("x", "wg", "q1", "s1", "q2", "s2", "ids", "weights", "y"):
        assert _layer(lib, p, **{key: None}) == INVALID, key
    for key in ("q1", "q2", "x", "y"):
        assert _layer(lib, p, **{key: A + 8}) == UNSUPPORTED, key
    assert _layer(lib, p, token_ids=A) == INVALID and _layer(lib, p, noise=A) == INVALID
    n = hm.moe_token_layer_int8_workspace_size(p)
    assert _layer(lib, p, bytes_=n - 1) == WORKSPACE
    p = hm.token_layer_params(**LAYER, dtype=hm.MOE_BF16, routed=True)
    assert _layer(lib, p) == INVALID  # wg of a routed layer


def test_wrappers_refuse_shapes(lib):
    t = torch.empty
    with pytest.raises(ValueError, match="quantized weights"):
        hm.experts_int8(t(2, 3, 64), t(2, 64, 32, dtype=torch.int8), t(2, 32), t(2, 64, 32, dtype=torch.int8), t(2, 64))
    with pytest.raises(ValueError, match="go together"):
        hm.embed_bwd(t(4, 64), t(5, dtype=torch.int32), 10)
    with pytest.raises(ValueError, match="accumulate"):
        hm.embed_bwd(t(4, 64), t(4, dtype=torch.int32), 10, accumulate=True)
    with pytest.raises(ValueError, match="one shape"):
        hm.dropout(t(4, 64), hm.dropout_mask(0.1, 1), residual=t(64))
    with pytest.raises(TypeError, match="step"):
        hm.dropout_mask(0.1, 1, step=t(1, dtype=torch.int32))
    with pytest.raises(ValueError, match="GPU"):
        hm.quantize(t(4, 64))
    with pytest.raises(TypeError):
        hm.quantize(t(4, 64, dtype=torch.float16))
