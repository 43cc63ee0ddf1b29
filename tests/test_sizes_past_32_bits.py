"""CPU checks of sizes past 32 bits, of which the C structs and calls would be handed the low ones: a table
of 2^32 + 5 rows would be read as one of 5.  Tensors of the meta device have the shapes without the memory."""

import pytest
import torch

import paper_2203_14685_amd as hm

BIG = 2 ** 32 + 16
REFUSED = "past 2\\^31 - 1"


def _t(*shape, dtype=torch.bfloat16):
    return torch.empty(shape, dtype=dtype, device="meta")


def test_parameters():
    for kw in (dict(T=BIG, V=5, d=8), dict(T=3, V=BIG, d=8), dict(T=3, V=5, d=BIG), dict(T=2 ** 31, V=5, d=8)):
        with pytest.raises(ValueError, match=REFUSED):
            hm.embed_params(**kw)
    assert hm.embed_params(2 ** 31 - 1, 5, 8).T == 2 ** 31 - 1
    for i in range(4):
        sizes = [2, 3, 16, 16]
        sizes[i] = BIG
        with pytest.raises(ValueError, match=REFUSED):
            hm.experts_params(*sizes)
    for i in range(5):
        sizes = [2, 16, 4, 2, 16]
        sizes[i] = BIG
        with pytest.raises(ValueError, match=REFUSED):
            hm.token_layer_params(*sizes)


def test_embedding():
    ids, long_ids = _t(4, dtype=torch.int32), _t(BIG, dtype=torch.int32)
    with pytest.raises(ValueError, match=REFUSED):
        hm.embed(long_ids, _t(5, 8))
    with pytest.raises(ValueError, match=REFUSED):
        hm.embed(ids, _t(BIG, 8))
    with pytest.raises(ValueError, match=REFUSED):
        hm.embed_bwd(_t(BIG, 8), long_ids, 5)
    with pytest.raises(ValueError, match=REFUSED):
        hm.embed_bwd(_t(4, 8), ids, BIG)


def test_integers():
    with pytest.raises(ValueError, match=REFUSED):
        hm.quantize(_t(2, BIG))
    for shape in ((1, BIG, 16), (1, 16, BIG), (BIG, 16, 16)):
        with pytest.raises(ValueError, match=REFUSED):
            hm.quantize_weights(_t(*shape))
    i8, f32 = torch.int8, torch.float32
    with pytest.raises(ValueError, match=REFUSED):
        hm.experts_int8(_t(1, BIG, 16), _t(1, 16, 16, dtype=i8), _t(1, 16, dtype=f32), _t(1, 16, 16, dtype=i8), _t(1, 16, dtype=f32))
    with pytest.raises(ValueError, match=REFUSED):
        hm.experts_int8(_t(1, 4, 16), _t(1, BIG, 16, dtype=i8), _t(1, BIG, dtype=f32), _t(1, 16, BIG, dtype=i8), _t(1, 16, dtype=f32))
    with pytest.raises(ValueError, match=REFUSED):
        hm.token_layer_int8(_t(BIG, 16), _t(2, 16, 16, dtype=i8), _t(2, 16, dtype=f32), _t(2, 16, 16, dtype=i8), _t(2, 16, dtype=f32),
                            ids=_t(BIG, 1, dtype=torch.int32), weights=_t(BIG, 1, dtype=f32))


def test_experts_with_dropout():
    w1, w2, m = _t(1, 16, 16), _t(1, 16, 16), hm.dropout_mask(0.1, 1)
    with pytest.raises(ValueError, match=REFUSED):
        hm.experts(_t(1, BIG, 16), w1, w2, dropout=m)
    x = _t(1, BIG, 16)
    with pytest.raises(ValueError, match=REFUSED):
        hm.experts_bwd(x, x, w1, w2, x, x, dropout=m)
