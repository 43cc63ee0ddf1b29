"""Clipping at norms whose scale is no normal fp32 number."""

import math

import pytest
import torch

import paper_2203_14685_amd as hm

pytestmark = pytest.mark.gpu

DEV = "cuda"
U32, U_BF16 = 2.0 ** -24, 2.0 ** -8


@pytest.fixture(autouse=True, scope="module")
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    hm.load()
    yield


def _norm64(grads):
    return math.sqrt(sum(float((t.double() ** 2).sum()) for t in grads))


@pytest.mark.parametrize("value,max_norm", [(3e38, 1.0), (3e38, 1e-3), (1e37, 1e-6), (2.0, 1e-38), (1e-3, 1e-39)])
def test_scale_below_the_normal_numbers(value, max_norm):
    """max_norm / norm below 2^-126 keeps its digits: the result is as near as with any other scale."""
    print(f"[case] clip {value} to {max_norm}", flush=True)
    grads = [torch.full((200_003,), value, device=DEV), torch.full((100_001,), -value, dtype=torch.bfloat16, device=DEV)]
    total = _norm64(grads)
    assert max_norm / total < 2.0 ** -126
    out = [torch.empty_like(t) for t in grads]
    hm.clip_grads(grads, max_norm, out=out)
    torch.cuda.synchronize()
    for o, t in zip(out, grads):
        v = t.double() * (max_norm / total)
        # where the result itself is below the normal numbers: half of its last place
        half = (U_BF16 if t.dtype == torch.bfloat16 else U32) + 4 * U32
        place = 2.0 ** -134 if t.dtype == torch.bfloat16 else 2.0 ** -150
        assert ((o.double() - v).abs() <= half * v.abs() + 2 * place).all(), (o[0], v[0])
