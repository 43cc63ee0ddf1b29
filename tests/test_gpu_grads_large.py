"""The gradient norm and clipping where a block takes several chunks, past the size from which
accesses are non-temporal, and at norms whose scale is no normal fp32 number."""

import math

import pytest
import torch

import paper_2203_14685_amd as hm

pytestmark = pytest.mark.gpu

DEV = "cuda"
U32, U_BF16 = 2.0 ** -24, 2.0 ** -8
CHUNK, BLOCKS = 8192, 2048  # values per chunk; blocks of a launch


@pytest.fixture(autouse=True, scope="module")
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    hm.load()
    yield


def _normal(n, dtype, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return torch.randn((n,), generator=g, device=DEV).to(dtype)


def _norm64(grads):
    return math.sqrt(sum(float((t.double() ** 2).sum()) for t in grads))


def _check_scaled(out, src, scale):
    for o, t in zip(out, src):
        v = t.double() * scale
        # the scale in fp32 and its fp64 inputs, the product's rounding
        half = (U_BF16 if t.dtype == torch.bfloat16 else U32) + 3 * U32
        assert o.dtype == t.dtype and ((o.double() - v).abs() <= half * v.abs() + 1e-40).all(), (t.shape, t.dtype)


def _both_ways(grads, max_norm):
    """Norm, repeated; clipped into other tensors and in place."""
    total = _norm64(grads)
    src = [t.clone() for t in grads]
    norm, sumsq = hm.grad_norm(grads)
    for _ in range(2):
        again = hm.grad_norm(grads)
        assert torch.equal(norm, again[0]) and torch.equal(sumsq, again[1])
    assert abs(float(sumsq) - total ** 2) <= 1e-9 * total ** 2
    assert abs(float(norm) - total) <= 2 * U32 * total
    out = [torch.full_like(t, -7.0) for t in grads]
    got = hm.clip_grads(grads, max_norm, out=out)
    assert torch.equal(got, norm)
    assert all(torch.equal(a, b) for a, b in zip(grads, src))
    _check_scaled(out, src, min(1.0, max_norm / total))
    hm.clip_grads(grads, max_norm)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(grads, out))


def test_blocks_that_take_several_chunks():
    """More chunks than blocks, of tensors of odd sizes: a block's later chunks lie in other tensors."""
    print("[case] grads of several chunks per block", flush=True)
    sizes = [9_000_001, 3, 5_000_017, CHUNK, CHUNK + 1, 6_000_011, 777]
    assert sum(-(-n // CHUNK) for n in sizes) > BLOCKS
    grads = [_normal(n, torch.bfloat16 if i % 2 else torch.float32, 3 + i) for i, n in enumerate(sizes)]
    _both_ways(grads, 11.0)


@pytest.mark.parametrize("share", [0.3, 2.0])
def test_beyond_the_infinity_cache(share):
    """More than 256 MB: aligned, misaligned and short tensors of both types, odd tails."""
    print(f"[case] grads beyond 256 MB, share {share}", flush=True)
    grads = [_normal(100_000_003, torch.bfloat16, 1), _normal(30_000_002, torch.bfloat16, 2)[1:],
             _normal(7_000_005, torch.float32, 3), _normal(5_000_004, torch.float32, 4)[3:], _normal(5, torch.float32, 5)]
    assert sum(t.numel() * t.element_size() for t in grads) > 256 << 20
    assert grads[1].data_ptr() % 16 == 2 and grads[3].data_ptr() % 16 == 12
    _both_ways(grads, share * _norm64(grads))


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
