"""Helpers of the expert-network tests: seeded inputs in an element type, their
fp64 values, and comparison against the oracle's value and bound."""

import numpy as np
import torch

import paper_2203_14685_amd as hm
from oracle import experts as ox

DEV = "cuda"
TORCH = {"f32": torch.float32, "bf16": torch.bfloat16}
ROUND = {"f32": 0.0, "bf16": ox.U_BF16}
# outputs in fp32 are also rounded once, which the sums' bounds hold already
ACTS = {"relu": hm.MOE_ACT_RELU, "gelu": hm.MOE_ACT_GELU, "silu": hm.MOE_ACT_SILU}


def announce(msg):
    print(f"[case] {msg}", flush=True)


def normal(rng, shape, dtype, scale=1.0):
    """A CPU tensor of the type and its exact fp64 values."""
    t = torch.from_numpy((rng.standard_normal(shape) * scale).astype(np.float32)).to(TORCH[dtype])
    return t, t.double().numpy()


def f64(t):
    return t.detach().cpu().double().numpy()


def check(gpu, ref, what):
    """|gpu - value| <= bound, element by element."""
    value, bound = ref
    g = f64(gpu)
    assert g.shape == value.shape, (what, g.shape, value.shape)
    bad = ~(np.abs(g - value) <= bound)
    if bad.any():
        i = tuple(int(v) for v in np.argwhere(bad)[0])
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.size} beyond the bound; first at {i}: "
                             f"gpu {g[i]} value {value[i]} bound {bound[i]}")


def weights(rng, E, d, h, gated, dtype, bias=True):
    """(device, fp64) pairs w1, b1, w2, b2."""
    h1 = 2 * h if gated else h
    w1 = normal(rng, (E, d, h1), dtype, d ** -0.5)
    w2 = normal(rng, (E, h, d), dtype, h ** -0.5)
    b1 = normal(rng, (E, h1), "f32", 0.3) if bias else (None, None)
    b2 = normal(rng, (E, d), "f32", 0.3) if bias else (None, None)
    return [(None if t is None else t.to(DEV), v) for t, v in (w1, b1, w2, b2)]
