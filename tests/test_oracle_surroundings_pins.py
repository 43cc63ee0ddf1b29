"""CPU pins of the oracle's dropout, embedding and 8-bit networks: published vectors of the
generator, brute force, closed forms, and gradients against differences."""

from fractions import Fraction

import numpy as np
import pytest

from oracle import dropout as od
from oracle import embed as oe
from oracle import experts as ox
from oracle import int8 as oi

# the known answers that its authors publish with the generator
KNOWN = [((0, 0, 0, 0), (0, 0), (0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8)),
         ((0xFFFFFFFF,) * 4, (0xFFFFFFFF,) * 2, (0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD)),
         ((0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344), (0xA4093822, 0x299F31D0),
          (0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1))]


@pytest.mark.parametrize("counter,key,answer", KNOWN)
def test_philox_known_answers(counter, key, answer):
    assert tuple(int(v) for v in od.philox4x32(np.array(counter, dtype=np.uint64), np.array(key, dtype=np.uint64))) == answer


def test_words_follow_the_blocks():
    seed, call = 0x299F31D0A4093822, 0x0370734413198A2E
    first = (0x85A308D3 << 32 | 0x243F6A88) * 8 % 2 ** 64
    assert first // 8 == (0x85A308D3 << 32 | 0x243F6A88) % 2 ** 61
    w = od.words(3, 21, 5, 7)
    assert np.array_equal(w, od.words(0, 24, 5, 7)[3:]) and w.max() < 65536
    block = od.philox4x32(np.array([2, 0, 0x13198A2E, 0x03707344], dtype=np.uint64), np.array([0xA4093822, 0x299F31D0], dtype=np.uint64))
    got = od.words(16, 8, seed, call)
    assert [int(v) for v in got] == [int(block[j // 2]) >> 16 * (j % 2) & 0xFFFF for j in range(8)]


def test_dropout_share_and_mean():
    f = od.factors(0, 200_000, 0.3, 11, 2)
    # binomial: 5 standard deviations of sqrt(0.3 * 0.7 / n) = 0.001
    assert abs((f == 0).mean() - 0.3) < 5.2e-3
    assert set(np.unique(f)) == {0.0, 65536.0 / (65536 - 19661)}
    assert (od.factors(0, 999, 0.0, 1, 1) == 1).all() and (od.factors(0, 999, 1.0, 1, 1) == 0).all()
    assert not np.array_equal(od.factors(0, 999, 0.5, 1, 1), od.factors(0, 999, 0.5, 1, 2))


@pytest.mark.parametrize("kind,gated", [(ox.SILU, True), (ox.GELU, False)])
def test_dropped_network_gradient_against_differences(kind, gated):
    rng = np.random.default_rng(3)
    E, C, d, h = 1, 4, 6, 8
    h1 = 2 * h if gated else h
    xe, w1, w2 = rng.standard_normal((E, C, d)), rng.standard_normal((E, d, h1)) / 2, rng.standard_normal((E, h, d)) / 2
    b1, b2, dye = rng.standard_normal((E, h1)), rng.standard_normal((E, d)), rng.standard_normal((E, C, d))
    f = od.factors(0, E * C * h, 0.4, 9, 1).reshape(E, C, h)

    def loss(xe, w1, b1, w2, b2):
        return (od.experts(xe, w1, b1, w2, b2, None, kind, gated, 0.0, f)["ye"][0] * dye).sum()

    o = od.experts(xe, w1, b1, w2, b2, None, kind, gated, 0.0, f)
    g = od.experts_bwd(dye, xe, w1, w2, None, o["pre"][0], o["hidden"][0], kind, gated, 0.0, f)
    args = [xe, w1, b1, w2, b2]
    for name, at in (("dxe", 0), ("dw1", 1), ("db1", 2), ("dw2", 3), ("db2", 4)):
        grad = g[name][0]
        for i in rng.integers(0, grad.size, 6):
            i = np.unravel_index(i, grad.shape)
            up, down = [a.copy() for a in args], [a.copy() for a in args]
            up[at][i] += 1e-5
            down[at][i] -= 1e-5
            diff = (loss(*up) - loss(*down)) / 2e-5
            # error of a central difference: third derivatives (some units) times 1e-10, rounding 1e-15 / 1e-5
            assert abs(diff - grad[i]) < 1e-7 * (1 + abs(diff)), (name, i)
    # p = 0 is the network without dropout
    ones = np.ones((E, C, h))
    plain = ox.experts(xe, w1, b1, w2, b2, None, kind, gated, 0.0)["ye"][0]
    assert np.allclose(od.experts(xe, w1, b1, w2, b2, None, kind, gated, 0.0, ones)["ye"][0], plain, rtol=1e-14)


def test_embed_and_gradient():
    rng = np.random.default_rng(0)
    table, dy, ids = rng.standard_normal((5, 3)), rng.standard_normal((7, 3)), np.array([4, 0, 4, -1, 5, 4, 2])
    y = oe.embed(ids, table, 3.0, 0.0)[0]
    assert np.array_equal(y[0], 3.0 * table[4]) and not y[3].any() and not y[4].any()
    g, bound = oe.embed_bwd(dy, ids, 5, 3.0, None, 0.0)
    assert np.allclose(g[4], 3.0 * (dy[0] + dy[2] + dy[5])) and not g[1].any() and not bound[3].any()
    # linear: the gradient is the difference quotient
    for v, j in ((4, 1), (0, 2), (1, 0)):
        up = table.copy()
        up[v, j] += 1.0
        assert np.isclose(((oe.embed(ids, up, 3.0, 0.0)[0] - y) * dy).sum(), g[v, j])
    there = rng.standard_normal((5, 3))
    assert np.array_equal(oe.embed_bwd(dy, ids, 5, 3.0, there, 0.0)[0][1], there[1])


def test_quantize_is_the_nearest_integer():
    rng = np.random.default_rng(1)
    x = rng.standard_normal((40, 48)).astype(np.float32).astype(np.float64)
    x[3] = 0.0
    x[4, 7] = x[4].__abs__().max() / 2  # half of the largest value lies on a border: 63.5
    x[5, :3] = [254.0, 127.0, -1.0]
    x[6, 1], x[7, 2] = np.inf, np.nan
    q, s = oi.quantize(x)
    for i in range(40):
        if i in (6, 7):
            assert np.isnan(s[i]) and not q[i].any()
            continue
        a = Fraction(float(np.abs(x[i]).max()))
        for j in range(48):
            exact = round(Fraction(float(x[i, j])) * 127 / a) if a else 0  # rounds halves to even
            assert q[i, j] == exact
        assert s[i] == np.float32(float(a) / 127.0)


@pytest.mark.parametrize("kind,gated", [(ox.SILU, True), (ox.RELU, False)])
def test_int8_network_near_the_unquantized_one(kind, gated):
    rng = np.random.default_rng(2)
    d, h = 64, 96
    h1 = 2 * h if gated else h
    x, w1, w2 = rng.standard_normal((9, d)), rng.standard_normal((1, d, h1)) / 8, rng.standard_normal((1, h, d)) / 8
    b1, b2 = rng.standard_normal(h1), rng.standard_normal(d)
    q1, s1 = oi.quantize_weights(w1)
    q2, s2 = oi.quantize_weights(w2)
    y, bound = oi.network(x, q1[0], s1[0], b1, q2[0], s2[0], b2, kind, gated, 2.0 ** -8)
    full = ox.network(x, w1[0], b1, w2[0], b2, kind, gated, 0.0)["y_unrounded"][0]
    # four quantizations, each off by at most half of 1/127 of the largest value (3 to 4 times the
    # usual one): 0.4 % to 0.5 % of a usual term on the average of their squares; 4 % is far above
    assert np.sqrt(((y - full) ** 2).mean() / (full ** 2).mean()) < 0.04
    assert (bound < 0.05 * np.abs(full).max()).all()
