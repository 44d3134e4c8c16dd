"""CPU pins of the oracle of the block operators: published generator vectors,
gradients against central differences in float64, closed forms."""
import math

import numpy as np
import pytest

from oracle import block as ob

H = 1e-6


def _rand(*shape, seed=0, std=1.0):
    return np.random.default_rng([seed, *shape]).standard_normal(shape) * std


def _differences(fn, t):
    """Central differences of the scalar fn over the array t (changed in place and restored)."""
    g = np.empty_like(t)
    for i in np.ndindex(*t.shape):
        v = t[i]
        t[i] = v + H
        hi = fn()
        t[i] = v - H
        lo = fn()
        t[i] = v
        g[i] = (hi - lo) / (2 * H)
    return g


@pytest.mark.parametrize("counter,key,want", [
    # the known answers published with the generator
    ((0, 0, 0, 0), (0, 0), (0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8)),
    ((0xFFFFFFFF,) * 4, (0xFFFFFFFF,) * 2, (0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD)),
    ((0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344), (0xA4093822, 0x299F31D0),
     (0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1)),
])
def test_generator_known_answers(counter, key, want):
    got = ob.philox([np.array([w]) for w in counter], key)
    assert tuple(int(w[0]) for w in got) == want


def test_keep_rate_and_independence():
    n, p = 1 << 16, 0.25
    m = ob.keep_mask(n, p, 1234, 5)
    # binomial: five standard deviations
    assert abs(m.mean() - 0.75) < 5 * math.sqrt(0.25 * 0.75 / n)
    assert np.array_equal(m, ob.keep_mask(n, p, 1234, 2, site=3))         # offset + site
    assert np.array_equal(m[:1001], ob.keep_mask(1001, p, 1234, 5))       # a prefix
    for other in (ob.keep_mask(n, p, 1235, 5), ob.keep_mask(n, p, 1234, 6)):
        assert abs((m == other).mean() - (0.75 ** 2 + 0.25 ** 2)) < 5 * math.sqrt(0.25 / n)
    assert ob.keep_mask(n, 0.0, 1, 1).all()
    assert math.isclose(ob.keep_factor(0.25), 4 / 3)


@pytest.mark.parametrize("act", ["silu", "gelu", "gelu_tanh"])
def test_activation_slopes(act):
    a = np.linspace(-6, 6, 49)
    f = lambda t: ob.act_and_slope(t, act)[0]
    # truncation H^2 |act'''| / 6 and cancellation 2^-52 |act| / H
    assert np.allclose(ob.act_and_slope(a, act)[1], (f(a + H) - f(a - H)) / (2 * H), rtol=0, atol=1e-8)


@pytest.mark.parametrize("act", ["silu", "gelu", "gelu_tanh"])
def test_ffn_gradients(act):
    x, wg, wu, wd, dy = _rand(3, 5), _rand(7, 5, seed=1), _rand(7, 5, seed=2), _rand(5, 7, seed=3), _rand(3, 5, seed=4)
    loss = lambda: float((ob.ffn_forward(x, wg, wu, wd, act).y * dy).sum())
    g = ob.ffn_backward(dy, x, wg, wu, wd, act)
    for name, t in (("x", x), ("w_gate", wg), ("w_up", wu), ("w_down", wd)):
        assert np.allclose(getattr(g, name), _differences(loss, t), rtol=0, atol=1e-7), name


@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("post,pre", [(True, True), (False, True), (True, False)])
@pytest.mark.parametrize("gate_rows", [0, 1, 2, 4])
def test_join_gradients(kind, post, pre, gate_rows):
    x, f, dy, dz = (_rand(4, 6, seed=i) for i in range(4))
    w1, b1, sc, w2, b2 = (_rand(6, seed=10 + i) for i in range(5))
    gate = _rand(gate_rows, 6, seed=20) if gate_rows else None
    drop = ob.keep_mask(24, 0.3, 7, 9).reshape(4, 6) * ob.keep_factor(0.3)
    t = dict(w1=w1 if post else None, b1=b1 if post else None, gate=gate, scale=sc, w2=w2 if pre else None,
             b2=b2 if pre else None)

    def loss():
        r = ob.join_forward(x, f, kind, 1e-3, post, pre, 0.7, drop=drop, **t)
        return float((r.y * dy).sum() + ((r.z * dz).sum() if pre else 0.0))

    g = ob.join_backward(dy, dz, x, f, kind, 1e-3, post, pre, 0.7, drop=drop, **t)
    names = dict(x=x, f=f, post_weight=t["w1"], post_bias=t["b1"], gate=gate, scale=sc, pre_weight=t["w2"],
                 pre_bias=t["b2"])
    for name, arr in names.items():
        if arr is not None:
            assert np.allclose(g[name], _differences(loss, arr), rtol=0, atol=1e-6), name


def test_norm_closed_forms():
    r = ob.join_forward(np.full((2, 8), 3.0), None, "rms", 0.0, False, True)
    assert np.allclose(r.z, 1.0, rtol=0, atol=1e-15)
    t = _rand(3, 9)
    z = ob.join_forward(t, None, "layer", 0.0, False, True).z
    assert np.allclose(z.mean(1), 0, atol=1e-14) and np.allclose((z * z).mean(1), 1, atol=1e-14)
