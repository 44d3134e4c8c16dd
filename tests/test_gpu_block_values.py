"""The block operators at values far from one, and at infinities, against the float64 oracle."""
import numpy as np
import pytest

from oracle import block as ob
from test_gpu_block import DEV, E, U, _dt, _gpu, _np, _tensor  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("act", ["silu", "gelu", "gelu_tanh"])
@pytest.mark.parametrize("size", [0, 4, 64, 70, 100])
def test_gate_activations_of_any_finite_size(size, act, dtype):
    """Gate projections of 2^e and -2^e, up projections of 2^-e: from 2^64 on the slopes have long reached 1 and 0, and
    nothing that is formed on the way may overflow. Powers of two make every product exact."""
    import torch
    from paper_2607_08754_amd import gated_ffn
    T, n, e = 70, 16, size
    ones = lambda *s: torch.ones(s, dtype=_dt(dtype), device=DEV)  # noqa: E731
    x, dy = ones(T, 1), ones(T, 1)
    wg, wu, wd = ones(n, 1) * 2.0 ** e, ones(n, 1) * 2.0 ** -e, ones(1, n) * 0.25
    wg[1::2] *= -1
    few = gated_ffn(x[:3], wg, wu, wd, act=act)
    leaves = [t.requires_grad_() for t in (x, wg, wu, wd)]
    y = gated_ffn(*leaves, act=act)
    got = [few, y, *torch.autograd.grad(y, leaves, dy)]
    xs, g, u, d, v = (_np(t) for t in (*leaves, dy))
    a, b = xs @ g.T, xs @ u.T
    f, s = ob.act_and_slope(a if e < 64 else np.zeros_like(a), act)
    if e >= 64:                                            # the limits, which double precision has reached as well
        f, s = np.maximum(a, 0.0), (a > 0) * 1.0
    dh, A = v @ d, np.abs
    da, db = dh * b * s, dh * f
    want = [(f * b)[:3] @ d.T, (f * b) @ d.T, da @ g + db @ u, da.T @ xs, db.T @ xs, v.T @ (f * b)]
    terms = [A(f * b)[:3] @ A(d).T, A(f * b) @ A(d).T, A(da) @ A(g) + A(db) @ A(u), A(da).T @ xs, A(db).T @ xs, v.T @ A(f * b)]
    for name, t, ref, top in zip(("few", "y", "x", "w_gate", "w_up", "w_down"), got, want, terms):
        t = _np(t)
        # activations off by 2^-17 relative (slopes by 2^-16 of 1), sums of 70 products at most by (6 * 70 + 29) 2^-24 <
        # 2^-15, and at most four roundings of u after each other
        assert (A(t - ref) <= (2.0 ** -13 + 4 * U[dtype]) * top + 2.0 ** -120).all(), (name, float(A(t - ref).max()))


@pytest.mark.parametrize("T", [20, 70])
@pytest.mark.parametrize("e", [90, 108, 112, 120, 125])
def test_fp32_weights_near_the_smallest_numbers(e, T):
    """Weights near 2^-e under activations near 2^e: as exact as at ordinary size down to 2^-110; below, the bf16 planes
    end at 2^-133 and a weight is off by half of that."""
    import torch
    from paper_2607_08754_amd import gated_ffn
    d, n, size = 72, 40, 2.0 ** e
    x = _tensor((T, d), "f32", 1) * size
    w = [_tensor((n, d), "f32", 2, d ** -0.5) / size, _tensor((n, d), "f32", 3, d ** -0.5) / size,
         _tensor((d, n), "f32", 4, n ** -0.5)]
    y = _np(gated_ffn(x, *w))
    x, wg, wu, wd = map(_np, (x, *w))
    A, r = np.abs, ob.ffn_forward(x, wg, wu, wd, "silu")
    gam = lambda k: (6 * k + 29) * E  # noqa: E731     (as in test_gpu_block.py)
    ea, eb = (gam(d) * (A(x) @ A(t).T) + 2.0 ** -134 * A(x).sum(1, keepdims=True) for t in (wg, wu))
    ef = 1.2 * ea + 2.0 ** -17 * A(r.f)
    eh = 1.1 * (A(r.b) * ef + A(r.f) * eb + ef * eb) + 2.0 ** -134
    tol = 1.1 * (eh @ A(wd).T + gam(n) * (A(r.h) @ A(wd).T)) + U["f32"] * A(r.y)
    assert (A(y - r.y) <= tol).all(), float((A(y - r.y) - tol).max())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T", [40, 70, 300])
def test_infinities_and_nans_stay_in_their_tokens(T, dtype):
    """Outputs and gradients of the other tokens are as they were; the token's own are not finite (in float32 from 65
    tokens on, and with gradients, a NaN where the formula has an infinity)."""
    import torch
    from paper_2607_08754_amd import gated_ffn
    d, n = 96, 72
    x, dy = _tensor((T, d), dtype, 1), _tensor((T, d), dtype, 2)
    w = [_tensor(s, dtype, 3 + i, 0.1) for i, s in enumerate(((n, d), (n, d), (d, n)))]

    def run(x):
        x = x.detach().requires_grad_()
        y = gated_ffn(x, *w)
        with torch.no_grad():
            alone = gated_ffn(x, *w)
        return [alone, y, torch.autograd.grad(y, x, dy)[0]]

    bad = x.clone()
    bad[7, 3], bad[20, 90], bad[33, 0] = float("nan"), float("inf"), float("-inf")
    rows = [i for i in range(T) if i not in (7, 20, 33)]
    for a, b in zip(run(x), run(bad)):
        assert torch.equal(a[rows], b[rows])
        for i in (7, 20, 33):
            assert not torch.isfinite(b[i]).all()


@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("e", [-61, -40, 0, 40, 56])
def test_norms_of_rows_of_any_size(e, dtype, kind):
    """Rows near 2^e without eps: their squares' sums are within fp32's range, and a power of two changes no rounding."""
    import torch
    from paper_2607_08754_amd import block_norm
    x, w, dz = _tensor((5, 300), dtype, 1), _tensor((300,), dtype, 2), _tensor((5, 300), dtype, 3)

    def run(scale):
        t = (x * scale).requires_grad_()
        z = block_norm(t, w, kind=kind, eps=0.0)
        return z, torch.autograd.grad(z, t, dz)[0] * scale

    for a, b in zip(run(1.0), run(2.0 ** e)):
        assert torch.equal(a, b)
