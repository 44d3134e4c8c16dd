"""The feed-forward at values far from one, against the float64 oracle."""
import numpy as np
import pytest

from oracle import block as ob
from test_gpu_block import DEV, U, _dt, _gpu, _np  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("act", ["silu", "gelu", "gelu_tanh"])
@pytest.mark.parametrize("e", [0, 4, 64, 70, 100])
def test_gate_activations_of_any_finite_size(e, act, dtype):
    """Gate projections of 2^e and -2^e, up projections of 2^-e: from 2^64 on the slopes have long reached 1 and 0, and
    nothing that is formed on the way may overflow. Powers of two make every product exact."""
    import torch
    from paper_2607_08754_amd import gated_ffn
    T, n = 70, 16
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
    for name, t, ref, size in zip(("few", "y", "x", "w_gate", "w_up", "w_down"), got, want, terms):
        t = _np(t)
        # activations off by 2^-17 relative (slopes by 2^-16 of 1), sums of 70 products at most by (6 * 70 + 29) 2^-24 <
        # 2^-15, and at most four roundings of u after each other
        assert (A(t - ref) <= (2.0 ** -13 + 4 * U[dtype]) * size + 2.0 ** -120).all(), (name, float(A(t - ref).max()))
