"""GPU tests of the joins' norms with any of their vectors absent, forward and
backward, against the float64 oracle: every subset of the two weights and the two
biases, for both kinds of norm, at widths that fill a block's columns (512, 4096,
8192) and at widths that do not. dz has a mean of one, so that what a column past
the row's end would add to a row's mean is far above the tolerances, which are
those of test_gpu_block.py."""
import itertools

import pytest

from test_gpu_block import DEV, _gpu, _join_check, _tensor  # noqa: F401

pytestmark = pytest.mark.gpu

VECTORS = ("post_weight", "post_bias", "pre_weight", "pre_bias")
SUBSETS = [c for n in range(5) for c in itertools.combinations(VECTORS, n)]


def _case(shape, dtype, given, post=True, pre=True, gate="none", scale=False, kind="layer", p=0.0):
    import torch
    B, S, D = shape
    t = {"x": _tensor(shape, dtype, 1, 2.0, 0.25), "f": _tensor(shape, dtype, 2, 0.5, -0.1)}
    gates = {"none": None, "channel": (D,), "batch": (B, 1, D), "token": shape}[gate]
    t["gate"] = None if gates is None else _tensor(gates, dtype, 3)
    t["scale"] = _tensor((D,), dtype, 4) if scale else None
    for i, name in enumerate(VECTORS):
        std, mean = ((0.2, 1.0), (0.3, 0.0))[i % 2]
        t[name] = _tensor((D,), dtype, 5 + i, std, mean) if name in given else None
    rng = torch.tensor([99, 7], dtype=torch.int64, device=DEV)
    kw = dict(kind=kind, eps=1e-5, p=p, rng=rng if p else None, site=1, alpha=0.7, post=post, pre=pre)
    return t, kw, _tensor(shape, dtype, 10), _tensor(shape, dtype, 11, 1.0, 1.0) if pre else None


def _run(dtype, *args, **kw):
    t, kw, dy, dz = _case(*args, **kw)
    _join_check(t, kw, dy, dz, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kind", ["layer", "rms"])
@pytest.mark.parametrize("D", [13, 512, 768, 1001, 4096, 4104, 8191, 8192])
def test_norms_without_some_of_their_vectors(D, kind, dtype):
    for given in SUBSETS:
        _run(dtype, (2, 3, D), dtype, given, kind=kind)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kind", ["layer", "rms"])
@pytest.mark.parametrize("gate,scale,p", [("none", True, 0.0), ("none", False, 0.25), ("channel", False, 0.0),
                                          ("batch", False, 0.1), ("token", False, 0.0), ("token", True, 0.3)])
def test_gates_scales_and_dropout_beside_absent_vectors(gate, scale, p, kind, dtype):
    for D in (200, 1280, 4999):
        for given in ((), ("post_bias",), ("pre_bias",), ("post_weight", "pre_bias")):
            _run(dtype, (3, 5, D), dtype, given, gate=gate, scale=scale, p=p, kind=kind)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kind", ["layer", "rms"])
@pytest.mark.parametrize("post,pre", [(True, False), (False, True), (False, False)])
def test_one_norm_without_vectors(post, pre, kind, dtype):
    for D in (24, 1280, 4104):
        for scale in (False, True):
            _run(dtype, (2, 4, D), dtype, (), post=post, pre=pre, scale=scale, kind=kind)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kind", ["layer", "rms"])
def test_gate_rows_of_many_sequences_without_vectors(kind, dtype):
    """More gate rows than blocks, so that a block takes several."""
    for given in ((), ("post_bias", "pre_bias")):
        _run(dtype, (4100, 2, 40), dtype, given, gate="batch", kind=kind)
        _run(dtype, (530, 2, 4104), dtype, given, gate="batch", kind=kind)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kind", ["layer", "rms"])
@pytest.mark.parametrize("shape", [(257, 2, 4097), (600, 3, 4104), (60, 4, 8192), (3, 2, 5000)])
def test_gate_rows_of_wide_rows(shape, kind, dtype):
    """Rows of two pieces per thread under a gate row for each few of them: blocks of one gate row and of several, with
    dropout and every vector, and with the gate alone; no gradient but the gate's."""
    import torch
    from paper_2607_08754_amd import block_join
    _run(dtype, shape, dtype, VECTORS, gate="batch", scale=True, kind=kind, p=0.2)
    t, kw, dy, dz = _case(shape, dtype, (), gate="batch", kind=kind)
    _join_check(t, kw, dy, dz, dtype)
    full = {k: v for k, v in t.items() if v is not None}
    y, z = block_join(**full, **kw)
    want = torch.autograd.grad([y, z], full["gate"], [dy, dz])[0]
    alone = full["gate"].detach().requires_grad_()
    y, z = block_join(**{k: alone if k == "gate" else v.detach() for k, v in full.items()}, **kw)
    assert torch.equal(torch.autograd.grad([y, z], alone, [dy, dz])[0], want)


@pytest.mark.parametrize("kind", ["layer", "rms"])
@pytest.mark.parametrize("D", [1, 7, 96, 513, 1280, 4097])
def test_block_norm_without_vectors(D, kind):
    """The norm alone against its definition in 64 bits: each of weight and bias there or not."""
    import torch
    from paper_2607_08754_amd import block_norm
    if kind == "layer" and D == 1:
        D = 2
    x, dz = _tensor((9, D), "f32", 1, 2.0, 0.5), _tensor((9, D), "f32", 2, 1.0, 1.0)
    for w, b in itertools.product((None, _tensor((D,), "f32", 3, 0.2, 1.0)), (None, _tensor((D,), "f32", 4))):
        leaves = [t.detach().requires_grad_() for t in (x, w, b) if t is not None]
        it = iter(leaves[1:])
        z = block_norm(leaves[0], None if w is None else next(it), None if b is None else next(it), kind=kind)
        got = [z, *torch.autograd.grad(z, leaves, dz)]
        wide = [t.detach().double().requires_grad_() for t in leaves]
        it = iter(wide[1:])
        c = wide[0] - wide[0].mean(1, keepdim=True) if kind == "layer" else wide[0]
        r = (c.square().mean(1, keepdim=True) + 1e-5).rsqrt()
        ref = c * r * (1.0 if w is None else next(it)) + (0.0 if b is None else next(it))
        want = [ref, *torch.autograd.grad(ref, wide, dz.double())]
        top = lambda t: t.abs().amax(1, keepdim=True)  # noqa: E731
        g = dz.double() * (1.0 if w is None else w.double())
        # 2^-16 of a row's (a column's) largest terms, as for the joins
        size = [top(ref) + top(c * r), 4 * r * top(g) + top(want[1])]
        size += [(dz.double().abs() * top(c * r)).sum(0) + dz.double().abs().sum(0)] * 2
        for a, e, s in zip(got, want, size):
            assert bool(((a.double() - e).abs() <= 2.0 ** -16 * s).all())
