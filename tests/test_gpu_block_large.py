"""GPU tests of the block operators at sizes where the feed-forward's launches are
cut in each of the ways they can be (256- and 128-tiles, whole, in parts along k,
and both in one launch), where a tensor's bytes pass 2^32, and for calls made in
unusual ways. Tolerances as in test_gpu_block.py, from its bounds()."""
import numpy as np
import pytest

from oracle import block as ob
from test_gpu_block import DEV, E, U, _ffn_inputs, _np, _rms, _tensor, bounds, check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T,d,n,dtype", [
    (2048, 1280, 3456, "bf16"), (7693, 590, 778, "bf16"), (12451, 133, 2700, "bf16"), (5533, 661, 2119, "bf16"),
    (11092, 781, 338, "bf16"), (761, 1070, 2337, "bf16"), (11325, 387, 644, "bf16"), (14365, 65, 526, "bf16"),
    (7386, 341, 1151, "f32"), (14592, 66, 2441, "f32"), (752, 386, 2756, "f32"), (13190, 1226, 203, "f32"),
    (13405, 518, 142, "f32"), (11069, 142, 1169, "f32")])
def test_ffn_cuts(T, d, n, dtype):
    import torch
    from paper_2607_08754_amd import gated_ffn
    act = ("silu", "gelu", "gelu_tanh")[(T + d + n) % 3]
    x, w, dy = _ffn_inputs(T, d, n, dtype, T)
    leaves = [t.requires_grad_() for t in (x, *w)]
    y = gated_ffn(x, *w, act=act)
    grads = torch.autograd.grad(y, leaves, dy)
    g, tol = bounds(*map(_np, (x, *w, dy)), act, dtype)
    terms = max(d, 2 * n, T)
    check("y", y, g.fwd.y, tol["y"], dtype, terms)
    for name, t in zip(("x", "w_gate", "w_up", "w_down"), grads):
        check(name, t, getattr(g, name), tol[name], dtype, terms)
    # one product in a launch of its own is cut in its own way
    one = gated_ffn(x, w[0], *(t.detach() for t in w[1:]), act=act)
    check("w_gate alone", torch.autograd.grad(one, w[0], dy)[0], g.w_gate, tol["w_gate"], dtype, terms)


@pytest.mark.parametrize("T,dtype", [(1200037, "bf16"), (600037, "f32")])
def test_ffn_past_32_bits(T, dtype):
    """The inner tensors pass 4 GiB: the first and last rows against the oracle, and dy zero between them, so that the
    weights' gradients are theirs alone."""
    import torch
    from paper_2607_08754_amd import gated_ffn
    d, n, k = 24, 1800, 64
    g = torch.Generator(device=DEV).manual_seed(5)
    _, w, _ = _ffn_inputs(1, d, n, dtype, 3)
    x = torch.randn(T, d, generator=g, device=DEV).to(w[0].dtype).requires_grad_()
    dy = torch.zeros_like(x)
    ends = list(range(k)) + list(range(T - k, T))
    with torch.no_grad():
        dy[ends] = _tensor((2 * k, d), dtype, 9)
    for t in w:
        t.requires_grad_()
    y = gated_ffn(x, *w)
    grads = torch.autograd.grad(y, [x, *w], dy)
    r, tol = bounds(_np(x[ends]), *map(_np, w), _np(dy[ends]), "silu", dtype)
    terms = 2 * n
    check("y", y[ends], r.fwd.y, tol["y"], dtype, terms)
    check("x", grads[0][ends], r.x, tol["x"], dtype, terms)
    assert not grads[0][k:T - k].any()
    for name, t in zip(("w_gate", "w_up", "w_down"), grads[1:]):
        check(name, t, getattr(r, name), tol[name], dtype, terms)


def test_join_past_32_bits():
    """Tensors of more than 2^31 elements: the last rows against a call on them alone, the vectors' gradients with
    gradients that are zero elsewhere."""
    import torch
    from paper_2607_08754_amd import block_join
    R, D, k = 1050001, 2056, 40
    x = torch.full((R, D), 0.5, dtype=torch.bfloat16, device=DEV)
    f, dy, dz = torch.zeros_like(x), torch.zeros_like(x), torch.zeros_like(x)
    for t, seed in ((x, 1), (f, 2), (dy, 3), (dz, 4)):
        t[R - k:] = _tensor((k, D), "bf16", seed)
    v = [_tensor((D,), "bf16", 5 + i, 0.2, 1.0).requires_grad_() for i in range(3)]

    def run(x, f, dy, dz):
        x, f = x.detach().requires_grad_(), f.detach().requires_grad_()
        y, z = block_join(x, f, post_weight=v[0], scale=v[1], pre_weight=v[2], eps=1e-5)
        return [y, z, *torch.autograd.grad([y, z], [x, f, *v], [dy, dz])]

    big, small = run(x, f, dy, dz), run(*(t[R - k:] for t in (x, f, dy, dz)))
    for a, b in zip(big[:4], small[:4]):
        assert torch.equal(a[R - k:], b)
    # the same terms in another order, some zero: fp32 sums of k terms and one rounding each
    for a, b in zip(big[4:], small[4:]):
        assert _rms(_np(a) - _np(b)) <= 2 * (U["bf16"] + (k + 40) * E) * _rms(_np(b))


def test_dropout_past_32_bits():
    import torch
    from paper_2607_08754_amd import dropout
    n, tail = (1 << 32) + 8 * 1000 + 5, 8 * 500 + 5
    x = torch.ones(n, dtype=torch.bfloat16, device=DEV)
    rng = torch.tensor([11, 13], dtype=torch.int64, device=DEV)
    y = dropout(x, 0.25, rng, site=2)
    first = n - tail
    want = ob.keep_mask(tail, 0.25, 11, 13, 2, first=first) * np.float32(ob.keep_factor(0.25))
    assert np.abs(_np(y[first:]) - want).max() <= U["bf16"] * 2
    assert (_np(y[first:]) != 0).tolist() == (want != 0).tolist()
    assert abs(float((y[: 1 << 20] != 0).float().mean()) - 0.75) < 0.01


def test_shared_tensors():
    """One tensor as several inputs: each use has its gradient, torch adds them."""
    import torch
    from paper_2607_08754_amd import block_join, gated_ffn
    x, w, dy = _ffn_inputs(70, 48, 64, "f32", 2)
    both, down = w[0].detach().requires_grad_(), w[2]
    got = torch.autograd.grad(gated_ffn(x, both, both, down), both, dy)[0]
    a, b = (w[0].detach().clone().requires_grad_() for _ in range(2))
    ga, gb = torch.autograd.grad(gated_ffn(x, a, b, down), [a, b], dy)
    assert torch.equal(got, ga + gb)
    x = x.detach().requires_grad_()
    v = _tensor((48,), "f32", 7).requires_grad_()
    y, z = block_join(x, x, post_weight=v, scale=v, pre_weight=v, gate=v)
    got = torch.autograd.grad([y, z], [x, v], [dy, dy])
    ins = [x.detach().clone().requires_grad_() for _ in range(2)] + [v.detach().clone().requires_grad_() for _ in range(4)]
    y2, z2 = block_join(ins[0], ins[1], post_weight=ins[2], scale=ins[3], pre_weight=ins[4], gate=ins[5])
    assert torch.equal(y, y2) and torch.equal(z, z2)
    g = torch.autograd.grad([y2, z2], ins, [dy, dy])
    for a, b in ((got[0], g[0] + g[1]), (got[1], sum(g[2:]))):
        # fp32 sums of two and four parts in any order
        assert float((a - b).abs().max()) <= 4 * E * float(sum(t.abs() for t in (g[:2] if a.dim() == 2 else g[2:])).max())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_weights_at_any_address(dtype):
    """Weights, vectors and activations as pieces of one buffer, at no multiple of 16 bytes."""
    import torch
    from paper_2607_08754_amd import block_join, gated_ffn
    T, d, n = 66, 41, 50
    x, w, dy = _ffn_inputs(T, d, n, dtype, 6)
    v = _tensor((d,), dtype, 8)
    flat = torch.cat([torch.zeros(1, dtype=x.dtype, device=DEV)] + [t.reshape(-1) for t in (x, *w, v, dy)])
    at, parts = 1, []
    for t in (x, *w, v, dy):
        parts.append(flat[at:at + t.numel()].view(t.shape))
        at += t.numel()
    assert any(t.data_ptr() % 16 for t in parts)

    def run(x, wg, wu, wd, v, dy):
        leaves = [t.detach().requires_grad_() for t in (x, wg, wu, wd, v)]
        y, z = block_join(leaves[0], gated_ffn(*leaves[:4]), pre_weight=leaves[4], post_weight=leaves[4])
        with torch.no_grad():
            alone = gated_ffn(*leaves[:4])
        return [y, z, alone, *torch.autograd.grad([y, z], leaves, [dy, dy])]

    for a, b in zip(run(*parts), run(x, *w, v, dy)):
        assert torch.equal(a, b)


def test_backward_twice():
    import torch
    from paper_2607_08754_amd import FeedForwardBlock
    torch.manual_seed(1)
    block = FeedForwardBlock(64, 96, post=True, scale=0.5, p=0.3, device=DEV)
    rng = torch.tensor([3, 4], dtype=torch.int64, device=DEV)
    x, dy = _tensor((90, 64), "bf16", 1).requires_grad_(), _tensor((90, 64), "bf16", 2)
    y = block(x, rng)
    first = torch.autograd.grad(y, [x, *block.parameters()], dy, retain_graph=True)
    for a, b in zip(first, torch.autograd.grad(y, [x, *block.parameters()], dy)):
        assert torch.equal(a, b)


def test_captured_backward_into_grad():
    """backward() into .grad captured once, replayed with the program's own work between: the accumulated gradients."""
    import gc

    import torch
    from paper_2607_08754_amd import FeedForwardBlock
    torch.manual_seed(2)
    block = FeedForwardBlock(64, 96, post=True, device=DEV, dtype=torch.float32)
    x, dy = _tensor((80, 64), "f32", 1), _tensor((80, 64), "f32", 2)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        block(x).backward(dy)
    torch.cuda.current_stream().wait_stream(side)
    want = [p.grad.clone() for p in block.parameters()]
    block.zero_grad(set_to_none=True)
    gc.collect()                                           # no eager graph lives on
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        block(x).backward(dy)
    for k in range(3):
        for p in block.parameters():
            p.grad.fill_(1.0)
        graph.replay()
        torch.cuda.synchronize()
        for p, w in zip(block.parameters(), want):
            assert torch.equal(p.grad, w)                  # the captured first backward writes .grad anew
        with torch.no_grad():
            gated = block(x)
        assert bool(torch.isfinite(gated).all())


def test_gradients_are_differentiable_once():
    """create_graph gives the gradients; differentiating them again is refused."""
    import torch
    from paper_2607_08754_amd import block_join, dropout, gated_ffn
    x, w, dy = _ffn_inputs(20, 24, 32, "f32", 4)
    x = x.requires_grad_()
    rng = torch.tensor([1, 2], dtype=torch.int64, device=DEV)
    for f in (lambda: gated_ffn(x, *w), lambda: block_join(x, x * 2, pre=True)[1], lambda: dropout(x, 0.5, rng)):
        want = torch.autograd.grad(f(), x, dy)[0]
        got = torch.autograd.grad(f(), x, dy, create_graph=True)[0]
        assert torch.equal(got, want)
        with pytest.raises(RuntimeError, match="once only"):
            got.sum().backward()


@pytest.mark.parametrize("T,dtype", [(1, "bf16"), (16, "bf16"), (17, "bf16"), (40, "bf16"), (64, "f32")])
def test_ffn_few_tokens_of_wide_layers(T, dtype):
    """Either side of the size from which a few tokens take the tiles."""
    from paper_2607_08754_amd import gated_ffn
    d, n = 1800, 6001
    x, w, dy = _ffn_inputs(T, d, n, dtype, T)
    g, tol = bounds(*map(_np, (x, *w, dy)), "silu", dtype)
    check("y", gated_ffn(x, *w), g.fwd.y, tol["y"], dtype, max(d, n))
