"""The block operators as programs use them beside plain eager calls: graphed callables,
two threads on streams of their own, compiled functions around them."""
import threading

import pytest

from test_gpu_block import DEV, _block, _gpu, _tensor  # noqa: F401

pytestmark = pytest.mark.gpu


def _pass(block, x, rng, dy):
    import torch
    leaves = [x, *block.parameters()]
    y = block(x, rng)
    return [y, *torch.autograd.grad(y, leaves, dy)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_graphed_callable(dtype):
    """make_graphed_callables captures forward and backward on their own and replays them around eager work."""
    import torch
    block, plain = _block(dtype), _block(dtype)
    x = _tensor((2, 70, 96), dtype, 1).requires_grad_()
    rng = torch.tensor([9, 100], dtype=torch.int64, device=DEV)
    graphed = torch.cuda.make_graphed_callables(block, (x.detach().clone().requires_grad_(), rng.clone()))
    for i in range(4):
        xi, dy = _tensor((2, 70, 96), dtype, 10 + i).requires_grad_(), _tensor((2, 70, 96), dtype, 20 + i)
        rng = rng + 3
        want = _pass(plain, xi, rng, dy)
        y = graphed(xi, rng)
        got = [y, *torch.autograd.grad(y, [xi, *block.parameters()], dy)]
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert torch.equal(a, b)


def test_two_threads():
    import torch
    cases = [("bf16", 1), ("f32", 2)]
    made = [(_block(d, seed=s), _tensor((3, 50, 96), d, s).requires_grad_(), torch.tensor([s, 4], dtype=torch.int64, device=DEV),
             _tensor((3, 50, 96), d, 5 + s)) for d, s in cases]
    want = [_pass(*m) for m in made]
    torch.cuda.synchronize()
    bad = []

    def work(i):
        try:
            with torch.cuda.stream(torch.cuda.Stream()):
                for _ in range(20):
                    if not all(torch.equal(a, b) for a, b in zip(_pass(*made[i]), want[i])):
                        bad.append(i)
        except Exception as e:                             # reported below
            bad.append(e)

    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not bad, bad


def test_inside_a_compiled_function():
    """The operators end a compiled graph and run as they are."""
    import torch
    from paper_2607_08754_amd import block_join, gated_ffn
    block = _block("f32", p=0.0)
    x, dy = _tensor((40, 96), "f32", 1).requires_grad_(), _tensor((40, 96), "f32", 2)
    w = [p.detach().requires_grad_() for p in block.matrices()]

    def f(x):
        y, z = block_join(x, gated_ffn(x * 2, *w), pre=True)
        return y + z

    leaves = [x, *w]
    compiled = torch.compile(f, backend="eager")
    with torch.no_grad():
        assert torch.equal(f(x), compiled(x))
    a, b = f(x), compiled(x)
    for s, t in zip([a, *torch.autograd.grad(a, leaves, dy)], [b, *torch.autograd.grad(b, leaves, dy)]):
        assert torch.equal(s, t)


def test_sites_of_any_size_and_factors_past_float32():
    """Sites count modulo 2^64, as the generator's offset does; a factor that float32 does not hold is refused."""
    import torch
    from paper_2607_08754_amd import block_join, block_norm, dropout
    x, f = _tensor((5, 40), "f32", 1), _tensor((5, 40), "f32", 2)
    rng = torch.tensor([9, 100], dtype=torch.int64, device=DEV)
    for fn in (lambda s: dropout(x, 0.5, rng, site=s), lambda s: block_join(x, f, p=0.5, rng=rng, site=s)[0]):
        want = fn(5)
        assert torch.equal(fn(5 + 2 ** 64), want) and torch.equal(fn(5 - 2 ** 64), want)
        assert torch.equal(fn(2 ** 63), fn(-2 ** 63)) and not torch.equal(fn(2 ** 63), want)
    for kw in (dict(alpha=1e39), dict(alpha=-1e300), dict(eps=1e39)):
        with pytest.raises(ValueError, match="eps must"):
            block_join(x, f, **kw)
    with pytest.raises(ValueError, match="eps must"):
        block_norm(x, eps=1e300)
    assert torch.isfinite(block_join(x, f, alpha=1e30)[0]).all()
