"""Transformations of the block operators that cannot see their kernels are refused:
a forward-mode derivative would come back without a tangent, a trace without the
launch that fills the outputs."""
import pytest

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


def _entries():
    import torch
    from paper_2607_08754_amd import FeedForwardBlock, block_join, block_norm, dropout, gated_ffn
    torch.manual_seed(0)
    w = [torch.randn(s, device=DEV) * 0.2 for s in ((24, 16), (24, 16), (16, 24))]
    f = torch.randn(5, 16, device=DEV)
    rng = torch.tensor([1, 2], dtype=torch.int64, device=DEV)
    block = FeedForwardBlock(16, 24, device=DEV, dtype=torch.float32)
    return {"gated_ffn": lambda x: gated_ffn(x, *w), "block_norm": lambda x: block_norm(x),
            "block_join": lambda x: block_join(x, f, pre=True)[1], "block_join f": lambda x: block_join(f, x)[0],
            "dropout": lambda x: dropout(x, 0.5, rng), "block": block}


def test_forward_mode_is_refused():
    import torch
    import torch.autograd.forward_ad as fw
    x = torch.randn(5, 16, device=DEV)
    for name, fn in _entries().items():
        for leaf in (False, True):
            with fw.dual_level():
                with pytest.raises(RuntimeError, match="forward-mode"):
                    fn(fw.make_dual(x.clone().requires_grad_(leaf), torch.ones_like(x)))
        with pytest.raises(RuntimeError):
            torch.func.jvp(fn, (x,), (torch.ones_like(x),))
        with pytest.raises((RuntimeError, ValueError)):     # (a mapped tensor has no memory of its own)
            torch.func.vmap(fn)(x.view(5, 1, 16))
        with fw.dual_level():                              # a plain tensor inside a dual level is an ordinary call
            y = fn(x)
        assert torch.equal(y, fn(x)), name


def test_traces_are_refused():
    import torch
    from torch.fx.experimental.proxy_tensor import make_fx
    x = torch.randn(5, 16, device=DEV)
    for fn in _entries().values():
        for leaf in (False, True):
            with pytest.raises(RuntimeError, match="traced"):
                torch.jit.trace(fn, (x.clone().requires_grad_(leaf),), check_trace=False)
        with torch.no_grad(), pytest.raises(RuntimeError, match="traced"):
            make_fx(fn)(x)
