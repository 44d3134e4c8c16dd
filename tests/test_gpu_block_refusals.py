"""What the Python entries of a regularised block's operators refuse, each before
any kernel runs."""
import pytest

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


@pytest.fixture(scope="module")
def t():
    import torch
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU")
    return lambda *shape, dtype=torch.bfloat16, device=DEV: torch.zeros(shape, dtype=dtype, device=device)


def test_gated_ffn(t):
    import torch
    from paper_2607_08754_amd import gated_ffn
    x, g, d = t(4, 16), t(24, 16), t(16, 24)

    def refused(match, *args, **kw):
        with pytest.raises(ValueError, match=match):
            gated_ffn(*args, **kw)

    refused("act must", x, g, g, d, act="relu")
    refused("last dimension", t(4, 0), t(24, 0), t(24, 0), t(0, 24))
    refused("last dimension", t(), g, g, d)
    refused("w_gate must be a matrix", x, t(16), g, d)
    refused("w_gate must be a matrix", x, t(0, 16), t(0, 16), t(16, 0))
    refused("w_gate must be a matrix", x, None, g, d)
    for name, i in (("w_gate", 1), ("w_up", 2), ("w_down", 3)):
        args = [x, g, g, d]
        for bad in (args[i].float(), args[i].cpu(), t(24, 24)):
            args[i] = bad
            refused(f"{name} must" if bad.shape != (24, 24) or i != 1 else "must be", *args)
        args[i] = [g, g, d][i - 1].t().contiguous().t()
        refused(f"{name} must be contiguous", *args)
    refused("w_up must", x, g, None, d)
    refused("w_down must", x, g, g, d.t().contiguous())
    refused("x must be a float32", x.half(), g, g, d)
    with torch.no_grad():
        refused("w_up must", x, g, t(23, 16), d)


def test_block_join(t):
    import torch
    from paper_2607_08754_amd import block_join, block_norm
    x, v = t(2, 3, 16), t(16)
    rng = torch.zeros(2, dtype=torch.int64, device=DEV)

    def refused(match, *args, fn=block_join, **kw):
        with pytest.raises(ValueError, match=match):
            fn(*args, **kw)

    refused("f is required", x, None)
    for bad in (t(3, 16), x.float(), x.cpu(), 3):
        refused("f must", x, bad)
    for name in ("post_weight", "post_bias", "scale", "pre_weight", "pre_bias"):
        for bad in (t(15), t(1, 16), v.float(), v.cpu(), t(32)[::2], 1.0):
            refused(f"{name} must", x, x, **{name: bad})
    for name in ("weight", "bias"):
        refused(f"pre_{name} must", x, fn=block_norm, **{name: t(8)})
    for bad in (t(2, 16), t(1, 3, 16), t(2, 2, 16), t(2, 3, 1, 16), t(2, 3, 1), v.float(), v.cpu(), t(), 2.0):
        refused("gate must", x, x, gate=bad)
    refused("post=False", x, x, post=False, post_weight=v)
    refused("post=False", x, x, post=False, post_bias=v)
    refused("pre=False", x, x, pre=False, pre_weight=v)
    refused("pre=False", x, x, pre=False, pre_bias=v)
    refused("kind must", x, x, kind="batch")
    refused("kind must", x, fn=block_norm, kind="l2")
    refused("at most 8192", t(1, 8193), t(1, 8193))
    refused("at most 8192", t(1, 8193), fn=block_norm)
    for kw in (dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")), dict(alpha=float("nan")),
               dict(alpha=float("inf"))):
        refused("eps must", x, x, **kw)
    for p in (-0.1, 1.0, 1 - 2.0 ** -18, float("nan")):
        refused("p must", x, x, p=p, rng=rng)
    refused("dropout needs rng", x, x, p=0.5)
    for bad in (rng.int(), rng.cpu(), torch.zeros(3, dtype=torch.int64, device=DEV),
                torch.zeros(4, dtype=torch.int64, device=DEV)[::2], 5):
        refused("rng must", x, x, p=0.5, rng=bad)


def test_dropout(t):
    import torch
    from paper_2607_08754_amd import dropout
    x, rng = t(3, 16), torch.zeros(2, dtype=torch.int64, device=DEV)
    for p in (-0.1, 1.0, 1 - 2.0 ** -18, float("nan")):
        with pytest.raises(ValueError, match="p must"):
            dropout(x, p, rng)
    with pytest.raises(ValueError, match="dropout needs rng"):
        dropout(x, 0.5, None)
    with pytest.raises(ValueError, match="rng must"):
        dropout(x, 0.5, rng.cpu())
    with pytest.raises(ValueError, match="x must"):
        dropout(x.half(), 0.5, rng)


def test_block_without_rng(t):
    import torch
    from paper_2607_08754_amd import FeedForwardBlock
    block = FeedForwardBlock(16, 24, p=0.5, device=DEV)
    with pytest.raises(ValueError, match="dropout needs rng"):
        block(t(2, 16))
    with torch.no_grad():
        assert block.eval()(t(2, 16)).shape == (2, 16)       # no dropout: none needed
