"""Transformations of the block operators that cannot see their kernels are refused,
before anything else is looked at: forward-mode derivatives and traces."""
import pytest
import torch
import torch.autograd.forward_ad as fw

from paper_2607_08754_amd import FeedForwardBlock, block_join, block_norm, dropout, gated_ffn

X = torch.randn(5, 16)
W = [torch.randn(s) for s in ((24, 16), (24, 16), (16, 24))]
V = torch.randn(16)
JOIN = ("f", "post_weight", "post_bias", "gate", "scale", "pre_weight", "pre_bias")


def _join_of(k):
    return lambda t: block_join(X, **{"f": X, k: t})[0]


ENTRIES = {
    "gated_ffn x": (X, lambda t: gated_ffn(t, *W)),
    "gated_ffn w_gate": (W[0], lambda t: gated_ffn(X, t, W[1], W[2])),
    "gated_ffn w_up": (W[1], lambda t: gated_ffn(X, W[0], t, W[2])),
    "gated_ffn w_down": (W[2], lambda t: gated_ffn(X, W[0], W[1], t)),
    "block_norm x": (X, lambda t: block_norm(t)),
    "block_norm weight": (V, lambda t: block_norm(X, t)),
    "block_norm bias": (V, lambda t: block_norm(X, None, t)),
    "block_join x": (X, lambda t: block_join(t, X)[0]),
    **{f"block_join {k}": (X if k == "f" else V, _join_of(k)) for k in JOIN},
    "dropout": (X, lambda t: dropout(t, 0.0, None)),
    "block": (X, FeedForwardBlock(16, 24, dtype=torch.float32)),
}


@pytest.mark.parametrize("leaf", [False, True])
@pytest.mark.parametrize("name", ENTRIES)
def test_forward_mode(name, leaf):
    t, fn = ENTRIES[name]
    with fw.dual_level():
        with pytest.raises(RuntimeError, match="forward-mode"):
            fn(fw.make_dual(t.clone().requires_grad_(leaf), torch.ones_like(t)))
        with pytest.raises(ValueError, match="GPU"):       # no tangent: an ordinary call
            fn(t)
    with pytest.raises(RuntimeError, match="forward-mode"):
        torch.func.jvp(fn, (t,), (t,))


@pytest.mark.parametrize("name", ENTRIES)
def test_traces(name):
    from torch.fx.experimental.proxy_tensor import make_fx
    t, fn = ENTRIES[name]
    for leaf in (False, True):
        with pytest.raises(RuntimeError, match="traced"):
            torch.jit.trace(fn, (t.clone().requires_grad_(leaf),), check_trace=False)
    with pytest.raises(RuntimeError, match="traced"):
        make_fx(fn)(t)
    with pytest.raises(ValueError, match="GPU"):
        fn(t)
