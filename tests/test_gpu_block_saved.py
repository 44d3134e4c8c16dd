"""Gradients where the saved tensors come back laid out otherwise than they were saved:
offloaded to the host and back, or recomputed by a checkpoint."""
import pytest

from test_gpu_block import DEV, _gpu, _tensor  # noqa: F401

pytestmark = pytest.mark.gpu


def _operators(dtype):
    """Each operator on inputs that are slices of wider buffers: (function, leaves, output gradient)."""
    import torch
    from paper_2607_08754_amd import block_join, dropout, gated_ffn
    B, S, D, n = 3, 30, 40, 56
    wide = lambda seed, s=S: _tensor((B, s, 96), dtype, seed)[..., 8:8 + D]  # noqa: E731
    rng = torch.tensor([3, 4], dtype=torch.int64, device=DEV)
    v = [_tensor((D,), dtype, 20 + i, 0.2, 1.0) for i in range(5)]
    w = [_tensor(s, dtype, 30 + i, 0.2) for i, s in enumerate(((n, D), (n, D), (D, n)))]

    def join(x, f, gate, *v):
        return torch.cat(block_join(x, f, post_weight=v[0], post_bias=v[1], gate=gate, scale=v[2], pre_weight=v[3],
                                    pre_bias=v[4], kind="layer", p=0.3, rng=rng))

    dy = _tensor((B, S, D), dtype, 40)
    return {"ffn": (gated_ffn, [wide(1), *w], dy), "join": (join, [wide(2), wide(3), wide(4, 1), *v], torch.cat([dy, dy])),
            "dropout": (lambda x: dropout(x, 0.5, rng), [wide(5)], dy)}


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("op", ["ffn", "join", "dropout"])
def test_offloaded_and_recomputed(op, dtype):
    import torch
    from torch.utils.checkpoint import checkpoint
    fn, ins, dy = _operators(dtype)[op]
    leaves = [t.detach().requires_grad_() for t in ins]
    y = fn(*leaves)
    want = [y, *torch.autograd.grad(y, leaves, dy)]
    with torch.autograd.graph.save_on_cpu():
        y = fn(*leaves)
    got = [y, *torch.autograd.grad(y, leaves, dy)]
    y = checkpoint(fn, *leaves, use_reentrant=False)
    again = [y, *torch.autograd.grad(y, leaves, dy)]
    unaligned = lambda t: torch.cat([t.new_zeros(1), t.reshape(-1)])[1:].view(t.shape)  # noqa: E731
    with torch.autograd.graph.saved_tensors_hooks(lambda t: t, unaligned):
        y = fn(*leaves)
        moved = [y, *torch.autograd.grad(y, leaves, dy)]
    for a, b, c, d in zip(want, got, again, moved):
        assert torch.equal(a, b) and torch.equal(a, c) and torch.equal(a, d)
