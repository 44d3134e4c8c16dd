"""Saved tensors of the block operators that come back laid out otherwise than they were
saved (saved_tensors_hooks may return any tensor of the same values): the backward
calls read no byte outside of what came back, and what came back with another shape,
type or device is refused. On the CPU: the library is replaced by one that checks
the spans of the buffers it is given."""
import contextlib

import pytest
import torch

from paper_2607_08754_amd import _lib, block


class Library:
    """Takes the calls and checks that each input's rows lie within the storage at its address."""

    def __init__(self):
        self.room = {}                     # address -> bytes from it to its storage's end
        self.calls = []

    def add(self, t):
        st = t.untyped_storage()
        self.room[t.data_ptr()] = st.data_ptr() + st.nbytes() - t.data_ptr()
        return t

    def rows(self, ptr, n, width, ld, name):
        if ptr:
            assert ptr in self.room, f"{name}: not a tensor's address"
            assert ((n - 1) * (ld or width) + width) * 4 <= self.room[ptr], f"{name}: rows {ld} apart leave the tensor"

    def slorr_ffn_sizes(self, d, *sizes):
        for s in sizes:
            if s is not None:
                s.value = 4096
        return 0

    def slorr_ffn_forward(self, d, *a):
        return 0

    def slorr_ffn_backward(self, d, dy, x, wg, wu, wd, state, *a):
        self.calls.append("ffn")
        self.rows(x, d.tokens, d.dim, d.ldx, "x")
        for w in (wg, wu, wd):
            self.rows(w, 1, d.dim * d.inner, 0, "weight")
        return 0

    def slorr_join_workspace(self, d, n):
        n.value = 4096
        return 0

    def slorr_join_forward(self, d, *a):
        return 0

    def slorr_join_backward(self, d, t, *a):
        self.calls.append("join")
        self.rows(t.x, d.rows, d.dim, d.ldx, "x")
        self.rows(t.f, d.rows, d.dim, d.ldf, "f")
        self.rows(t.gate, d.gate_rows, d.dim, d.ld_gate, "gate")
        for name in ("post_weight", "post_bias", "scale", "pre_weight", "pre_bias"):
            self.rows(getattr(t, name), 1, d.dim, 0, name)
        return 0

    def slorr_dropout(self, *a):
        self.calls.append("dropout")
        return 0


@pytest.fixture
def lib(monkeypatch):
    stand_in = Library()
    monkeypatch.setattr(block, "lib", lambda: stand_in)
    monkeypatch.setattr(block, "_device", lambda t: contextlib.nullcontext())
    monkeypatch.setattr(block, "_stream", lambda t: 0)
    return stand_in


def hooks(lib, unpack):
    return torch.autograd.graph.saved_tensors_hooks(lambda t: t, lambda t: lib.add(unpack(t)))


LAYOUTS = {
    "as saved": lambda t: t,
    "contiguous": lambda t: t.contiguous().clone(),
    "columns": lambda t: t if t.dim() < 2 or t.dtype != torch.float32 else t.t().contiguous().t() if t.dim() == 2 else t,
    "unaligned": lambda t: torch.cat([t.new_zeros(1), t.reshape(-1)])[1:].view(t.shape) if t.dtype == torch.float32 else t,
}


def ffn_pass(lib):
    x = torch.randn(6, 40)[:, :16].requires_grad_()
    w = [torch.randn(s).requires_grad_() for s in ((24, 16), (24, 16), (16, 24))]
    y = block._GatedFfn.apply(x, *w, _lib.SILU)
    torch.autograd.grad(y, [x, *w], torch.ones_like(y))


def join_pass(lib):
    D = 16
    x, f = (torch.randn(6, 40)[:, :D].requires_grad_() for _ in range(2))
    gate = torch.randn(3, 64)[:, :D].requires_grad_()
    v = [torch.randn(D).requires_grad_() for _ in range(5)]
    d = block._Call(6, D, _lib.F32, _lib.LAYER, _lib.JOIN_POST | _lib.JOIN_PRE, 3, 1e-5, 1.0, 0.5, 0)
    rng = torch.zeros(2, dtype=torch.int64)
    y, z = block._Join.apply(d, rng, x, f, v[0], v[1], gate, v[2], v[3], v[4])
    torch.autograd.grad([y, z], [x, f, gate, *v], [torch.ones_like(y)] * 2)


def dropout_pass(lib):
    x = torch.randn(6, 16).requires_grad_()
    y = block._Dropout.apply(x, 0.5, torch.zeros(2, dtype=torch.int64), 0)
    torch.autograd.grad(y, x, torch.ones_like(y))


PASSES = {"ffn": ffn_pass, "join": join_pass, "dropout": dropout_pass}


@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("op", PASSES)
def test_saved_tensors_in_other_layouts(lib, op, layout, monkeypatch):
    for name in ("_rows", "_aligned", "_at16"):            # copies that the backward makes are tensors as well
        if hasattr(block, name):
            fn = getattr(block, name)

            def wrapped(*a, fn=fn):
                r = fn(*a)
                lib.add(r[0] if isinstance(r, tuple) else r)
                return r

            monkeypatch.setattr(block, name, wrapped)
    with hooks(lib, LAYOUTS[layout]):
        PASSES[op](lib)
    assert lib.calls[-1] == op


WRONG = {
    "type": lambda t: t.to(torch.bfloat16) if t.dtype == torch.float32 else t.to(torch.int32) if t.dtype == torch.int64 else t,
    "shape": lambda t: t[:1].clone(),
    "device": lambda t: t.to("meta"),                      # (no memory)
}


@pytest.mark.parametrize("what", WRONG)
@pytest.mark.parametrize("op", PASSES)
def test_other_saved_tensors_are_refused(lib, op, what):
    n = len(lib.calls)
    with torch.autograd.graph.saved_tensors_hooks(lambda t: t, WRONG[what]):
        with pytest.raises((RuntimeError, ValueError), match="saved tensor|no memory"):
            PASSES[op](lib)
    assert [c for c in lib.calls[n:] if c != "dropout"] == [] and lib.calls[n:].count("dropout") <= 1


@pytest.mark.parametrize("create", [False, True])
def test_a_tangent_of_the_output_gradient_is_refused(lib, create):
    import torch.autograd.forward_ad as fw
    x = torch.randn(6, 16).requires_grad_()
    y = block._Dropout.apply(x, 0.5, torch.zeros(2, dtype=torch.int64), 0)
    with fw.dual_level(), pytest.raises(RuntimeError, match="forward-mode"):
        torch.autograd.grad(y, x, fw.make_dual(torch.ones_like(y), torch.ones_like(y)), create_graph=create)


def test_tensors_without_memory_are_refused(lib):
    """A vector whose storage was released is not an absent one."""
    x = torch.randn(6, 16)
    v = torch.randn(16)
    v.untyped_storage().resize_(0)
    d = block._Call(6, 16, _lib.F32, _lib.LAYER, _lib.JOIN_PRE, 0, 1e-5, 1.0, 0.0, 0)
    with pytest.raises(ValueError, match="no memory"):
        block._join_run(d, x.shape, *block._join_layout(16, (x, None, None, None, None, None, v, None)), None)
