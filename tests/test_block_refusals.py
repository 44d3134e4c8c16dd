"""What the operators of a regularised block refuse, on the CPU: every argument
error of their C entries is reported before anything touches a device (the
buffers below are host memory that no call may reach), and the Python entries
that can be refused without a GPU."""
import ctypes

import pytest
import torch

INVALID, UNSUPPORTED, WORKSPACE = 1, 2, 4


@pytest.fixture(scope="module")
def L():
    import paper_2607_08754_amd._lib as lib_mod
    return lib_mod


@pytest.fixture(scope="module")
def arena():
    """Addresses 1 MiB apart, 256-byte aligned."""
    buf = ctypes.create_string_buffer(40 << 20)
    base = (ctypes.addressof(buf) + 255) & ~255
    yield lambda i: base + (i << 20)
    del buf


def status(L, st, code, text=""):
    assert st == code, (st, L.lib().slorr_last_error())
    if code:
        assert text in L.lib().slorr_last_error().decode(), L.lib().slorr_last_error()


def test_status_codes(L):
    names = [L.lib().slorr_status_string(c).decode() for c in (INVALID, UNSUPPORTED, WORKSPACE)]
    assert [n.split("_", 2)[-1] for n in names] == ["INVALID_ARGUMENT", "UNSUPPORTED", "WORKSPACE"], names


def ffn(L, tokens=4, dim=16, inner=24, dtype=0, act=0, ldx=0, lddy=0):
    return L.Ffn(tokens, dim, inner, dtype, act, ldx, lddy)


@pytest.mark.parametrize("change,code,text", [
    (dict(dtype=7), UNSUPPORTED, "dtype"), (dict(act=3), UNSUPPORTED, "act"), (dict(act=-1), UNSUPPORTED, "act"),
    (dict(tokens=-1), INVALID, "tokens"), (dict(dim=0), INVALID, "dim"), (dict(inner=0), INVALID, "inner"),
    (dict(dim=-8), INVALID, "dim"), (dict(tokens=1 << 31), UNSUPPORTED, "limits"),
    (dict(dim=(1 << 20) + 1), UNSUPPORTED, "limits"), (dict(inner=(1 << 20) + 1), UNSUPPORTED, "limits"),
    (dict(tokens=1 << 30, dim=1 << 20), UNSUPPORTED, "limit"),
    (dict(ldx=15), INVALID, "stride"), (dict(lddy=15), INVALID, "stride"), (dict(ldx=-16), INVALID, "stride"),
    (dict(ldx=1 << 22), UNSUPPORTED, "stride"), (dict(lddy=1 << 22), UNSUPPORTED, "stride"),
])
def test_ffn_shapes(L, arena, change, code, text):
    lib, d = L.lib(), ffn(L, **change)
    a = [arena(i) for i in range(12)]
    n = ctypes.c_size_t()
    status(L, lib.slorr_ffn_sizes(d, n, n, n), code, text)
    status(L, lib.slorr_ffn_forward(d, *a[:6], a[6], 1 << 20, None), code, text)
    status(L, lib.slorr_ffn_backward(d, *a[:10], a[10], 1 << 20, None), code, text)


def test_ffn_sizes(L):
    lib = L.lib()
    st, f, b = ctypes.c_size_t(), ctypes.c_size_t(), ctypes.c_size_t()
    status(L, lib.slorr_ffn_sizes(None, st, f, b), INVALID, "NULL")
    status(L, lib.slorr_ffn_sizes(ffn(L), None, None, None), 0)
    for dtype in (0, 1):
        status(L, lib.slorr_ffn_sizes(ffn(L, tokens=0, dtype=dtype), st, f, b), 0)
        assert min(st.value, f.value, b.value) > 0
        last = 0
        for tokens in (1, 100, 10000, 1000000):                # room grows with the work
            status(L, lib.slorr_ffn_sizes(ffn(L, tokens=tokens, dtype=dtype), st, f, b), 0)
            elem = 4 if dtype == 0 else 2
            assert st.value >= 2 * tokens * 24 * elem and b.value >= 3 * tokens * 24 * 2 and f.value >= tokens * 24 * 2
            assert b.value >= last
            last = b.value


@pytest.mark.parametrize("dtype", [0, 1])
def test_ffn_buffers(L, arena, dtype):
    lib, d = L.lib(), ffn(L, dtype=dtype)
    st, f, b = ctypes.c_size_t(), ctypes.c_size_t(), ctypes.c_size_t()
    status(L, lib.slorr_ffn_sizes(d, st, f, b), 0)
    names = ["x", "w_gate", "w_up", "w_down", "y", "state"]

    def forward(code, text, ws=arena(9), have=f.value, **new):
        p = [new.get(k, arena(i)) for i, k in enumerate(names)]
        status(L, lib.slorr_ffn_forward(d, *p, ws, have, None), code, text)

    for k in names:
        if k != "state":
            forward(INVALID, f"{k} is NULL", **{k: None})
        forward(INVALID, f"{k} must be 16-byte aligned", **{k: arena(20) + 8})
    for k in names[:4]:
        forward(INVALID, "overlap", y=arena(names.index(k)))
        forward(INVALID, "overlap", state=arena(names.index(k)) + 32)
        forward(INVALID, "overlap", ws=arena(names.index(k)))
    forward(INVALID, "overlap", y=arena(5) - 16)
    forward(WORKSPACE, "NULL", ws=None)
    forward(WORKSPACE, "aligned", ws=arena(9) + 128)
    forward(WORKSPACE, "too small", have=f.value - 1)

    back = ["dy", "x", "w_gate", "w_up", "w_down", "state", "dx", "dw_gate", "dw_up", "dw_down"]

    def backward(code, text, ws=arena(12), have=b.value, **new):
        p = [new.get(k, arena(i)) for i, k in enumerate(back)]
        status(L, lib.slorr_ffn_backward(d, *p, ws, have, None), code, text)

    for k in back:
        if back.index(k) < 6:
            backward(INVALID, f"{k} is NULL", **{k: None})
        backward(INVALID, f"{k} must be 16-byte aligned", **{k: arena(20) + 8})
    for out in back[6:]:
        for k in back:
            if k != out:
                backward(INVALID, "overlap", **{out: arena(back.index(k)) + 16})
    backward(INVALID, "overlap", ws=arena(5))
    backward(WORKSPACE, "NULL", ws=None)
    backward(WORKSPACE, "aligned", ws=arena(12) + 16)
    backward(WORKSPACE, "too small", have=b.value - 1)
    backward(0, "", dx=None, dw_gate=None, dw_up=None, dw_down=None)            # nothing is asked for


def test_ffn_strided_overlap(L, arena):
    """The gaps of a strided input belong to it."""
    lib, d = L.lib(), ffn(L, ldx=64)
    n = ctypes.c_size_t()
    status(L, lib.slorr_ffn_sizes(d, None, n, None), 0)
    st = lib.slorr_ffn_forward(d, arena(0), arena(1), arena(2), arena(3), arena(0) + 3 * 64 * 4, None, arena(5), n.value, None)
    status(L, st, INVALID, "overlap")


def test_ffn_no_tokens(L, arena):
    lib, d = L.lib(), ffn(L, tokens=0)
    n = ctypes.c_size_t()
    status(L, lib.slorr_ffn_sizes(d, None, n, None), 0)
    status(L, lib.slorr_ffn_forward(d, None, arena(1), arena(2), arena(3), None, None, arena(4), n.value, None), 0)


def join(L, rows=6, dim=16, dtype=0, norm=0, flags=3, gate_rows=0, ldx=0, ldf=0, ld_gate=0, eps=1e-5, alpha=1.0, p=0.0,
         site=0):
    return L.Join(rows, dim, dtype, norm, flags, gate_rows, ldx, ldf, ld_gate, eps, alpha, p, site)


NAMES = ["x", "f", "post_weight", "post_bias", "gate", "scale", "pre_weight", "pre_bias"]


class Calls:
    """Forward and backward of one join, with some tensors replaced."""

    def __init__(self, L, arena):
        self.L, self.arena = L, arena

    def run(self, code, text, d=None, rng="rng", y="y", z="z", dy="dy", dz="dz", grads=None, ws="ws", have=1 << 20,
            only=None, **new):
        L, arena, lib = self.L, self.arena, self.L.lib()
        d = d if d is not None else join(L, gate_rows=1)
        at = {k: arena(i) for i, k in enumerate([*NAMES, "rng", "y", "z", "dy", "dz", "ws"])}
        t = {k: new.get(k, at[k]) for k in NAMES}
        g = {k: (arena(20 + i) if t[k] else None) for i, k in enumerate(NAMES)}
        g.update(grads or {})
        ptr = lambda v: at[v] if isinstance(v, str) else v  # noqa: E731
        if only != "backward":
            st = lib.slorr_join_forward(d, L.JoinTensors(*t.values()), ptr(rng), ptr(y), ptr(z), None)
            status(L, st, code, text)
        if only != "forward":
            st = lib.slorr_join_backward(d, L.JoinTensors(*t.values()), ptr(rng), ptr(dy), ptr(dz),
                                         L.JoinTensors(*g.values()), ptr(ws), have, None)
            status(L, st, code, text)


@pytest.mark.parametrize("change,code,text", [
    (dict(dtype=5), UNSUPPORTED, "dtype"), (dict(norm=2), UNSUPPORTED, "norm"), (dict(flags=4), INVALID, "flags"),
    (dict(rows=-1), INVALID, "rows"), (dict(dim=0), INVALID, "dim"), (dict(dim=8193), UNSUPPORTED, "limits"),
    (dict(rows=(1 << 40) + 1), UNSUPPORTED, "limits"), (dict(rows=1 << 40, ldx=1 << 20), UNSUPPORTED, "limit"),
    (dict(ldx=8), INVALID, "stride"), (dict(ldf=8), INVALID, "stride"), (dict(ld_gate=8), INVALID, "stride"),
    (dict(ldx=1 << 22), UNSUPPORTED, "stride"), (dict(ldf=1 << 22), UNSUPPORTED, "stride"),
    (dict(ld_gate=1 << 22), UNSUPPORTED, "stride"), (dict(ldx=-16), INVALID, "stride"),
    (dict(eps=-1.0), INVALID, "eps"), (dict(eps=float("nan")), INVALID, "eps"), (dict(eps=float("inf")), INVALID, "eps"),
    (dict(alpha=float("inf")), INVALID, "alpha"), (dict(alpha=float("nan")), INVALID, "alpha"),
    (dict(p=-0.1), INVALID, "p must"), (dict(p=1.0), INVALID, "p must"), (dict(p=float("nan")), INVALID, "p must"),
    (dict(p=1 - 2.0 ** -18), INVALID, "p rounds"),
    (dict(gate_rows=4), INVALID, "divide"), (dict(gate_rows=-1), INVALID, "divide"),
])
def test_join_shapes(L, arena, change, code, text):
    d = join(L, **{"gate_rows": 1, **change})
    Calls(L, arena).run(code, text, d=d)
    n = ctypes.c_size_t()
    status(L, L.lib().slorr_join_workspace(d, n), code, text)


def test_join_gate_needs_rows(L, arena):
    Calls(L, arena).run(INVALID, "divide", d=join(L, gate_rows=0))
    Calls(L, arena).run(INVALID, "divide", d=join(L, gate_rows=7))


def test_join_buffers(L, arena):
    c, lib = Calls(L, arena), L.lib()
    n = ctypes.c_size_t()
    status(L, lib.slorr_join_workspace(None, n), INVALID, "NULL")
    status(L, lib.slorr_join_workspace(join(L), None), INVALID, "NULL")
    status(L, lib.slorr_join_workspace(join(L, gate_rows=1), n), 0)
    assert n.value > 0
    status(L, lib.slorr_join_forward(None, L.JoinTensors(), None, None, None, None), INVALID, "NULL")
    status(L, lib.slorr_join_forward(join(L), None, None, None, None, None), INVALID, "NULL")
    c.run(INVALID, "x is NULL", x=None)
    for k in NAMES:
        c.run(INVALID, f"{k} must be 16-byte aligned", **{k: arena(30) + 4})
        c.run(INVALID, "overlap", only="forward", **{k: arena(9)})
        c.run(INVALID, "overlap", only="backward", **{k: arena(13)})
        c.run(INVALID, "must be 16-byte aligned", only="backward", grads={k: arena(30) + 8})
        c.run(INVALID, "overlap", only="backward", grads={k: arena(NAMES.index("f" if k == "x" else "x"))})
        if k not in ("x", "f"):
            c.run(INVALID, "without the input", only="backward", d=join(L, gate_rows=1), **{k: None}, grads={k: arena(20)})
    for flags, k in ((2, "post_weight"), (2, "post_bias"), (1, "pre_weight"), (1, "pre_bias")):
        rest = {j: None for j in NAMES[2:] if j != k and (j.startswith("post") if flags == 2 else j.startswith("pre"))}
        c.run(INVALID, "without P", d=join(L, flags=flags, gate_rows=1), **rest)
    vectors = {k: None for k in NAMES[1:]}
    c.run(INVALID, "without f", d=join(L, flags=3), **vectors)
    c.run(INVALID, "without f", d=join(L, flags=2, gate_rows=1), **{**vectors, "gate": arena(4)})
    c.run(INVALID, "without f", d=join(L, flags=2), **{**vectors, "scale": arena(4)})
    c.run(INVALID, "nothing to do", d=join(L, flags=0), **vectors)
    c.run(INVALID, "y is NULL", only="forward", y=None)
    c.run(INVALID, "z is NULL", only="forward", z=None)
    c.run(INVALID, "y and z overlap", only="forward", z="y")
    c.run(INVALID, "y must be", only="forward", y=arena(9) + 8)
    c.run(INVALID, "z must be", only="forward", z=arena(9) + 8)
    no_pre = {"pre_weight": None, "pre_bias": None}
    c.run(INVALID, "z without PRE", only="forward", d=join(L, flags=1, gate_rows=1), **no_pre)
    c.run(INVALID, "dz without PRE", only="backward", d=join(L, flags=1, gate_rows=1), **no_pre)
    c.run(INVALID, "dy must be", only="backward", dy=arena(11) + 8)
    c.run(INVALID, "dz must be", only="backward", dz=arena(12) + 8)
    c.run(INVALID, "rng is NULL", d=join(L, gate_rows=1, p=0.5), rng=None)
    c.run(INVALID, "rng must be", d=join(L, gate_rows=1, p=0.5), rng=arena(8) + 4)
    c.run(INVALID, "overlap", only="backward", grads={"x": arena(8)})
    c.run(INVALID, "overlap", only="backward", grads={"x": arena(11)})
    c.run(INVALID, "overlap", only="backward", grads={"x": arena(21)})
    c.run(WORKSPACE, "NULL", only="backward", ws=None)
    c.run(WORKSPACE, "aligned", only="backward", ws=arena(13) + 16)
    c.run(WORKSPACE, "too small", only="backward", have=n.value - 1)
    d, t = join(L, gate_rows=1), L.JoinTensors(*(arena(i) for i in range(8)))
    status(L, lib.slorr_join_backward(d, t, None, None, None, None, arena(13), 1 << 20, None), INVALID, "grads is NULL")


def test_dropout(L, arena):
    lib, x, y, rng = L.lib(), arena(0), arena(1), arena(2)

    def run(code, text, n=100, dtype=0, p=0.5, rng=rng, x=x, y=y):
        status(L, lib.slorr_dropout(n, dtype, p, rng, 0, x, y, None), code, text)

    run(UNSUPPORTED, "dtype", dtype=9)
    run(INVALID, "n must", n=-1)
    run(UNSUPPORTED, "limit", n=(1 << 50) + 1)
    for p in (-1e-9, 1.0, 2.0, float("nan")):
        run(INVALID, "p must", p=p)
    run(INVALID, "p rounds", p=1 - 2.0 ** -18)
    run(INVALID, "rng is NULL", rng=None)
    run(INVALID, "rng must", rng=rng + 4)
    run(INVALID, "x is NULL", x=None)
    run(INVALID, "y is NULL", y=None)
    run(INVALID, "x must", x=x + 8)
    run(INVALID, "y must", y=y + 4)
    run(INVALID, "overlap", y=x + 16)
    run(INVALID, "overlap", rng=y + 392)
    run(0, "", n=0, x=None, y=None)


def test_python_entries_need_a_gpu():
    from paper_2607_08754_amd import FeedForwardBlock, block_join, block_norm, dropout, gated_ffn
    x, w, v = torch.zeros(2, 8), torch.zeros(16, 8), torch.zeros(8, 16)
    with pytest.raises(ValueError, match="x must be on a GPU"):
        gated_ffn(x, w, w, v)
    with pytest.raises(ValueError, match="x must be on a GPU"):
        block_norm(x)
    with pytest.raises(ValueError, match="x must be on a GPU"):
        block_join(x, x)
    with pytest.raises(ValueError, match="x must be on a GPU"):
        dropout(x, 0.5, torch.zeros(2, dtype=torch.int64))
    for bad in (x.half(), x.double(), x.long(), [[1.0]], None):
        with pytest.raises(ValueError, match="x must be a float32 or bfloat16 tensor"):
            gated_ffn(bad, w, w, v)
        with pytest.raises(ValueError, match="x must be a float32 or bfloat16 tensor"):
            block_join(bad, x)
        with pytest.raises(ValueError, match="x must be a float32 or bfloat16 tensor"):
            dropout(bad, 0.1, None)
    block = FeedForwardBlock(8, 16, dtype=torch.float32)
    assert [tuple(m.shape) for m in block.matrices()] == [(16, 8), (16, 8), (8, 16)]
    with pytest.raises(ValueError, match="on a GPU"):
        block(x)
    for kw in (dict(act="relu"), dict(kind="batch"), dict(p=1.0), dict(p=-0.5), dict(dtype=torch.float16)):
        with pytest.raises(ValueError):
            FeedForwardBlock(8, 16, **kw)
    for sizes in ((0, 8), (8, 0), (8193, 8)):
        with pytest.raises(ValueError):
            FeedForwardBlock(*sizes)
