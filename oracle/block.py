"""Oracle of the operators of a regularised feed-forward block, plain NumPy float64.

Written from the definitions in include/slorr.h; gradients are the formulas of
the backward pass, which the tests check against differences of the forward.

  ffn_forward / ffn_backward     y = (act(x Wg^T) * (x Wu^T)) Wd^T
  join_forward / join_backward   y = x + alpha scale gate drop(N(f) w1 + b1), z = N(y) w2 + b2
  keep_mask                      the dropout decision of every element
"""
from __future__ import annotations

import math
from types import SimpleNamespace

import numpy as np

try:
    from scipy.special import erf as _erf
except ImportError:                                     # pragma: no cover
    _erf = np.vectorize(math.erf, otypes=[np.float64])


# ---------------------------------------------------------------- generator

def philox(counter, key):
    """Philox4x32-10 (Salmon et al. 2011): four uint32 arrays of counter words and
    two of key words to four uint32 arrays."""
    c = [np.asarray(w, dtype=np.uint64) for w in counter]
    k = [int(w) for w in key]
    mask = np.uint64(0xFFFFFFFF)
    for _ in range(10):
        p0 = c[0] * np.uint64(0xD2511F53)
        p1 = c[2] * np.uint64(0xCD9E8D57)
        c = [(p1 >> np.uint64(32)) ^ c[1] ^ np.uint64(k[0]), p1 & mask,
             (p0 >> np.uint64(32)) ^ c[3] ^ np.uint64(k[1]), p0 & mask]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return [w.astype(np.uint32) for w in c]


def threshold(p):
    return int(round(p * 65536))


def keep_mask(n, p, key, offset, site=0, first=0):
    """Truth values of the n elements from `first` (a multiple of 8) on: the 16-bit number e mod 8 of block e div 8 is
    at least threshold(p)."""
    key, off = key % 2 ** 64, (offset + site) % 2 ** 64
    i = np.arange(first // 8, first // 8 + (n + 7) // 8, dtype=np.uint64)
    lo = np.uint64(0xFFFFFFFF)
    words = philox([i & lo, i >> np.uint64(32), np.full_like(i, off & 0xFFFFFFFF), np.full_like(i, off >> 32)],
                   [key & 0xFFFFFFFF, key >> 32])
    halves = np.stack([h for w in words for h in (w & 0xFFFF, w >> 16)], axis=1)
    return halves.reshape(-1)[:n] >= threshold(p)


def keep_factor(p):
    return 65536.0 / (65536.0 - threshold(p))


# ------------------------------------------------------------- feed-forward

def act_and_slope(a, kind):
    if kind == "silu":
        g = 1.0 / (1.0 + np.exp(-a))
        return a * g, g + a * g * (1.0 - g)
    if kind == "gelu":
        c = 0.5 * (1.0 + _erf(a / math.sqrt(2.0)))
        return a * c, c + a * np.exp(-0.5 * a * a) / math.sqrt(2.0 * math.pi)
    k = math.sqrt(2.0 / math.pi)
    t = np.tanh(k * (a + 0.044715 * a ** 3))
    return 0.5 * a * (1.0 + t), 0.5 * (1.0 + t) + 0.5 * a * (1.0 - t * t) * k * (1.0 + 3 * 0.044715 * a * a)


def ffn_forward(x, wg, wu, wd, act):
    a, b = x @ wg.T, x @ wu.T
    f, s = act_and_slope(a, act)
    h = f * b
    return SimpleNamespace(a=a, b=b, f=f, s=s, h=h, y=h @ wd.T)


def ffn_backward(dy, x, wg, wu, wd, act):
    r = ffn_forward(x, wg, wu, wd, act)
    dh = dy @ wd
    da, db = dh * r.b * r.s, dh * r.f
    return SimpleNamespace(fwd=r, dh=dh, da=da, db=db, x=da @ wg + db @ wu, w_gate=da.T @ x, w_up=db.T @ x,
                           w_down=dy.T @ r.h)


# --------------------------------------------------------------------- join

def _norm(t, kind, eps):
    c = t - t.mean(axis=1, keepdims=True) if kind == "layer" else t
    r = 1.0 / np.sqrt((c * c).mean(axis=1, keepdims=True) + eps)
    return c * r, r


def _norm_back(g, n, r, kind):
    out = g - n * (g * n).mean(axis=1, keepdims=True)
    if kind == "layer":
        out = out - g.mean(axis=1, keepdims=True)
    return r * out


def join_forward(x, f, kind, eps, post, pre, alpha=1.0, w1=None, b1=None, gate=None, scale=None, w2=None, b2=None,
                 drop=None):
    """x, f: (rows, dim); gate: (gate_rows, dim); drop: the dropout factors (rows, dim) or None."""
    one = lambda t, v: v if t is None else t
    r = SimpleNamespace(fn=f, rf=None, g=1.0, m=alpha)
    y = x
    if f is not None:
        if post:
            r.fn, r.rf = _norm(f, kind, eps)
        r.u = r.fn * one(w1, 1.0) + one(b1, 0.0)
        if gate is not None:
            r.g = np.repeat(gate, x.shape[0] // gate.shape[0], axis=0) if x.shape[0] else gate[:0]
        r.m = alpha * (1.0 if drop is None else drop)
        y = x + r.m * one(scale, 1.0) * r.g * r.u
    r.y, r.z = y, None
    if pre:
        r.yn, r.ry = _norm(y, kind, eps)
        r.z = r.yn * one(w2, 1.0) + one(b2, 0.0)
    return r


def join_backward(dy, dz, x, f, kind, eps, post, pre, alpha=1.0, w1=None, b1=None, gate=None, scale=None, w2=None,
                  b2=None, drop=None):
    one = lambda t, v: v if t is None else t
    r = join_forward(x, f, kind, eps, post, pre, alpha, w1, b1, gate, scale, w2, b2, drop)
    g = {}
    d = np.zeros_like(x) if dy is None else dy
    if pre:
        e = np.zeros_like(x) if dz is None else dz
        g["pre_weight"], g["pre_bias"] = (e * r.yn).sum(0), e.sum(0)
        d = d + _norm_back(e * one(w2, 1.0), r.yn, r.ry, kind)
    g["x"] = d
    if f is None:
        return g
    t = d * r.m * r.u
    g["scale"] = (t * r.g).sum(0)
    if gate is not None:
        g["gate"] = (t * one(scale, 1.0)).reshape(gate.shape[0], x.shape[0] // gate.shape[0], x.shape[1]).sum(1)
    du = d * r.m * one(scale, 1.0) * r.g
    g["f"] = du
    if post:
        g["post_weight"], g["post_bias"] = (du * r.fn).sum(0), du.sum(0)
        g["f"] = _norm_back(du * one(w1, 1.0), r.fn, r.rf, kind)
    return g
