"""CPU reference of what stands between the mini-sequence blocks, in numpy float64: the norm before a block, the gated and
scaled residual after it, their gradients, and the 8-bit checkpoint of a tensor.

Written from the definitions; shares no code with the HIP path.  Every function that returns computed values can also return their
*reach*: the same expression with every term replaced by its magnitude, which is what rounding errors of the terms are
relative to.
"""
from __future__ import annotations

import numpy as np


# ------------------------------------------------------------------ 8-bit checkpoint
def checkpoint(x):
    """(codes int8 [S, d], exps uint8 [S, ceil(d/32)]) of float64 values: per block of 32 columns the smallest power of two
    2^(E - 127), E >= 0, more than the largest magnitude / 127.5; codes the entries over it, to nearest, ties to even.  E = 255 where the
    block has a NaN, an infinity or a magnitude from 127.5 * 2^121 on."""
    x = np.asarray(x, np.float64)
    S, d = x.shape
    blocks = np.zeros((S, -(-d // 32), 32))
    blocks.reshape(S, -1)[:, :d] = x
    top = np.abs(blocks).max(2)
    with np.errstate(invalid="ignore"):
        none = ~(top < 127.5 * 2.0 ** 121)
    top = np.where(none, 0.0, top)
    k = np.maximum(-127.0, np.floor(np.log2(np.maximum(top, 2.0 ** -200))) - 8)
    for _ in range(3):                                   # floor(log2) - 8 is 2 or 3 too small
        k += ~(top < 127.5 * 2.0 ** k)
    assert (top < 127.5 * 2.0 ** k).all()
    codes = np.rint(np.where(none[:, :, None], 0.0, blocks) / 2.0 ** k[:, :, None])
    return codes.reshape(S, -1)[:, :d].astype(np.int8), np.where(none, 255, k + 127).astype(np.uint8)


def restore(codes, exps):
    """float64 values that a checkpoint stands for."""
    d = codes.shape[1]
    e = np.repeat(exps.astype(np.float64), 32, axis=1)[:, :d]
    with np.errstate(over="ignore"):
        return np.where(e == 255, np.nan, codes.astype(np.float64) * 2.0 ** (e - 127))


# ------------------------------------------------------------------------- operators
def rstd(x, eps):
    return 1.0 / np.sqrt((x * x).mean(1, keepdims=True) + eps)


def weight(w, offset, d):
    return offset + (np.ones(d) if w is None else w)


def prenorm(x, w, offset, eps):
    """H."""
    return x * rstd(x, eps) * weight(w, offset, x.shape[1])


def norm_bwd(dn, x, w, offset, eps, dn_reach=None):
    """Gradients of x and of the weight of norm(x) * weight, dn being that of the result, and the reach of both."""
    q = rstd(x, eps)
    wt = weight(w, offset, x.shape[1])
    n = x * q
    a = dn * wt
    dx = q * (a - n * (a * n).mean(1, keepdims=True))
    m = np.abs(dn) if dn_reach is None else dn_reach
    am = m * np.abs(wt)
    dx_reach = q * (am + np.abs(n) * (am * np.abs(n)).mean(1, keepdims=True))
    return dx, (dn * n).sum(0), dx_reach, (m * np.abs(n)).sum(0)


def gate_of_rows(gate, gate_rows, S, d):
    return np.ones((S, d)) if gate is None else gate[np.arange(S) // gate_rows]


def branch(o, normalize, w, offset, eps):
    return prenorm(o, w, offset, eps) if normalize else o


def residual(o, x, normalize, w, offset, eps, gate, gate_rows, scale):
    """(Y, reach)."""
    n = scale * gate_of_rows(gate, gate_rows, *x.shape) * branch(o, normalize, w, offset, eps)
    return x + n, np.abs(x) + np.abs(n)


def residual_bwd(dy, o, normalize, w, offset, eps, gate, gate_rows, scale, dy_reach=None):
    """dict of dO, dw, dgate and, under name + "_reach", their reach; o may be None without norm and gate."""
    S, d = dy.shape
    m = np.abs(dy) if dy_reach is None else dy_reach
    g = gate_of_rows(gate, gate_rows, S, d) * scale
    out = {"dw": None, "dgate": None}
    if gate is not None:
        n = branch(o, normalize, w, offset, eps)
        out["dgate"], out["dgate_reach"] = np.zeros(gate.shape), np.zeros(gate.shape)
        np.add.at(out["dgate"], np.arange(S) // gate_rows, scale * dy * n)
        np.add.at(out["dgate_reach"], np.arange(S) // gate_rows, np.abs(scale) * m * np.abs(n))
    if not normalize:
        out["dO"], out["dO_reach"] = g * dy, np.abs(g) * m
        return out
    out["dO"], out["dw"], out["dO_reach"], out["dw_reach"] = norm_bwd(g * dy, o, w, offset, eps, np.abs(g) * m)
    return out
