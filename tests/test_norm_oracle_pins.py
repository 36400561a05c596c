"""Pins of oracle/norm_oracle.py: torch's autograd in float64, differences, closed forms, brute force."""
import math

import numpy as np
import pytest
import torch

from oracle import norm_oracle as orc

EPS = 1e-5


def _t(x):
    return None if x is None else torch.tensor(x, dtype=torch.float64, requires_grad=True)


def _torch_junction(o, x, w_post, gate, gate_rows, scale, w_pre, offset, normalize):
    norm = lambda v: v / torch.sqrt((v * v).mean(1, keepdim=True) + EPS)  # noqa: E731
    n = norm(o) * (offset + w_post) if normalize else o
    g = gate[torch.arange(x.shape[0]) // gate_rows] if gate is not None else 1.0
    y = x + scale * g * n
    return y, norm(y) * (offset + w_pre)


@pytest.mark.parametrize("normalize", [True, False])
@pytest.mark.parametrize("gate_rows", [0, 1, 3, 7])
def test_gradients_match_autograd(normalize, gate_rows):
    rng = np.random.default_rng(5 + gate_rows)
    S, d, scale, offset = 7, 24, 0.7, 1.0
    o, x, dh, dres = (rng.standard_normal((S, d)) for _ in range(4))
    wo, wp = (0.1 * rng.standard_normal(d) for _ in range(2))
    gate = rng.standard_normal((-(-S // gate_rows), d)) if gate_rows else None
    to, tx, two, twp, tg = _t(o), _t(x), _t(wo), _t(wp), _t(gate)
    y, h = _torch_junction(to, tx, two, tg, gate_rows, scale, twp, offset, normalize)
    y.retain_grad()
    ((h * torch.tensor(dh)).sum() + (y * torch.tensor(dres)).sum()).backward()
    oy, _ = orc.residual(o, x, normalize, wo, offset, EPS, gate, gate_rows, scale)
    assert np.allclose(oy, y.detach(), rtol=1e-13, atol=1e-13)
    assert np.allclose(orc.prenorm(oy, wp, offset, EPS), h.detach(), rtol=1e-13, atol=1e-13)
    dy, dwp, reach, dwp_reach = orc.norm_bwd(dh, oy, wp, offset, EPS)
    dy = dy + dres
    got = orc.residual_bwd(dy, o, normalize, wo, offset, EPS, gate, gate_rows, scale)
    for a, b in ((dy, y.grad), (dwp, twp.grad), (got["dO"], to.grad), (dy, tx.grad)):
        assert np.allclose(a, b, rtol=1e-11, atol=1e-12)
    if normalize:
        assert np.allclose(got["dw"], two.grad, rtol=1e-11, atol=1e-12)
    if gate is not None:
        assert np.allclose(got["dgate"], tg.grad, rtol=1e-11, atol=1e-12)
    assert (reach >= np.abs(dy - dres) * (1 - 1e-12)).all() and (dwp_reach >= np.abs(dwp) * (1 - 1e-12)).all()


def test_gradients_match_differences():
    rng = np.random.default_rng(11)
    S, d, offset, scale = 3, 16, 0.0, 0.5
    o, x, dy = (rng.standard_normal((S, d)) for _ in range(3))
    w, gate = rng.standard_normal(d), rng.standard_normal((2, d))
    value = lambda o, w, g: float((orc.residual(o, x, True, w, offset, EPS, g, 2, scale)[0] * dy).sum())  # noqa: E731
    got = orc.residual_bwd(dy, o, True, w, offset, EPS, gate, 2, scale)
    h = 1e-6
    for arr, grad, at in ((o, got["dO"], 0), (w, got["dw"], 1), (gate, got["dgate"], 2)):
        for i in list(np.ndindex(arr.shape))[::5]:
            args = [[o, w, gate], [o, w, gate]]
            for sign, a in zip((1, -1), args):
                a[at] = arr.copy()
                a[at][i] += sign * h
            slope = (value(*args[0]) - value(*args[1])) / (2 * h)
            assert math.isclose(slope, grad[i], rel_tol=1e-6, abs_tol=1e-7)


def test_norm_of_a_constant_row_and_its_gradient():
    """x = c: norm(x) = c / sqrt(c^2 + eps); a gradient along x is scaled by eps / (c^2 + eps)."""
    c, eps, d = 3.0, 0.5, 8
    x = np.full((1, d), c)
    assert np.allclose(orc.prenorm(x, None, 0.0, eps), c / math.sqrt(c * c + eps))
    dx, dw, _, _ = orc.norm_bwd(np.ones((1, d)), x, None, 0.0, eps)
    q = 1 / math.sqrt(c * c + eps)
    assert np.allclose(dx, q * (1 - c * c * q * q)) and np.allclose(dw, c * q)
    assert np.allclose(orc.prenorm(np.zeros((1, d)), None, 1.0, eps), 0.0)      # a row of zeros


def test_checkpoint_by_brute_force():
    """The scale is the smallest with every code below 127.5, and no other code is nearer."""
    rng = np.random.default_rng(3)
    x = rng.standard_normal((6, 72)) * 10.0 ** rng.integers(-30, 30, (6, 1))
    x = x.astype(np.float32).astype(np.float64)
    codes, exps = orc.checkpoint(x)
    back = orc.restore(codes, exps)
    for s in range(6):
        for b in range(3):
            block, got = x[s, 32 * b:32 * b + 32], back[s, 32 * b:32 * b + 32]
            step = 2.0 ** (int(exps[s, b]) - 127)
            top = np.abs(block).max()
            assert top < 127.5 * step and not top < 127.5 * step / 2
            every = np.arange(-127, 128) * step
            assert np.array_equal(np.abs(got - block), np.abs(every[None, :] - block[:, None]).min(1))
            assert np.abs(got - block).max() <= top / 127.5


def test_checkpoint_of_ties_borders_and_what_has_no_scale():
    x = np.zeros((9, 32))
    x[0, :4] = 127.0, 0.5, 1.5, -2.5                  # ties to even
    x[1, 0] = 127.5                                   # the next scale
    x[2, 0] = np.nextafter(np.float32(127.5), np.float32(0))
    x[3, :2] = np.inf, 1.0
    x[4, 1] = np.nan
    x[5, 0] = 2.0 ** -140                             # less than half a step of the least scale
    x[6, :2] = 2.0 ** -127, 1.5 * 2.0 ** -127
    x[7, 0] = float(np.finfo(np.float32).max)
    x[8, 0] = -127.0 * 2.0 ** 121
    codes, exps = orc.checkpoint(x)
    assert codes[0, :4].tolist() == [127, 0, 2, -2] and exps[0, 0] == 127
    assert codes[1, 0] == 64 and exps[1, 0] == 128
    assert codes[2, 0] == 127 and exps[2, 0] == 127
    assert exps[3:5, 0].tolist() == [255, 255] and exps[7, 0] == 255
    assert codes[5, 0] == 0 and exps[5, 0] == 0
    assert codes[6, :2].tolist() == [1, 2] and exps[6, 0] == 0
    assert codes[8, 0] == -127 and exps[8, 0] == 248
    back = orc.restore(codes, exps)
    assert np.isnan(back[[3, 4, 7]]).all() and np.isfinite(np.delete(back, [3, 4, 7], 0)).all()
