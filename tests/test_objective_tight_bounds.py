"""The bounds of objective_tight_bounds tell what they are for from what they are not: plausible mistakes, planted into the oracle's numbers,
are outside of them, and the oracle's own numbers rounded to float32 inside."""
import numpy as np
import pytest

from tests.objective_gpu_harness import Problem
from tests.objective_tight_bounds import check, divergence_bound

SOFT = dict(K=9, tail=True, temperature=4.0, sigma=1.0, short=0, empty=0, labels=False)
LABELS = dict(K=30, tail=True, label_coef=0.5, temperature=2.0, weights=True)


def as_given(r):
    """The oracle's numbers as a call would give them."""
    import torch
    f = np.float32
    dH = torch.from_numpy(r["dH"]).to(torch.bfloat16).double().numpy()
    return {"loss": float(f(r["loss"])), "n": r["n"], "nll": f(r["nll"]).astype(float), "kd": f(r["kd"]).astype(float), "lse": f(r["lse"]).astype(float),
            "dH": dH, "dW": f(r["dW"]).astype(float)}


def outputs(p):
    r = p.oracle()
    got = as_given(r)
    got["rows"] = got["kd"] if p.K else got["lse"]
    if p.labels is None:
        got["nll"] = None
    return r, got


PROBLEMS = [(40, 64, 900, SOFT), (300, 64, 1500, LABELS), (300, 64, 1500, dict(weights=True, z_coef=1e-3, softcap=1e5))]


@pytest.mark.parametrize("S,d,V,o", PROBLEMS)
def test_the_oracles_numbers_are_inside(S, d, V, o):
    p = Problem(S, d, V, **o)
    r, got = outputs(p)
    assert max(check(p, got, r).values()) < 0.6


def test_a_divergence_of_float32_differences_is_outside():
    """sum q (log q - log p) of float32 logarithms, which cancel where the student is nearly the teacher."""
    f = np.float32
    p = Problem(200, 64, 4000, **SOFT)
    p.lse = np.float32(np.log(np.exp(p.H @ p.W.T / 4.0).sum(1))).astype(np.float64)
    p.logits = np.float32(np.take_along_axis(p.H @ p.W.T, p.index.astype(np.int64), 1) * 1.001).astype(np.float64)      # nearly the student itself
    r = p.oracle()
    y = f(r["Z"]) / f(4.0)
    lse = np.log(np.exp(y).sum(1, dtype=f)).astype(f)
    kd = np.zeros(p.S)
    for s in range(p.S):
        log_q = f(f(p.logits[s]) / f(4.0)) - f(p.lse[s])
        q = np.exp(log_q)
        rest = f(1) - q.sum(dtype=f)
        others = np.ones(p.V, dtype=bool)
        others[p.index[s]] = False
        log_rest = f(np.log(np.exp(y[s, others]).sum(dtype=f)) - lse[s])
        kd[s] = (q * (log_q - (y[s, p.index[s]] - lse[s]))).sum(dtype=f) + rest * (np.log(rest) - log_rest)
    off = np.abs(kd - r["kd"]) / divergence_bound(p, r)
    print(off.max(), (off > 1).mean())
    assert (off > 1).any()


def test_a_loss_that_is_summed_in_float32_is_outside():
    p = Problem(300, 64, 1500, **LABELS)
    r, got = outputs(p)
    w = p.weights.astype(np.float64)
    total = np.float32(0)
    for x in np.float32(w * (0.5 * got["nll"] + 4.0 * got["rows"])):
        total = np.float32(total + x)
    got["loss"] = float(total) * r["gamma"]
    with pytest.raises(AssertionError, match="loss"):
        check(p, got, r)


def test_a_cap_that_is_half_a_step_of_itself_off_is_outside():
    """c - 2 c u in float32, with u next to 1/2 where the logit is small against the cap."""
    f = np.float32
    for cap in (1e3, 1e5):
        p = Problem(100, 64, 1500, softcap=cap, ignore=0.0)
        r, got = outputs(p)
        z = f(r["Z"])
        u = f(1) / (f(1) + np.exp2(np.abs(z) * f(2 / np.log(2) / cap)))
        y = np.copysign(f(cap) - f(2) * f(cap) * u, z).astype(np.float64)
        lse = np.log(np.exp(y - y.max(1, keepdims=True)).sum(1)) + y.max(1)
        got["nll"] = lse - y[np.arange(p.S), p.labels]
        with pytest.raises(AssertionError, match="nll"):
            check(p, got, r)
