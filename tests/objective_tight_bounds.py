"""What the outputs of the LM head's other objectives may be off by, without room for cancellation: a cap's rounding in half steps of the
capped logit and not of the cap, a divergence's error in what the two distributions differ by, the loss as a sum of the call's own losses."""
from __future__ import annotations

import copy

import numpy as np

from oracle import objective_oracle as orc
from tests import objective_gpu_harness as harness

H = harness.HALF_FP32


def capped(z, cap):
    return cap * np.tanh(z / cap) if cap else z


def as_bent(p, r):
    """p with a cap that is no larger than the logits: harness.bounds takes 16 half steps of it for a capped logit and 16 of `top`, and
    c tanh(z / c) is formed with relative errors of up to 8 half steps (near 0: one of z / c's square, small against 1, and one of the last
    step; elsewhere of 1 - 2 u, u = 1 / (1 + exp(2 |z| / c)) <= 0.27, with three half steps in the exponent's argument, two in exp2, one in the
    sum, two in the reciprocal and one at the end)."""
    q = copy.copy(p)
    cap = p.objective.get("softcap", 0.0)
    if cap:
        q.objective = dict(p.objective, softcap=min(cap, max(np.abs(r["Z"]).max(), 1e-30)))
    return q


def divergence_bound(p, r):
    """Of each row's divergence.  With w = log p - log q it is formed as the sum over entries and rest of q (exp(w) - 1 - w), and Q + rest - 1.
    - A capped logit off by e_v, and log-sum-exps off by less than `arg` in the shares' logarithms: the derivative by log p_v is p_v - q_v where
      Q + rest = 1, in general (Q + rest) p_v - q_v; and at most arg^2 beyond that.
    - A part is q times a series where |w| < 1/4, seven roundings of terms of one sign or falling by 12, 16 half steps; w itself is rounded, half a
      step of w times |p - q|.  Elsewhere p and q come from exponentials that are 4 half steps off, and q w.
    - The entries' own log-sum-exp (no rest) shifts all log q: 40 half steps of it are a sum of up to 256 exponentials; the derivative is the divergence.
    - The rest is 1 - Q, off by 4 half steps of Q, with the derivative w_rest + 1; its rounding and the last steps are 4 half steps of 1."""
    o = p.objective
    T, cap = o.get("temperature", 1.0), o.get("softcap", 0.0)
    largest = np.abs(r["Z"]).max()
    bent = min(cap, largest) if cap else largest
    top = max(bent + np.log(p.V), 1.0, *(np.abs(x[np.isfinite(x)]).max(initial=0.0) for x in (p.logits, p.lse) if x is not None))
    dz = 4 * np.sqrt(p.d) * H * max(largest, 1.0)
    arg = (2 * dz + 16 * H * (top + bent) + 16 * H * top) / T + 16 * H
    y = capped(r["Z"], cap) / T
    b = np.zeros(p.S)
    for s in range(p.S):
        v, t = orc.teacher_of_row(p.index[s], p.logits[s], p.V)
        if not len(v) or (p.lse is None and not t.max() > -np.inf):
            continue
        log_p = y[s] - orc._lse(y[s])
        log_q = t / T - (p.lse[s] if p.lse is not None else orc._lse(t / T))
        others = np.ones(p.V, dtype=bool)
        others[v] = False
        q, P = np.exp(log_q), np.exp(log_p[v])
        Q = q.sum()
        rest = max(0.0, 1 - Q) if p.lse is not None and others.any() else 0.0
        p_rest = np.exp(log_p[others]).sum()
        differ = np.abs((Q + rest) * P - q).sum() + abs((Q + rest) * p_rest - rest)
        with np.errstate(invalid="ignore", divide="ignore"):
            w = np.where(q > 0, log_p[v] - log_q, 0.0)
            w_rest = np.log(p_rest) - np.log(rest) if rest > 0 else 0.0
        q_all, p_all, w_all = np.append(q, rest), np.append(P, p_rest), np.append(w, w_rest)
        part = np.where(q_all > 0, q_all * (np.expm1(w_all) - w_all), p_all)
        steps = np.where(np.abs(w_all) < 0.25, 16 * np.abs(part) + np.abs(p_all - q_all) * np.abs(w_all), 4 * (p_all + q_all) + 5 * q_all * np.abs(w_all))
        b[s] = arg * differ + arg * arg + H * steps.sum() + 40 * H * abs(r["kd"][s])
        if p.lse is not None:
            b[s] += 4 * H * Q * (abs(w_rest) + 1) + 4 * H
    return b


def loss_of_rows(p, got, r):
    """The loss as the float64 sum of what the call gave for each row, and its bound: a row's loss has at most six roundings, which are independent
    of each other (12 half steps of the root of the squares' sum are more than six standard deviations, and more than six of one row), and the
    quotient one."""
    f = np.float32
    o = p.objective
    w = np.ones(p.S) if p.weights is None else p.weights.astype(np.float64)
    w = np.where(w == 0, 0.0, w)
    labelled = p.labels != -100 if p.labels is not None else np.zeros(p.S, dtype=bool)
    alpha = float(f(o.get("label_coef", 0.0 if p.K else 1.0)))
    terms = [alpha * np.where(labelled, got["nll"], 0.0)] if p.labels is not None else []
    if p.K:
        terms.append(float(f(o.get("teacher_coef", 1.0))) * float(f(o.get("temperature", 1.0))) ** 2 * got["rows"])
    else:
        terms.append(float(f(o.get("z_coef", 0.0))) * np.where(labelled, got["rows"], 0.0) ** 2)
    by = r["gamma"]
    size = sum(np.abs(w * t) for t in terms)
    loss = sum((w * t).sum() for t in terms) * by
    return loss, H * abs(loss) + 12 * H * np.sqrt((size ** 2).sum()) * by + 1e-38


def with_others(p, r):
    """r with each row's shares among the vocabulary entries that are not the teacher's, and what multiplies them (harness.bounds)."""
    T = p.objective.get("temperature", 1.0)
    y = capped(r["Z"], p.objective.get("softcap", 0.0)) / T
    share, scale = np.zeros_like(y), np.zeros((p.S, 1))
    for s in range(p.S):
        v, _ = orc.teacher_of_row(p.index[s], p.logits[s], p.V)
        others = np.ones(p.V, dtype=bool)
        others[v] = False
        if len(v) and others.any():
            share[s, others] = np.exp(y[s, others] - orc._lse(y[s, others]))
            scale[s] = abs(p.objective.get("teacher_coef", 1.0)) * T * (1.0 if p.weights is None else abs(p.weights[s]))
    return dict(r, others_share=share, others_scale=scale)


def check(p, got, r, backward=True):
    """Every output of a call and its gradients (grad_loss 1) under the bounds here; the largest errors as parts of their bounds."""
    if p.K and p.lse is not None:
        r = with_others(p, r)
    b = harness.bounds(as_bent(p, r), r)
    rows = "kd" if p.K else "lse"
    if p.K:
        b["kd"] = divergence_bound(p, r)
    refs = {"nll": (got["nll"], r["nll"]), rows: (got["rows"], r[rows]), "dH": (got["dH"], r["dH"]), "dW": (got["dW"], r["dW"])}
    loss, b["loss"] = loss_of_rows(p, got, r)
    refs["loss"] = (got["loss"], loss)
    assert got["n"] == r["n"]
    worst = {}
    for name, (x, ref) in refs.items():
        if x is None or (not backward and name in ("dH", "dW")):
            continue
        assert np.isfinite(x).all(), name
        off = np.abs(x - ref)
        worst[name] = float((off / np.maximum(b[name], 1e-300)).max())
        assert (off <= b[name]).all(), (name, float(off.max()), worst[name])
    return worst
