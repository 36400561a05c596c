"""Definition of the LM head's weighted cross-entropy of capped logits and of distillation from a teacher's largest logits, row by
row in numpy fp64, with the gradients of the logits written out.  Independent of the library: used by tests only."""
from __future__ import annotations

import numpy as np


def _lse(x):
    m = x.max()
    if not np.isfinite(m):
        return m
    return m + np.log(np.exp(x - m).sum())


def teacher_of_row(index, logits, V):
    """(vocabulary indices, logits) of a row's entries: those at or above 0, the first of each."""
    seen, at = set(), []
    for k, v in enumerate(index):
        if v >= V:
            raise ValueError("teacher index out of range")
        if v >= 0 and int(v) not in seen:
            seen.add(int(v))
            at.append(k)
    return np.asarray(index)[at].astype(np.int64), np.asarray(logits, dtype=np.float64)[at]


def objective(H, W, labels=None, ignore_index=-100, weights=None, softcap=0.0, z_coef=0.0, label_coef=1.0, teacher_index=None,
              teacher_logits=None, teacher_lse=None, teacher_coef=0.0, temperature=1.0, divisor=0, grad_loss=1.0):
    """loss, n, per-row nll, lse, kd; G: gradient of the logits without grad_loss / n, G_abs: the sum of its terms' magnitudes; kd_abs: that
    of kd's terms, rest_abs: of kd's slope by the rest; dH, dW.
    teacher_index None: the weighted cross-entropy (label_coef 1)."""
    S, V, T = H.shape[0], W.shape[0], float(temperature)
    Z = H.astype(np.float64) @ W.astype(np.float64).T
    nll, lses, kds, row_loss, kd_abs, rest_abs = (np.zeros(S) for _ in range(6))
    G, G_abs = np.zeros((S, V)), np.zeros((S, V))
    n = 0
    for s in range(S):
        z = Z[s]
        t = np.tanh(z / softcap) if softcap else None
        y = softcap * t if softcap else z
        w = 1.0 if weights is None else float(weights[s])
        g, g_abs, loss, counts = np.zeros(V), np.zeros(V), 0.0, False
        lses[s] = _lse(y)
        if labels is not None and labels[s] != ignore_index:
            if not 0 <= labels[s] < V:
                raise ValueError("label out of range")
            counts = True
            nll[s] = lses[s] - y[labels[s]]
            loss += label_coef * nll[s] + z_coef * lses[s] ** 2
            p = np.exp(y - lses[s])
            g += (label_coef + 2 * z_coef * lses[s]) * p
            g_abs += (abs(label_coef) + abs(2 * z_coef * lses[s])) * p
            g[labels[s]] -= label_coef
            g_abs[labels[s]] += abs(label_coef)
        if teacher_index is not None:
            v, tl = teacher_of_row(teacher_index[s], teacher_logits[s], V)
            if len(v) and (teacher_lse is not None or tl.max() > -np.inf):
                counts = True
                log_q = tl / T - (teacher_lse[s] if teacher_lse is not None else _lse(tl / T))
                q = np.exp(log_q)
                others = np.ones(V, dtype=bool)
                others[v] = False
                rest = max(0.0, 1 - q.sum()) if teacher_lse is not None and others.any() else 0.0
                log_p = y / T - _lse(y / T)
                some = q > 0
                kd = (q[some] * (log_q[some] - log_p[v][some])).sum()
                kd_abs[s] = (q[some] * np.abs(log_q[some] - log_p[v][some])).sum()
                c = T * teacher_coef
                p = np.exp(log_p)
                part, part_abs = p * (q.sum() + rest), p * (q.sum() + rest)
                if rest > 0:
                    log_rest = _lse(log_p[others])
                    kd += rest * (np.log(rest) - log_rest)
                    kd_abs[s] += rest * abs(np.log(rest) - log_rest)
                    rest_abs[s] = 1 + abs(np.log(rest) - log_rest)
                    part[others] -= rest * np.exp(log_p[others] - log_rest)
                    part_abs[others] += rest * np.exp(log_p[others] - log_rest)
                part[v] -= q
                part_abs[v] += q
                kds[s] = kd
                loss += teacher_coef * T * T * kd
                g += c * part
                g_abs += abs(c) * part_abs
        n += counts
        # 1 - tanh^2 as 1 / cosh^2: the difference is 0 from |z| = 19 softcap on
        slope = 1 / np.cosh(np.minimum(np.abs(z / softcap), 350.0)) ** 2 if softcap else 1.0
        row_loss[s] = w * loss if w else 0.0
        G[s], G_abs[s] = w * g * slope, abs(w) * g_abs * slope
    by = 0.0 if n == 0 else 1.0 / (divisor or n)
    gamma = grad_loss * by
    return {"loss": row_loss.sum() * by, "row_loss": row_loss, "n": n, "nll": nll, "lse": lses, "kd": kds, "kd_abs": kd_abs, "rest_abs": rest_abs, "Z": Z, "G": G, "G_abs": G_abs,
            "gamma": gamma, "dH": gamma * G @ W.astype(np.float64), "dW": gamma * G.T @ H.astype(np.float64)}
