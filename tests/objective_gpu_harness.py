"""Runs the LM head's other objectives through the binding on device copies of seeded inputs, and what the outputs may be off by."""
from __future__ import annotations

import numpy as np

from oracle import objective_oracle as orc

HALF_BF16 = 2.0 ** -8      # half a step of bfloat16, relative to the value
HALF_FP32 = 2.0 ** -24


def bf16(x):
    """x rounded to bfloat16, as float64."""
    import torch
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).to(torch.bfloat16).double().numpy()


class Problem:
    """Inputs of one call, as numpy arrays whose values the GPU holds exactly."""

    def __init__(self, S, d, V, K=0, seed=0, sigma=2.0, labels=True, ignore=0.1, weights=False, tail=False, short=0.2, empty=0.1, teacher="fp32",
                 M=1, **objective):
        rng = np.random.default_rng(1000 * seed + S + d + V + K)
        self.S, self.d, self.V, self.K, self.M, self.teacher = S, d, V, K, M, teacher
        self.H = bf16(rng.standard_normal((S, d)))
        self.W = bf16(rng.standard_normal((V, d)) * sigma / np.sqrt(d))
        self.labels = None
        if labels:
            self.labels = rng.integers(0, V, S).astype(np.int32)
            self.labels[rng.random(S) < ignore] = -100
        self.weights = None
        if weights:
            self.weights = np.float32(rng.uniform(-0.5, 2.0, S))
            self.weights[rng.random(S) < 0.2] = 0.0
        self.objective = dict(objective)
        self.index = self.logits = self.lse = None
        T = objective.get("temperature", 1.0)
        if K:
            t = 1.5 * self.H @ self.W.T + rng.standard_normal((S, V))
            # some of the largest, in no order, and some others
            keep = np.argsort(-t, axis=1)[:, :K]
            self.index = rng.permuted(keep, axis=1).astype(np.int32)
            logits = np.take_along_axis(t, self.index.astype(np.int64), 1)
            self.logits = bf16(logits) if teacher == "bf16" else np.float32(logits).astype(np.float64)
            self.lse = np.float32([orc._lse(row / T) for row in t]).astype(np.float64) if tail else None
            for s in range(S):
                if rng.random() < short:
                    self.index[s, rng.random(K) < 0.5] = -1
                if rng.random() < empty:
                    self.index[s] = -1
            if self.labels is not None:                          # half of the labels are entries of the teacher
                pick = (rng.random(S) < 0.5) & (self.index[:, 0] >= 0) & (self.labels != -100)
                self.labels[pick] = self.index[pick, 0]

    def oracle(self, grad_loss=1.0):
        o = dict(self.objective)
        if self.K:
            o.setdefault("label_coef", 0.0)
            o.update(teacher_index=self.index, teacher_logits=self.logits, teacher_lse=self.lse, teacher_coef=o.get("teacher_coef", 1.0))
        return orc.objective(self.H, self.W, self.labels, weights=self.weights, grad_loss=grad_loss, **o)


class Run:
    """Forward and backward on the GPU.  Every output is poisoned before, and has a border that has to stay as it was."""

    def __init__(self, p: Problem):
        import torch
        import paper_2407_15892_amd as mst
        self.p, self.mst, self.torch = p, mst, torch
        dev = lambda x, t: None if x is None else torch.from_numpy(np.ascontiguousarray(x)).to("cuda").to(t)  # noqa: E731
        self.H, self.W = dev(p.H, torch.bfloat16), dev(p.W, torch.bfloat16)
        self.labels, self.weights = dev(p.labels, torch.int32), dev(p.weights, torch.float32)
        self.index, self.lse_in = dev(p.index, torch.int32), dev(p.lse, torch.float32)
        self.logits = dev(p.logits, torch.bfloat16 if p.teacher == "bf16" else torch.float32)
        self.bytes = mst.mst_objective_bytes(p.S, p.d, p.V, p.M, p.K)
        self.borders = []
        self.ws = self.room(max(self.bytes[:2]))
        self.saved = self.room(self.bytes[2])
        f32 = torch.float32
        self.loss, self.n = self.out((1,), f32), self.out((1,), torch.int64)
        self.nll = self.out((p.S,), f32) if self.labels is not None else None
        self.rows = self.out((p.S,), f32)                        # kd or lse
        self.dH, self.dW = self.out((p.S, p.d), torch.bfloat16), self.out((p.V, p.d), f32)

    def room(self, n):
        t = self.torch.full((n + 512,), 0xA5, dtype=self.torch.uint8, device="cuda")
        self.borders.append(t[n:])
        return t[:n]

    def out(self, shape, dtype):
        n = int(np.prod(shape)) * self.torch.empty((), dtype=dtype).element_size()
        raw = self.torch.full(((n + 255) // 256 * 256 + 256,), 0xA5, dtype=self.torch.uint8, device="cuda")
        raw[:n] = 0xFF                                           # NaN, -1
        self.borders.append(raw[n:])
        return raw[:n].view(dtype).view(shape)

    def forward(self, saved=True, stream=None):
        p, o = self.p, self.p.objective
        common = dict(saved=self.saved if saved else None, weights=self.weights, nll=self.nll, n_valid=self.n, stream=stream, **o)
        if p.K:
            self.mst.mst_lmhead_distill_fwd(self.H, self.W, self.index, self.logits, p.M, self.ws, self.loss, teacher_lse=self.lse_in,
                                            labels=self.labels, kd=self.rows, **common)
        else:
            self.mst.mst_lmhead_wce_fwd(self.H, self.W, self.labels, -100, p.M, self.ws, self.loss, lse=self.rows, **common)

    def backward(self, grad_loss=1.0, M=None, stream=None):
        M = self.p.M if M is None else M
        if self.p.K:
            self.mst.mst_lmhead_distill_bwd(self.H, self.W, self.p.K, M, grad_loss, self.saved, self.ws, self.dH, self.dW, stream=stream)
        else:
            self.mst.mst_lmhead_wce_bwd(self.H, self.W, M, grad_loss, self.saved, self.ws, self.dH, self.dW, stream=stream)

    def outputs(self):
        self.torch.cuda.synchronize()
        assert all(bool((b == 0xA5).all()) for b in self.borders), "written past the end of an output"
        f = lambda t: None if t is None else t.detach().double().cpu().numpy()  # noqa: E731
        return {"loss": float(self.loss), "n": int(self.n), "nll": f(self.nll), "rows": f(self.rows), "dH": f(self.dH), "dW": f(self.dW)}


def bounds(p: Problem, r: dict, grad_loss=1.0):
    """Largest errors of the outputs.

    A logit is a float32 sum of d exact products: d roundings of at most half a step of the partial sums, none of which is larger
    than a few of the largest logit; as independent errors they come to sqrt(d / 3) of that, of which 4 sqrt(d) are more than six
    standard deviations: dz.  What a row's loss is made of are differences of numbers no larger than `top`, each a few roundings (16 half
    steps are more than they take), and log-sum-exps, which are off by no more than their logits; the cap's tanh is off by a few
    half steps of the cap.  A share is relatively off by what its logarithm is: arg.
    """
    o = p.objective
    T = o.get("temperature", 1.0)
    cap = o.get("softcap", 0.0)
    largest = np.abs(r["Z"]).max()
    dz = 4 * np.sqrt(p.d) * HALF_FP32 * max(largest, 1.0)
    top = min(cap, largest) if cap else largest
    top = max(top + np.log(p.V), 1.0, *(np.abs(x[np.isfinite(x)]).max(initial=0.0) for x in (p.logits, p.lse) if x is not None))
    row = 2 * dz + 16 * HALF_FP32 * (top + cap)
    arg = (row + 16 * HALF_FP32 * top) / min(T, 1.0) + 16 * HALF_FP32
    b = {"nll": row, "lse": row}
    # kd: shares times logarithms, both off by arg; the rest is off by what the shares are together
    b["kd"] = 2 * arg * (1 + r["kd_abs"]) + (arg + 2 * HALF_FP32) * r["rest_abs"]
    w = 1.0 if p.weights is None else np.abs(p.weights).max()
    lse_top = np.abs(r["lse"]).max() if np.isfinite(r["lse"]).all() else 0.0
    b["row_loss"] = w * (abs(o.get("label_coef", 1.0)) * b["nll"] + abs(o.get("teacher_coef", 1.0)) * T * T * (b["kd"] if p.K else 0.0) +
                         2 * abs(o.get("z_coef", 0.0)) * lse_top * b["lse"]) + 8 * HALF_FP32 * np.abs(r["row_loss"]).max()
    b["loss"] = np.sum(b["row_loss"] * np.ones(p.S)) * abs(r["gamma"] / grad_loss) + 4 * HALF_FP32 * abs(r["loss"])
    # the logits' gradient: its terms off by their shares' error (the rest's share of the others by the rest's own as well), then rounded
    share = 4 * arg + 8 * HALF_FP32
    # the cap's slope 1 / cosh^2(z / cap), whose logarithm changes by at most 2 / cap for each unit of z: the logit's error, and the
    # roundings of its exponential's argument 2 z / cap and of 2 z / cap in base 2
    if cap:
        share += 2 / cap * dz + 8 * HALF_FP32 * (2 * largest / cap + 1)
    if p.K and p.lse is not None:
        share += 8 * arg
    dG = HALF_BF16 * np.abs(r["G"]) + share * r["G_abs"]
    if p.K and p.lse is not None:     # rest = 1 - Q: absolute error of what Q is off by, over the others' shares
        dG = dG + 8 * arg * r["others_share"] * r["others_scale"]
    g = abs(r["gamma"])
    acc_h = p.V * HALF_FP32 * (np.abs(r["G"]) @ np.abs(p.W))
    acc_w = p.S * HALF_FP32 * (np.abs(r["G"]).T @ np.abs(p.H))
    b["dH"] = (g * (dG @ np.abs(p.W) + acc_h) * (1 + HALF_BF16) + HALF_BF16 * np.abs(r["dH"])) * (1 + 4 * HALF_FP32) + 1e-38
    b["dW"] = g * (dG.T @ np.abs(p.H) + acc_w) + 8 * HALF_FP32 * np.abs(r["dW"]) + 1e-38
    return b


def check(p: Problem, got: dict, r: dict, grad_loss=1.0, backward=True):
    T = p.objective.get("temperature", 1.0)
    if p.K and p.lse is not None:
        # where the rest goes: shares among the others, and what multiplies them
        y = r["Z"] if not p.objective.get("softcap") else p.objective["softcap"] * np.tanh(r["Z"] / p.objective["softcap"])
        share, scale = np.zeros_like(y), np.zeros((p.S, 1))
        for s in range(p.S):
            v, _ = orc.teacher_of_row(p.index[s], p.logits[s], p.V)
            others = np.ones(p.V, dtype=bool)
            others[v] = False
            if len(v) and others.any():
                share[s, others] = np.exp(y[s, others] / T - orc._lse(y[s, others] / T))
                scale[s] = abs(p.objective.get("teacher_coef", 1.0)) * T * (1.0 if p.weights is None else abs(p.weights[s]))
        r = dict(r, others_share=share, others_scale=scale)
    b = bounds(p, r, grad_loss)
    assert got["n"] == r["n"]
    worst = {}

    def near(name, x, ref, tol):
        off = np.abs(np.asarray(x) - ref)
        assert np.isfinite(x).all(), name
        worst[name] = float((off / np.maximum(tol, 1e-300)).max())
        assert (off <= tol).all(), (name, float(off.max()), worst[name])

    near("loss", got["loss"], r["loss"], b["loss"])
    if got["nll"] is not None:
        near("nll", got["nll"], r["nll"], b["nll"])
    near("kd" if p.K else "lse", got["rows"], r["kd"] if p.K else r["lse"], b["kd"] if p.K else b["lse"])
    if backward:
        near("dH", got["dH"], r["dH"], b["dH"])
        near("dW", got["dW"], r["dW"], b["dW"])
    return worst
