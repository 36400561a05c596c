"""Helpers of the GPU tests of norms, residuals and checkpoints: seeded inputs, guarded outputs, calls, and the tolerances."""
from __future__ import annotations

import numpy as np

from mst_inputs import bf16_bits_to_f64, f32_to_bf16_bits

EPS = 1e-5
GUARD = 256        # entries behind every output that a call must leave alone


def rounded(x, stream="bf16"):
    """float64 copy of x rounded to the type."""
    x = np.asarray(x, np.float32)
    return x.astype(np.float64) if stream == "fp32" else bf16_bits_to_f64(f32_to_bf16_bits(x))


def f64(t):
    return t.detach().cpu().double().numpy()


class Out:
    """A device tensor of a shape, full of NaN (or 0x5A bytes), with a guard behind it."""

    def __init__(self, shape, dtype):
        import torch
        n = int(np.prod(shape))
        self.flat = torch.empty(n + GUARD, dtype=dtype, device="cuda")
        if dtype.is_floating_point:
            self.flat.fill_(float("nan"))
        else:
            self.flat.fill_(0x5A)
        self.t = self.flat[:n].view(*shape)
        self.before = self.flat[n:].clone()

    def check(self):
        import torch
        kept = self.flat[self.t.numel():]
        same = torch.equal(kept.view(torch.uint8), self.before.view(torch.uint8))
        assert same, "written behind the end of an output"
        return self.t


class Case:
    """Inputs of one call on CPU (float64, rounded to their types) and on the GPU."""

    def __init__(self, S, d, stream="bf16", gate_rows=0, weights=True, normalize=True, offset=0.0, scale=1.0, seed=0):
        import torch
        rng = np.random.default_rng([S, d, gate_rows, seed])
        self.S, self.d, self.stream, self.gate_rows, self.normalize, self.offset, self.scale = S, d, stream, gate_rows, normalize, offset, scale
        size = np.exp(0.5 * rng.standard_normal(d))
        size[rng.integers(0, d, max(1, d // 512))] *= 20
        self.x = rounded(rng.standard_normal((S, d)) * size, stream)
        self.y = rounded(rng.standard_normal((S, d)) * size, stream)
        self.o = rounded(rng.standard_normal((S, d)) * 0.7)
        self.dh = rounded(rng.standard_normal((S, d)) * 1e-3)
        self.dres = rounded(rng.standard_normal((S, d)) * 1e-3, stream)
        around_one = lambda: rounded(1 - offset + 0.2 * rng.standard_normal(d))  # noqa: E731
        self.w_pre = around_one() if weights else None
        self.w_post = around_one() if weights and normalize else None
        self.gate = rounded(rng.standard_normal((-(-S // gate_rows), d)) * 0.5) if gate_rows else None
        self.type = torch.float32 if stream == "fp32" else torch.bfloat16

    def gpu(self, name):
        import torch
        v = getattr(self, name)
        if v is None:
            return None
        return torch.tensor(v, dtype=torch.float32, device="cuda").to(self.type if name in ("x", "y", "dres") else torch.bfloat16)

    def rows(self, dtype=None):
        return Out((self.S, self.d), self.type if dtype is None else dtype)

    def checkpoint_room(self):
        import torch
        return Out((self.S, self.d), torch.int8), Out((self.S, -(-self.d // 32)), torch.uint8)

    def workspace(self):
        import torch
        import paper_2407_15892_amd as mst
        n = mst.mst_norm_workspace_bytes(self.S, self.d, self.gate_rows)
        w = Out((n,), torch.uint8)
        w.t.fill_(0xFF)          # NaN in every float
        return w


# A rounding to bf16 is off by at most half a step, 2^-8 of the value; fp32 outputs and what precedes the rounding by the
# errors of fp32 sums and products, at most (operations in a row) * 2^-24 of the reach (every term at its magnitude).
HALF_STEP = {"bf16": 2.0 ** -8, "fp32": 0.0}
# Operations in a row of a row's sum: 16 entries of a lane, 4 steps and 2 additions in a wave, 16 waves; the mean, eps, the root
# and the products around it: 24 more.  The backward of both norms has two such sums one after the other.
ROW_OPS = 16 + 6 + 16 + 24
TINY = 2.0 ** -134       # half a step of bf16's subnormals


def close(got, want, reach, ops, to="bf16"):
    got = f64(got) if not isinstance(got, np.ndarray) else got
    tol = HALF_STEP[to] * np.abs(want) + (1 + HALF_STEP[to]) * ops * 2.0 ** -24 * reach + TINY
    bad = ~(np.abs(got - want) <= tol)
    if bad.any():
        at = np.argwhere(bad)[0]
        raise AssertionError(f"{bad.sum()} of {bad.size} off, first at {at.tolist()}: {got[tuple(at)]} for {want[tuple(at)]}, "
                             f"tolerance {tol[tuple(at)]}; worst {np.nanmax(np.abs(got - want) / tol)} tolerances")


def column_ops(S, d, gate_rows=0, prenorm=True):
    """Operations in a row of a sum over rows: the rows of a team, the teams of a workgroup, then the workgroups: a 128th each, then
    7 steps; and the products with gate, weight and scale."""
    import paper_2407_15892_amd as mst
    info = mst.mst_norm_bwd_info(S, d, gate_rows, prenorm)
    return 2 * info["rows"] + info["teams"] + -(-info["workgroups"] // 128) + 7 + 4
