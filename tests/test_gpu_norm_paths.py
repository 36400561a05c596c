"""The ways that the backward kernels go over rows, and tensors that are read past the caches, at sizes where real calls take
them: every output element by element against oracle/norm_oracle.py.

The rows of the inputs repeat with a short period, those of the gate with another, so that a few hundred rows of the oracle
stand for all of them; sums over rows are the oracle's rows times how often each of them comes."""
import numpy as np
import pytest

from oracle import norm_oracle as orc
from tests.norm_gpu_harness import EPS, HALF_STEP, ROW_OPS, TINY, Case, Out, column_ops, rounded

pytestmark = pytest.mark.gpu

CACHE = 192 << 20       # bytes of a call from which on its inputs are read past the caches


@pytest.fixture(scope="module")
def mst():
    import paper_2407_15892_amd as m
    return m


class Periodic:
    """S rows of which row r is row r % 64 of `tile`; gate row g is row g % 7 of `gates` (one row with gate_rows = 0)."""

    P, G = 64, 7

    def __init__(self, S, d, stream, gate_rows, normalize=True, scale=0.5):
        import torch
        self.S, self.d, self.stream, self.gate_rows, self.normalize, self.scale = S, d, stream, gate_rows, normalize, scale
        self.tile = Case(self.P, d, stream, normalize=normalize)
        G = self.G if gate_rows else 1
        rng = np.random.default_rng([S, d, gate_rows])
        self.gates = rounded(rng.standard_normal((G, d)) * 0.5) if gate_rows else None
        self.n_gates = -(-S // gate_rows) if gate_rows else 0
        row = np.arange(S)
        gate_of = row // gate_rows if gate_rows else np.zeros(S, np.int64)
        self.key = gate_of % G * self.P + row % self.P              # the row of the oracle's that a row is
        self.n_keys = G * self.P
        # how often a row of the tile comes in each row of the gate, a key in all
        self.in_gate = np.zeros((self.n_gates, self.P))
        if gate_rows:
            np.add.at(self.in_gate, (gate_of, row % self.P), 1)
        self.of_key = np.bincount(self.key, minlength=self.n_keys).astype(np.float64)
        self.of_tile = np.bincount(row % self.P, minlength=self.P).astype(np.float64)
        self.rows_of_tile = torch.from_numpy(row % self.P).cuda()
        self.key_gpu = torch.from_numpy(self.key).cuda()

    def gpu(self, name):
        import torch
        if name == "gate":
            if self.gates is None:
                return None
            g = torch.tensor(self.gates, dtype=torch.float32, device="cuda").to(torch.bfloat16)
            return g[torch.arange(self.n_gates, device="cuda") % self.G]
        t = self.tile.gpu(name)
        return t if t is None or t.dim() == 1 else t[self.rows_of_tile]

    def out(self, dtype=None):
        return Out((self.S, self.d), self.tile.type if dtype is None else dtype)

    def by_gate(self, f):
        """f(row of gates or None), which gives arrays of the tile's rows, for each of the gates: arrays of the keys' rows."""
        got = [f(None if self.gates is None else self.gates[g:g + 1]) for g in range(self.n_keys // self.P)]
        return [np.concatenate(a) for a in zip(*got)]

    def close_rows(self, got, want, reach, ops, to="bf16", by_key=True):
        """Every row of got, with the tolerance of tests/norm_gpu_harness.py."""
        import torch
        tol = HALF_STEP[to] * np.abs(want) + (1 + HALF_STEP[to]) * ops * 2.0 ** -24 * reach + TINY
        want, tol = torch.from_numpy(want).cuda(), torch.from_numpy(tol).cuda()
        which = self.key_gpu if by_key else self.rows_of_tile
        for r in range(0, self.S, 2048):
            at = which[r:r + 2048]
            off = (got[r:r + 2048].double() - want[at]).abs() / tol[at]
            worst = off.nan_to_num(nan=float("inf")).max().item()
            assert worst <= 1, (r, worst, off.argmax().item())

    def close_sums(self, got, want, reach, ops):
        got = got.double().cpu().numpy()
        off = np.abs(got - want) / (ops * 2.0 ** -24 * reach + TINY)
        assert not np.isnan(off).any() and off.max() <= 1, off.max()


def forward(mst, p, parts):
    import torch
    c, bf = p.tile, torch.bfloat16
    H, Y = p.out(bf), p.out()
    codes, exps = [Out((p.S, p.d), torch.int8) for _ in range(2)], [Out((p.S, -(-p.d // 32)), torch.uint8) for _ in range(2)]
    branch = dict(gate=p.gpu("gate"), gate_rows=p.gate_rows, scale=p.scale, normalize=p.normalize, eps=EPS)
    o, x = p.gpu("o"), p.gpu("x")
    stored = x
    if parts == "pre":
        mst.mst_prenorm_fwd(x, p.gpu("w_pre"), H.t, EPS, codes=codes[1].t, exps=exps[1].t)
        y, reach = c.x, np.abs(c.x)
    else:
        if parts == "res":
            mst.mst_residual_fwd(o, x, Y.t, w=p.gpu("w_post"), codes=codes[0].t, exps=exps[0].t, **branch)
        else:
            mst.mst_residual_prenorm_fwd(o, x, Y.t, H.t, p.gpu("w_pre"), w_post=p.gpu("w_post"), codes_o=codes[0].t, exps_o=exps[0].t,
                                         codes_y=codes[1].t, exps_y=exps[1].t, **branch)
        y, reach = p.by_gate(lambda g: orc.residual(c.o, c.x, p.normalize, c.w_post, 0.0, EPS, g, p.P, p.scale))
        p.close_rows(Y.check(), y, reach, ROW_OPS, p.stream)
        want = [on_gpu(a)[p.rows_of_tile] for a in orc.checkpoint(c.o)]
        assert torch.equal(codes[0].check(), want[0]) and torch.equal(exps[0].check(), want[1])
        stored = Y.t
    if parts == "res":
        return
    q = orc.rstd(y, EPS) * np.abs(orc.weight(c.w_pre, 0.0, p.d))
    h_reach = q * (reach + np.abs(y) * ((reach * np.abs(y)).mean(1, keepdims=True) / ((y * y).mean(1, keepdims=True) + EPS)))
    p.close_rows(H.check(), orc.prenorm(y, c.w_pre, 0.0, EPS), h_reach, 2 * ROW_OPS, by_key=parts == "both")
    # the checkpoint is that of Y as it is stored: the bits of the call that only packs
    again = Out((p.S, p.d), torch.int8), Out((p.S, -(-p.d // 32)), torch.uint8)
    mst.mst_ckpt_pack(stored, again[0].t, again[1].t)
    assert torch.equal(codes[1].check(), again[0].check()) and torch.equal(exps[1].check(), again[1].check())
    some = np.unique(np.r_[:min(3, p.S), p.S // 2, max(0, p.S - 3):p.S])
    want = orc.checkpoint(stored[torch.from_numpy(some).cuda()].cpu().double().numpy())
    assert np.array_equal(again[0].t[some].cpu().numpy(), want[0]) and np.array_equal(again[1].t[some].cpu().numpy(), want[1])


def on_gpu(a):
    import torch
    return torch.from_numpy(a).cuda()


def backward(mst, p, parts, from_checkpoint):
    import torch
    c, bf, f32 = p.tile, torch.bfloat16, torch.float32
    dX, dO, dwp = p.out(), p.out(bf), Out((p.d,), f32)
    dwo = Out((p.d,), f32) if p.normalize else None
    dg = Out((p.n_gates, p.d), f32) if p.gate_rows else None
    ws = Out((mst.mst_norm_workspace_bytes(p.S, p.d, p.gate_rows),), torch.uint8)
    ws.t.fill_(0xFF)
    t = lambda out: None if out is None else out.t  # noqa: E731
    y, o = c.y, c.o
    from_y, from_o = dict(Y=p.gpu("y")), dict(O=p.gpu("o"))
    if from_checkpoint:
        (cy, ey), (co, eo) = orc.checkpoint(c.y), orc.checkpoint(c.o)
        y, o = orc.restore(cy, ey), orc.restore(co, eo)
        from_y = dict(codes_y=on_gpu(cy)[p.rows_of_tile], exps_y=on_gpu(ey)[p.rows_of_tile])
        from_o = dict(codes_o=on_gpu(co)[p.rows_of_tile], exps_o=on_gpu(eo)[p.rows_of_tile])
    alone = lambda kw: {"X" if n == "Y" else n.split("_")[0]: v for n, v in kw.items()}  # noqa: E731
    branch = dict(gate=p.gpu("gate"), gate_rows=p.gate_rows, dgate=t(dg), scale=p.scale, normalize=p.normalize, eps=EPS)
    dres = p.gpu("dres")
    if parts == "pre":
        mst.mst_prenorm_bwd(p.gpu("dh"), p.gpu("w_pre"), dX.t, dwp.t, ws.t, EPS, dres=dres, **alone(from_y))
    elif parts == "res":
        mst.mst_residual_bwd(dres, dO.t, ws.t, w=p.gpu("w_post"), dw=t(dwo), **alone(from_o), **branch)
    else:
        mst.mst_residual_prenorm_bwd(p.gpu("dh"), dres, dX.t, dO.t, ws.t, p.gpu("w_pre"), dwp.t, w_post=p.gpu("w_post"), dw_post=t(dwo),
                                     **from_y, **from_o, **branch)
    torch.cuda.synchronize()
    ws.check()
    cols = column_ops(p.S, p.d, p.gate_rows if parts != "pre" else 0, parts != "res") + ROW_OPS
    dy, reach, ops = c.dres, np.abs(c.dres), 0
    if parts != "res":
        wt, q = orc.weight(c.w_pre, 0.0, p.d), orc.rstd(y, EPS)
        dy, _, reach, _ = orc.norm_bwd(c.dh, y, c.w_pre, 0.0, EPS)
        dy, reach, ops = dy + c.dres, reach + np.abs(c.dres), 2 * ROW_OPS
        p.close_rows(dX.check(), dy, reach, ops, p.stream, by_key=False)
        terms = c.dh * y * q
        p.close_sums(dwp.check(), p.of_tile @ terms, p.of_tile @ np.abs(terms), cols)
    if parts == "pre":
        return

    def by_row(g):                  # the tile as rows of one row of the gate; the terms of dw_post beside dO
        out = orc.residual_bwd(dy, o, p.normalize, c.w_post, 0.0, EPS, g, p.P, p.scale, reach)
        f = p.scale * (np.ones((1, p.d)) if g is None else g)
        n = o * orc.rstd(o, EPS)
        return out["dO"], out["dO_reach"], f * dy * n, np.abs(f) * reach * np.abs(n)

    dO_want, dO_reach, terms, terms_reach = p.by_gate(by_row)
    p.close_rows(dO.check(), dO_want, dO_reach, ops + 2 * ROW_OPS)
    if p.normalize:
        p.close_sums(dwo.check(), p.of_key @ terms, p.of_key @ terms_reach, ops + cols)
    if p.gate_rows:
        n = orc.branch(o, p.normalize, c.w_post, 0.0, EPS)
        p.close_sums(dg.check(), p.in_gate @ (p.scale * dy * n), p.in_gate @ (p.scale * reach * np.abs(n)), ops + cols)


def streamed(p, parts, from_checkpoint=None):
    """Whether the call's inputs and outputs are more than the caches hold (a checkpoint that a forward leaves is not counted)."""
    t, ck = (4 if p.stream == "fp32" else 2), from_checkpoint
    pre, res = parts != "res", parts != "pre"
    if ck is None:
        per = t + (2 if pre else 0) + (2 + t if res else 0)
    else:
        per = (2 + 2 * t + (1 if ck else t) if pre else t) + (3 if res else 0)
    return p.S * p.d * per > CACHE


# S * d is more than the caches hold of the smallest call, the norm's forward of bf16 (4 bytes an entry)
@pytest.mark.parametrize("parts,stream,gate_rows", [
    ("pre", "bf16", 0), ("pre", "fp32", 0),
    ("res", "bf16", 0), ("res", "bf16", 1), ("res", "fp32", 4301), ("res", "fp32", 5),
    ("both", "bf16", 4301), ("both", "bf16", 1), ("both", "fp32", 0), ("both", "fp32", 5)])
def test_tensors_that_the_caches_cannot_hold(mst, parts, stream, gate_rows):
    p = Periodic(12553, 4104, stream, gate_rows)
    assert streamed(p, parts)
    forward(mst, p, parts)
    for from_checkpoint in (True, False):
        assert streamed(p, parts, from_checkpoint)
        backward(mst, p, parts, from_checkpoint)


@pytest.mark.parametrize("parts,stream,gate_rows", [("both", "bf16", 1), ("both", "fp32", 3), ("res", "fp32", 2), ("pre", "bf16", 0)])
def test_long_rows_that_the_caches_cannot_hold(mst, parts, stream, gate_rows):
    p = Periodic(6301, 8200, stream, gate_rows)
    assert streamed(p, parts)
    forward(mst, p, parts)
    for from_checkpoint in (True, False):
        assert streamed(p, parts, from_checkpoint)
        backward(mst, p, parts, from_checkpoint)


@pytest.mark.parametrize("S,d,gate_rows", [(20011, 264, 3), (35004, 264, 7), (34003, 136, 4), (16391, 520, 3), (9001, 1032, 4), (4099, 4104, 5)])
@pytest.mark.parametrize("parts", ["res", "both"])
@pytest.mark.parametrize("stream", ["bf16", "fp32"])
def test_teams_that_take_one_row_of_the_gate_after_another(mst, S, d, gate_rows, parts, stream):
    """Whole rows of the gate, several to a team, the last one short."""
    info = mst.mst_norm_bwd_info(S, d, gate_rows, parts == "both")
    assert info["whole"] and info["workgroups"] > 1 and info["rows"] >= 2 * gate_rows and S % gate_rows
    for normalize in (True, False):
        p = Periodic(S, d, stream, gate_rows, normalize)
        for from_checkpoint in (True, False):
            backward(mst, p, parts, from_checkpoint)


LONG = [(701, 8200, 0), (701, 8200, 1), (701, 8200, 2), (701, 8200, 300), (523, 12288, 1), (1025, 12288, 3), (300, 16384, 0), (517, 16384, 1)]


@pytest.mark.parametrize("S,d,gate_rows,parts", [(*shape, parts) for shape in LONG for parts in ("pre", "res", "both") if parts != "pre" or not shape[2]])
@pytest.mark.parametrize("stream", ["bf16", "fp32"])
def test_many_long_rows(mst, S, d, gate_rows, parts, stream):
    """More than 8192 columns: two chunks of them per lane, teams that take several rows."""
    info = mst.mst_norm_bwd_info(S, d, gate_rows, parts != "res")
    assert info["rows"] >= 2 and info["whole"] == (gate_rows in (1, 2, 3))
    p = Periodic(S, d, stream, gate_rows)
    forward(mst, p, parts)
    for from_checkpoint in (True, False):
        backward(mst, p, parts, from_checkpoint)
