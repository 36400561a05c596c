"""Norm, residual and checkpoint calls on the GPU where values or arguments are at an edge (tolerances: tests/norm_gpu_harness.py)."""
import numpy as np
import pytest

from oracle import norm_oracle as orc
from tests.norm_gpu_harness import EPS, ROW_OPS, Case, Out, close, column_ops, f64

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def mst():
    import paper_2407_15892_amd as m
    return m


def on_gpu(a):
    import torch
    return torch.from_numpy(a).cuda()


# one chunk of columns per lane and two; rows of the gate shared by workgroups and whole ones of a team
@pytest.mark.parametrize("S,d,gate_rows,whole", [(37, 264, 10, False), (37, 264, 1, True), (40, 8200, 20, False), (300, 8200, 1, True)])
@pytest.mark.parametrize("stream", ["bf16", "fp32"])
@pytest.mark.parametrize("from_checkpoint", [True, False])
@pytest.mark.parametrize("parts", ["res", "both"])
def test_without_a_norm_dO_does_not_depend_on_O(mst, S, d, gate_rows, whole, stream, from_checkpoint, parts):
    """dO = scale * gate * dY also where O, which only dgate reads, has an infinity or a NaN."""
    import torch
    assert mst.mst_norm_bwd_info(S, d, gate_rows, parts == "both")["whole"] == whole
    c = Case(S, d, stream, gate_rows, normalize=False, scale=0.5)
    finite = c.o.copy()
    c.o[3, 5], c.o[4, 40], c.o[S - 1, d - 1] = np.inf, np.nan, -np.inf
    off = np.zeros((S, d), bool)                       # entries that are not finite: in dgate they may show, and nowhere else
    for r, j in ((3, 5), (4, 40), (S - 1, d - 1)):
        first, n = (j // 32 * 32, 32) if from_checkpoint else (j, 1)
        off[r, first:first + n] = True
    o = orc.restore(*orc.checkpoint(finite)) if from_checkpoint else finite
    f32 = torch.float32
    dY, dO, dg, dwp, ws = c.rows(), c.rows(torch.bfloat16), Out(c.gate.shape, f32), Out((d,), f32), c.workspace()
    codes, exps = orc.checkpoint(c.o)
    of_o = dict(O=c.gpu("o")) if not from_checkpoint else {"codes_o" if parts == "both" else "codes": on_gpu(codes),
                                                            "exps_o" if parts == "both" else "exps": on_gpu(exps)}
    branch = dict(gate=c.gpu("gate"), gate_rows=gate_rows, dgate=dg.t, scale=0.5, normalize=False, eps=EPS)
    if parts == "res":
        mst.mst_residual_bwd(c.gpu("dres"), dO.t, ws.t, **of_o, **branch)
        dy, reach, ops = c.dres, np.abs(c.dres), 0
    else:
        mst.mst_residual_prenorm_bwd(c.gpu("dh"), c.gpu("dres"), dY.t, dO.t, ws.t, c.gpu("w_pre"), dwp.t, Y=c.gpu("y"), **of_o, **branch)
        dy, _, reach, _ = orc.norm_bwd(c.dh, c.y, c.w_pre, 0.0, EPS)
        dy, reach, ops = dy + c.dres, reach + np.abs(c.dres), 2 * ROW_OPS
        close(dY.check(), dy, reach, ops, stream)
    want = orc.residual_bwd(dy, o, False, None, 0.0, EPS, c.gate, gate_rows, 0.5, reach)
    close(dO.check(), want["dO"], want["dO_reach"], ops + 2 * ROW_OPS)
    got, bad = f64(dg.check()), np.zeros(c.gate.shape, bool)
    np.logical_or.at(bad, np.arange(S) // gate_rows, off)
    assert not np.isfinite(got[bad]).any()
    ops += column_ops(S, d, gate_rows, parts == "both") + ROW_OPS
    close(np.where(bad, 0, got), np.where(bad, 0, want["dgate"]), want["dgate_reach"], ops, "fp32")
    ws.check()
