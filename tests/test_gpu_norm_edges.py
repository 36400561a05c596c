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


def launches_of(call):
    """Kernels that a call enqueues: the nodes of the HIP graph that it is captured into."""
    import ctypes
    import torch
    call()                                      # eager once, as the header asks
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph(keep_graph=True)
    with torch.cuda.graph(graph):
        call()
    n = ctypes.c_size_t(0)
    status = ctypes.CDLL(None).hipGraphGetNodes(ctypes.c_void_p(graph.raw_cuda_graph()), None, ctypes.byref(n))
    assert status == 0
    return n.value


# whether teams take whole rows of the gate and write their gradients; workgroups; with a weight's gradient to sum up
@pytest.mark.parametrize("S,gate_rows,whole,normalize,launches", [
    (37, 1, True, False, 1), (37, 1, True, True, 2), (37, 10, False, False, 2), (37, 10, False, True, 2), (3, 1, True, True, 1), (3, 3, False, True, 1)])
def test_sums_of_workgroups_are_launched_only_where_there_are_any(mst, S, gate_rows, whole, normalize, launches):
    import torch
    d, f32 = 264, torch.float32
    info = mst.mst_norm_bwd_info(S, d, gate_rows, False)
    assert info["whole"] == whole and (info["workgroups"] == 1) == (S == 3)
    c = Case(S, d, gate_rows=gate_rows, normalize=normalize)
    dO, dg, ws = c.rows(torch.bfloat16), Out(c.gate.shape, f32), c.workspace()
    dw = Out((d,), f32).t if normalize else None
    args = dict(dY=c.gpu("dres"), O=c.gpu("o"), w=c.gpu("w_post"), gate=c.gpu("gate"))
    assert launches_of(lambda: mst.mst_residual_bwd(dO=dO.t, workspace=ws.t, dw=dw, dgate=dg.t, gate_rows=gate_rows, normalize=normalize,
                                                    eps=EPS, **args)) == launches
    torch.cuda.synchronize()
    want = orc.residual_bwd(c.dres, c.o, normalize, c.w_post, 0.0, EPS, c.gate, gate_rows, 1.0)
    close(dg.check(), want["dgate"], want["dgate_reach"], column_ops(S, d, gate_rows, False) + ROW_OPS, "fp32")
