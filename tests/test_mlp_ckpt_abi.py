"""CPU-side checks of the MLP's backward from a checkpoint: workspace and refusals before anything is launched."""
import os

import pytest

NULL, SHAPE, BAD_M, WORKSPACE, ALIGNMENT, NO_DEVICE, ARGUMENT = -1, -2, -3, -4, -5, -7, -8
S, D, I, M = 64, 40, 96, 2


@pytest.fixture(scope="module")
def mst():
    import paper_2407_15892_amd as m
    if not os.path.exists(m.mlp_binding.MLP_LIB_PATH) or not os.path.exists(m.binding.LIB_PATH):
        from paper_2407_15892_amd.build import build
        build()
    m.load_mlp_library()
    return m


def P(i):
    return 0x100000 * (i + 1)      # never read: every call below is refused first


def call(mst, **change):
    good = dict(codes=P(0), exps=P(1), normalize=1, w=P(2), offset=0.0, eps=1e-5, Wg=P(3), Wu=P(4), Wd=P(5), dO=P(6), S=S, d=D, I=I, M=M,
                ws=P(7), size=mst.mst_mlp_ckpt_workspace_bytes(S, D, I, M), dX=P(8), dWg=P(9), dWu=P(10), dWd=P(11))
    assert set(change) <= set(good)
    return mst.load_mlp_library().mst_mlp_bwd_ckpt(*{**good, **change}.values(), None)


def test_workspace_holds_the_largest_group_beside_the_backward(mst):
    for s, d, i, m in ((S, D, I, M), (8192, 4096, 14336, 2), (1, 8, 8, 1), (5003, 1544, 5384, 3), (31999, 416, 1160, 77)):
        extra = mst.mst_mlp_ckpt_workspace_bytes(s, d, i, m) - mst.mst_mlp_workspace_bytes(s, d, i, m)[1]
        for overlaps in (False, True):
            largest = max(g["rows"] for g in mst.mst_mlp_bwd_groups(s, d, i, m, overlaps))
            assert extra >= largest * d * 2
        assert extra <= s * d * 2 + 255
    for bad, status in (((0, D, I, 1), SHAPE), ((S, 12, I, 1), SHAPE), ((S, 16392, 8, 1), SHAPE), ((S, D, I, 0), BAD_M)):
        with pytest.raises(mst.MstError) as e:
            mst.mst_mlp_ckpt_workspace_bytes(*bad)
        assert e.value.status == status


def test_refusals(mst):
    for n in ("codes", "exps", "Wg", "Wu", "Wd", "dO", "dX", "dWg", "dWu", "dWd"):
        assert call(mst, **{n: None}) == NULL, n
    assert call(mst, normalize=0) == ARGUMENT and call(mst, eps=0.0) == ARGUMENT and call(mst, offset=float("nan")) == ARGUMENT
    size = mst.mst_mlp_ckpt_workspace_bytes(S, D, I, M)
    assert call(mst, ws=None) == WORKSPACE and call(mst, size=size - 1) == WORKSPACE
    for n in ("codes", "w", "Wg", "Wu", "Wd", "dO", "dX", "dWg", "dWu", "dWd"):
        assert call(mst, **{n: P(20) + 8}) == ALIGNMENT, n
    assert call(mst, ws=P(20) + 128) == ALIGNMENT
    for out in ("dX", "dWg", "dWu", "dWd", "ws"):
        for n in ("codes", "exps", "w"):
            assert call(mst, **{out: P(20), n: P(20)}) == ARGUMENT, (out, n)
    assert call(mst, S=0) == SHAPE and call(mst, d=36) == SHAPE and call(mst, M=65) == BAD_M


def test_the_binding_refuses_wrong_tensors(mst):
    import torch
    bf, f32 = torch.bfloat16, torch.float32
    z = lambda *shape, dtype=bf: torch.zeros(shape, dtype=dtype)  # noqa: E731
    good = dict(codes=z(S, D, dtype=torch.int8), exps=z(S, 2, dtype=torch.uint8), w_pre=z(D), Wg=z(I, D), Wu=z(I, D), Wd=z(D, I), dO=z(S, D), M=M,
                workspace=z(1 << 20, dtype=torch.uint8), dX=z(S, D), dWg=z(I, D, dtype=f32), dWu=z(I, D, dtype=f32), dWd=z(D, I, dtype=f32))

    def status(**kw):
        with pytest.raises(mst.MstError) as e:
            mst.mst_mlp_bwd_ckpt(**{**good, **kw})
        return e.value.status

    assert status() == NO_DEVICE
    assert status(dO=z(S, D, dtype=f32)) == ARGUMENT and status(dWg=z(I, D)) == ARGUMENT and status(dX=z(S, D, dtype=f32)) == ARGUMENT
    assert status(Wd=z(I, D)) == SHAPE and status(dWd=z(I, D, dtype=f32)) == SHAPE and status(exps=z(S, 1, dtype=torch.uint8)) == SHAPE
    assert status(Wu=z(D, I).t()) == ARGUMENT
