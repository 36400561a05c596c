"""The MLP's backward from a checkpoint where it takes another path than at the sizes of tests/test_gpu_block_parity.py: its bits are those
of the rebuilt input and mst_mlp_bwd."""
import numpy as np
import pytest

from tests.norm_gpu_harness import EPS, Out

pytestmark = pytest.mark.gpu


# rows of more than 8192 columns; a rebuilt input of more than the caches hold; dX in the memory of dO, a chunk of rows before it
@pytest.mark.parametrize("S,d,I,M,in_dO", [(70, 8200, 64, 1, False), (600, 8200, 48, 7, False), (16500, 4096, 64, 1, False), (1500, 136, 400, 30, True),
                                           (301, 264, 72, 5, True), (9, 40, 8, 1, True)])
@pytest.mark.parametrize("normalize", [True, False])
def test_bits_of_the_rebuilt_input(S, d, I, M, in_dO, normalize):
    import torch
    import paper_2407_15892_amd as mst
    gen = torch.Generator(device="cuda").manual_seed(S)
    normal = lambda *shape, std=1.0: torch.randn(shape, generator=gen, device="cuda").mul_(std).to(torch.bfloat16)  # noqa: E731
    f32, C = torch.float32, -(-S // M)
    x, upstream, w = normal(S, d), normal(S, d), normal(d, std=0.2) + 1
    Wg, Wu, Wd = normal(I, d, std=d ** -0.5), normal(I, d, std=d ** -0.5), normal(d, I, std=I ** -0.5)
    codes, exps = torch.empty((S, d), dtype=torch.int8, device="cuda"), torch.empty((S, -(-d // 32)), dtype=torch.uint8, device="cuda")
    mst.mst_ckpt_pack(x, codes, exps)
    X = torch.empty_like(x)
    if normalize:
        mst.mst_prenorm_rebuild(codes, exps, w, X, EPS, 0.25)
    else:
        mst.mst_ckpt_unpack(codes, exps, X)

    def run(call, need, *args, **kw):
        both, ws = Out((S + C, d), torch.bfloat16), Out((need,), torch.uint8)
        dO, dX = (both.t[C:], both.t[:S]) if in_dO else (upstream, both.t[:S])
        if in_dO:
            dO.copy_(upstream)
        sums = [Out(shape, f32) for shape in ((I, d), (I, d), (d, I))]
        call(*args, Wg, Wu, Wd, dO, M, ws.t, dX, *(o.t for o in sums), **kw)
        torch.cuda.synchronize()
        ws.check()
        both.check()
        return [dX.clone()] + [o.check() for o in sums]

    want = run(mst.mst_mlp_bwd, mst.mst_mlp_workspace_bytes(S, d, I, M)[1], X)
    got = run(mst.mst_mlp_bwd_ckpt, mst.mst_mlp_ckpt_workspace_bytes(S, d, I, M), codes, exps, w if normalize else None, normalize=normalize, eps=EPS,
              w_offset=0.25)
    for a, b in zip(got, want):
        assert torch.equal(a, b) and not a.isnan().any()
    # dX alone in 64 bits, so that both are not wrong alike: 8 rows
    rows = torch.from_numpy(np.unique(np.r_[0, S // 2, S - 1])).cuda()
    a = X[rows].double() @ Wg.double().T
    b, dA = X[rows].double() @ Wu.double().T, upstream[rows].double() @ Wd.double()
    s = torch.sigmoid(a)
    dX = (dA * b * s * (1 + a * (1 - s))) @ Wg.double() + (dA * a * s) @ Wu.double()
    # dA, dG and dU are rounded to bf16 before the products and dX behind them: 4 roundings of 2^-8 at most, of terms whose sum of squares is dX's
    assert float((got[0][rows].double() - dX).norm() / dX.norm()) <= 4 * 2.0 ** -8
