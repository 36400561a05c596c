"""Two blocks with norms, gated residuals and the LM head, forward and backward as a training program calls them, with weights
that lie far apart: every gradient against 64 bits, within a bound that a wrong or a missing factor breaks."""
import numpy as np
import pytest

from tests.norm_gpu_harness import EPS, Out, f64, rounded
from tests.test_gpu_block_parity import bf16, reference

S, D, I, V, M, L, SCALE = 200, 264, 520, 1000, 3, 70, 0.8

# Relative to a gradient's 2-norm.  A checkpoint's rounding is uniform in a step of between 1 and 2 / 127.5 of the largest of 32 entries, which is
# about 2.1 standard deviations of them (2.7 where columns lie as far apart as here): off by at most 2 * 2.7 / 127.5 / sqrt(12)
# = 1.2 % of them.  A gradient goes through 6 uses of a checkpoint (5 norms' backward passes, of which 2 also rebuild the
# MLP's input), each of which moves it by at most about twice that.  The uses have roundings of their own, independent of each
# other: sqrt(6) * 2.4 % = 5.9 %.  About 20 roundings to bf16, uniform in a step of at most 2^-7 of the value: 2^-7 / sqrt(12) = 0.23 %
# each, sqrt(20) of them 1 %.  Together 6 %.
BOUND = 0.06


def inputs(stream):
    """Weights of 0.3 to 3, gates of both signs around 0.7."""
    rng = np.random.default_rng(23)
    spread = lambda: rounded(np.exp(0.5 * rng.standard_normal(D)))  # noqa: E731
    x = rounded(rng.standard_normal((S, D)), stream)
    blocks = [dict(w_pre=spread(), w_post=spread(), Wg=rounded(rng.standard_normal((I, D)) / D ** 0.5),
                   Wu=rounded(rng.standard_normal((I, D)) / D ** 0.5), Wd=rounded(rng.standard_normal((D, I)) / I ** 0.5)) for _ in range(2)]
    gates = [rounded(rng.standard_normal((3, D)) * 0.7) for _ in range(2)]
    return x, blocks, rounded(rng.standard_normal((V, D)) / D ** 0.5), rng.integers(0, V, S), gates


def gradients(x, blocks, W, y, gates, scale=SCALE):
    """Of the reference in 64 bits, by name."""
    _, dx, dblocks, dW, dgates, dfinal = reference(x, blocks, W, y, L, scale, gates)
    out = {"x": dx, "W": dW, "w_final": dfinal}
    for i in range(2):
        out.update({f"{i} {k}": v for k, v in dblocks[i].items()})
        out[f"{i} gate"] = dgates[i]
    return out


def off(got, want):
    return np.linalg.norm(got - want) / np.linalg.norm(want)


def ones_for(blocks, i, name):
    return [dict(b, **{name: np.ones(D)}) if j == i else b for j, b in enumerate(blocks)]


WRONG = {
    "the other block's w_pre": lambda b, g: ([dict(b[0], w_pre=b[1]["w_pre"]), dict(b[1], w_pre=b[0]["w_pre"])], g),
    "block 1 with block 0's w_pre": lambda b, g: ([b[0], dict(b[1], w_pre=b[0]["w_pre"])], g),
    "no w_pre in block 0": lambda b, g: (ones_for(b, 0, "w_pre"), g),
    "no w_post in block 0": lambda b, g: (ones_for(b, 0, "w_post"), g),
    "no w_post in block 1": lambda b, g: (ones_for(b, 1, "w_post"), g),
    "w_pre where w_post belongs": lambda b, g: ([dict(v, w_post=v["w_pre"]) for v in b], g),
    "the gates exchanged": lambda b, g: (b, g[::-1]),
    "the gate's first row for all": lambda b, g: (b, [np.repeat(v[:1], 3, 0) for v in g]),
}


@pytest.mark.parametrize("what", WRONG)
def test_the_bound_tells_a_wrong_factor(what):
    """With one factor wrong in the reference at least one gradient is off by more than twice the bound (no GPU)."""
    x, blocks, W, y, gates = inputs("bf16")
    want = gradients(x, blocks, W, y, gates)
    got = gradients(x, *(lambda b, g: (b, W, y, g))(*WRONG[what](blocks, gates)))
    assert max(off(got[k], want[k]) for k in want) > 2 * BOUND


@pytest.mark.gpu
@pytest.mark.parametrize("stream", ["bf16", "fp32"])
def test_every_gradient_of_a_training_step(stream):
    import torch
    import paper_2407_15892_amd as mst
    x, blocks, W, y, gates = inputs(stream)
    bf, f32 = torch.bfloat16, torch.float32
    dtype = f32 if stream == "fp32" else bf
    new = lambda *shape, dtype=bf: Out(shape, dtype).t  # noqa: E731
    room = lambda: (new(S, D, dtype=torch.int8), new(S, -(-D // 32), dtype=torch.uint8))  # noqa: E731
    b = [{k: bf16(v) for k, v in block.items()} for block in blocks]
    g, head, final = [bf16(v) for v in gates], bf16(W), torch.ones(D, dtype=bf, device="cuda")
    after = [b[1]["w_pre"], final]                       # weight of the norm behind each block
    labels = torch.tensor(y, dtype=torch.int32, device="cuda")
    ck, ck_o = [room() for _ in range(3)], [room() for _ in range(2)]
    ws = new(max(mst.mst_norm_workspace_bytes(S, D, L), mst.mst_norm_workspace_bytes(S, D), mst.mst_mlp_ckpt_workspace_bytes(S, D, I, M),
                 *mst.mst_workspace_bytes(S, D, V, M)), dtype=torch.uint8)
    junction = lambda i: dict(w_post=b[i]["w_post"], gate=g[i], gate_rows=L, scale=SCALE, eps=EPS, codes_o=ck_o[i][0], exps_o=ck_o[i][1],  # noqa: E731
                              codes_y=ck[i + 1][0], exps_y=ck[i + 1][1])

    X, H = torch.tensor(x, dtype=f32, device="cuda").to(dtype), new(S, D)
    mst.mst_prenorm_fwd(X, b[0]["w_pre"], H, EPS, codes=ck[0][0], exps=ck[0][1])
    for i in range(2):
        O, Y, next_H = new(S, D), new(S, D, dtype=dtype), new(S, D)
        mst.mst_mlp_fwd(H, b[i]["Wg"], b[i]["Wu"], b[i]["Wd"], M, ws, O)
        mst.mst_residual_prenorm_fwd(O, X, Y, next_H, after[i], **junction(i))
        X, H = Y, next_H
    loss, lse, n_valid = new(1, dtype=f32), new(S, dtype=f32), torch.empty(1, dtype=torch.int64, device="cuda")
    mst.mst_lmhead_ce_fwd(H, head, labels, -100, M, ws, loss, lse, n_valid)

    dH, dW, got = new(S, D), new(V, D, dtype=f32), {}
    mst.mst_lmhead_ce_bwd(H, head, labels, -100, M, 1.0, lse, n_valid, ws, dH, dW)
    dres, got["W"] = None, dW
    for i in (1, 0):
        dY, dO, dw_after, dw_post, dg = new(S, D, dtype=dtype), new(S, D), new(D, dtype=f32), new(D, dtype=f32), new(3, D, dtype=f32)
        mst.mst_residual_prenorm_bwd(dH, dres, dY, dO, ws, after[i], dw_after, dw_post=dw_post, dgate=dg, **junction(i))
        got["w_final" if i == 1 else "1 w_pre"] = dw_after
        got.update({f"{i} w_post": dw_post, f"{i} gate": dg})
        dH, dWg, dWu, dWd = new(S, D), new(I, D, dtype=f32), new(I, D, dtype=f32), new(D, I, dtype=f32)
        mst.mst_mlp_bwd_ckpt(*ck[i], b[i]["w_pre"], b[i]["Wg"], b[i]["Wu"], b[i]["Wd"], dO, M, ws, dH, dWg, dWu, dWd, eps=EPS)
        got.update({f"{i} Wg": dWg, f"{i} Wu": dWu, f"{i} Wd": dWd})
        dres = dY
    dX, dw = new(S, D, dtype=dtype), new(D, dtype=f32)
    mst.mst_prenorm_bwd(dH, b[0]["w_pre"], dX, dw, ws, EPS, codes=ck[0][0], exps=ck[0][1], dres=dres)
    got.update({"x": dX, "0 w_pre": dw})
    torch.cuda.synchronize()
    want = gradients(x, blocks, W, y, gates)
    assert set(got) == set(want)
    far = {k: off(f64(got[k]), want[k]) for k in want}
    print(stream, {k: round(float(v), 4) for k, v in far.items()}, flush=True)
    assert max(far.values()) <= BOUND, far
