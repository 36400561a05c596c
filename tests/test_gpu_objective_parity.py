"""The LM head's weighted cross-entropy and distillation on the GPU against their definition in 64 bits, element by element."""
import numpy as np
import pytest

from tests.objective_gpu_harness import Problem, Run, check

pytestmark = pytest.mark.gpu

WCE = [
    # S, d, V, options
    (1, 8, 1, dict()),                                              # one class: everything is 0
    (1, 64, 300, dict(softcap=30.0)),
    (3, 16, 2, dict(softcap=5.0, weights=True)),
    (37, 72, 256, dict(z_coef=1e-2, weights=True)),
    (64, 128, 257, dict(softcap=2.0, z_coef=1e-3)),                 # the cap bends most logits
    (130, 136, 1000, dict(weights=True, M=3)),
    (255, 264, 511, dict(softcap=30.0, weights=True, M=2, divisor=1000)),
    (300, 520, 2048, dict(softcap=50.0, z_coef=1e-4, M=4)),
    (600, 64, 5003, dict(weights=True, softcap=1.0, sigma=0.5, M=2)),
    (257, 256, 8200, dict(z_coef=1e-4, sigma=6.0)),                 # sharp
    (40, 64, 300, dict(ignore=1.0, weights=True)),                  # no label at all
]
DISTILL = [
    (1, 8, 1, dict(K=1)),
    (1, 8, 1, dict(K=1, tail=True)),
    (1, 64, 300, dict(K=32, tail=True)),
    (5, 16, 7, dict(K=7, tail=True, label_coef=0.5)),               # the entries are the whole vocabulary
    (9, 16, 7, dict(K=5, tail=True, temperature=4.0, label_coef=0.5, weights=True)),
    (37, 72, 256, dict(K=256, temperature=2.0)),
    (64, 128, 257, dict(K=255, tail=True, softcap=5.0)),            # two others in most rows, in another tile or not
    (130, 136, 1000, dict(K=64, tail=True, label_coef=0.3, teacher_coef=0.7, weights=True, M=3, teacher="bf16")),
    (130, 136, 1000, dict(K=64, label_coef=0.3, teacher_coef=0.7, temperature=2.0, weights=True, M=3, teacher="bf16")),
    (255, 264, 511, dict(K=20, tail=True, label_coef=0.5, temperature=0.5, softcap=30.0, M=2, divisor=77)),
    (300, 520, 2048, dict(K=1, label_coef=0.5, M=4)),
    (257, 256, 8200, dict(K=128, tail=True, labels=False, sigma=6.0)),
    (600, 64, 5003, dict(K=200, tail=True, temperature=3.0, label_coef=0.1, M=2)),
    (70, 64, 300, dict(K=16, empty=1.0, label_coef=0.5)),           # no teacher at all
    (70, 64, 300, dict(K=16, ignore=1.0, empty=0.5, label_coef=0.5, temperature=2.0)),
]


def _ids(cases):
    return ["%dx%dx%d-%s" % (*c[:3], "-".join("%s=%s" % kv for kv in c[3].items())) for c in cases]


@pytest.mark.parametrize("S,d,V,o", WCE + DISTILL, ids=_ids(WCE + DISTILL))
def test_outputs_and_gradients(S, d, V, o):
    p = Problem(S, d, V, **o)
    run = Run(p)
    run.forward()
    run.backward(grad_loss=1.5)
    print(check(p, run.outputs(), p.oracle(1.5), 1.5))


@pytest.mark.parametrize("schedule", [1, 2, 3])
@pytest.mark.parametrize("o", [dict(K=40, tail=True, label_coef=0.5, temperature=2.0, weights=True), dict(softcap=20.0, weights=True, z_coef=1e-3)])
def test_orders_of_the_backward_pass(schedule, o):
    import paper_2407_15892_amd as mst
    p = Problem(700, 264, 3001, M=3, **o)
    run = Run(p)
    run.forward()
    mst.mst_set_bwd_schedule(schedule)
    try:
        run.backward()
        run.torch.cuda.synchronize()
    finally:
        mst.mst_set_bwd_schedule(mst.BWD_SCHEDULE_AUTO)
    print(check(p, run.outputs(), p.oracle()))


@pytest.mark.parametrize("rows", [20, 100, 200, 400, 1500])
def test_tiles_of_the_forward_pass(rows):
    """Every height of the forward's tiles, with entries at the borders of tiles and lanes."""
    import paper_2407_15892_amd as mst
    V = 12800
    p = Problem(rows, 64, V, K=48, tail=True, label_coef=0.5, temperature=2.0, softcap=10.0)
    edges = np.array([0, 1, 31, 32, 127, 128, 255, 256, 257, 511, 512, V - 1, V - 2, V - 256, V - 257], dtype=np.int32)
    for s in range(0, rows, 3):
        p.index[s, :] = -1
        p.index[s, 3:3 + len(edges)] = edges[::-1]
    print(mst.mst_forward_tile_rows(rows, 64, V, 1), mst.mst_forward_launch(rows, 64, V, 1))
    run = Run(p)
    run.forward()
    run.backward()
    print(check(p, run.outputs(), p.oracle()))


@pytest.mark.parametrize("S", [1, 2, 15, 16, 17, 31, 32, 33])
@pytest.mark.parametrize("d", [8, 72, 256, 776])
def test_a_few_rows(S, d):
    for o in (dict(K=33, tail=True, label_coef=0.5, temperature=2.0, weights=True), dict(softcap=4.0, z_coef=1e-3)):
        p = Problem(S, d, 1003, seed=S, **o)
        run = Run(p)
        run.forward()
        run.backward()
        print(check(p, run.outputs(), p.oracle()))


@pytest.mark.parametrize("S,d,V", [(17, 1032, 2049), (20, 8, 9000), (33, 1032, 4000), (100, 1032, 8000), (256, 1032, 4000), (400, 1032, 2100), (1000, 64, 700),
                                   (2000, 64, 500)])
def test_several_tiles_of_few_rows(S, d, V):
    """Several row tiles of 64 vocabulary entries, their losses from one workgroup (one, two, four or sixteen threads a row) or from two launches."""
    for o in (dict(K=33, tail=True, label_coef=0.5, temperature=2.0, weights=True), dict(softcap=4.0, z_coef=1e-3, weights=True)):
        p = Problem(S, d, V, **o)
        run = Run(p)
        run.forward()
        run.backward()
        print(check(p, run.outputs(), p.oracle()))


@pytest.mark.parametrize("S,d,V", [(5000, 72, 300), (9001, 264, 130), (20000, 64, 257), (6000, 1032, 40), (30001, 520, 8), (8191, 2048, 260)])
def test_many_rows_of_a_small_vocabulary(S, d, V):
    """The weights' gradient from parts of the rows; the same bits whatever M is."""
    for o in (dict(K=7, tail=True, label_coef=0.5, temperature=2.0, weights=True), dict(softcap=4.0, z_coef=1e-3, weights=True)):
        p = Problem(S, d, V, **o)
        run = Run(p)
        run.forward()
        run.backward(M=S // 300)
        first = run.dW.clone()
        run.backward()
        assert run.torch.equal(first, run.dW)
        print(check(p, run.outputs(), p.oracle()))


@pytest.mark.parametrize("S,d,V,mini_sequences", [(2300, 64, 150000, 3), (4196, 4096, 40960, 2)])
@pytest.mark.parametrize("o", [dict(K=30, tail=True, label_coef=0.5, temperature=2.0, weights=True), dict(softcap=20.0, weights=True, z_coef=1e-3)])
def test_several_mini_sequences(S, d, V, mini_sequences, o):
    """More than 512 MiB of float32 logits: every row's outputs and gradient are those of a call of its own rows (one mini-sequence),
    and the weights' gradient is the sum of these calls'.  The forward of the second shape deals its tiles out of queues, the calls of
    its parts do not."""
    import torch
    import paper_2407_15892_amd as mst
    assert (mst.mst_forward_launch(S, d, V, mini_sequences) == "queues") == (d == 4096)
    g = torch.Generator(device="cuda").manual_seed(5)
    H = torch.randn((S, d), generator=g, device="cuda").bfloat16()
    W = (torch.randn((V, d), generator=g, device="cuda") * 2 / d ** 0.5).bfloat16()
    labels = torch.randint(0, V, (S,), generator=g, device="cuda", dtype=torch.int32)
    labels[::7] = -100
    weights = torch.rand(S, generator=g, device="cuda") if o.get("weights") else None
    K = o.get("K", 0)
    if K:
        index = torch.randint(-1, V, (S, K), generator=g, device="cuda", dtype=torch.int32)
        index[:, :4] = index[:, :4] % 300
        logits = torch.randn((S, K), generator=g, device="cuda")
        lse = torch.full((S,), 6.0, device="cuda")

    def call(rows, M):
        n = len(range(*rows.indices(S)))
        f, b, sv = mst.mst_objective_bytes(n, d, V, M, K)
        ws, saved = (torch.empty(x, dtype=torch.uint8, device="cuda") for x in (max(f, b), sv))
        loss, cnt = torch.empty(1, device="cuda"), torch.empty(1, dtype=torch.int64, device="cuda")
        nll, other = torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
        dH, dW = torch.empty((n, d), dtype=torch.bfloat16, device="cuda"), torch.empty((V, d), device="cuda")
        kw = dict(saved=saved, weights=None if weights is None else weights[rows], divisor=1000, nll=nll, n_valid=cnt)
        if K:
            mst.mst_lmhead_distill_fwd(H[rows], W, index[rows], logits[rows], M, ws, loss, teacher_lse=lse[rows], labels=labels[rows],
                                       label_coef=0.5, temperature=2.0, kd=other, **kw)
            mst.mst_lmhead_distill_bwd(H[rows], W, K, M, 1.0, saved, ws, dH, dW)
        else:
            mst.mst_lmhead_wce_fwd(H[rows], W, labels[rows], -100, M, ws, loss, lse=other, softcap=20.0, z_coef=1e-3, **kw)
            mst.mst_lmhead_wce_bwd(H[rows], W, M, 1.0, saved, ws, dH, dW)
        return loss.double().item(), int(cnt), nll, other, dH, dW

    assert mst.mst_objective_bytes(S, d, V, 5, K)[1] == -(-S // mini_sequences) * V * 4
    whole = call(slice(0, S), 5)
    parts = [call(slice(a, b), 1) for a, b in ((0, 300), (300, 1000), (1000, 1500), (1500, S))]
    assert whole[1] == sum(p[1] for p in parts)
    assert abs(whole[0] - sum(p[0] for p in parts)) <= 8 * 2.0 ** -24 * sum(p[0] for p in parts)
    assert torch.equal(whole[2], torch.cat([p[2] for p in parts])) and torch.equal(whole[3], torch.cat([p[3] for p in parts]))
    # dH: the same logits' gradient, another split of the contraction and a bf16 rounding each: two half steps and little more
    dH = torch.cat([p[4] for p in parts]).double()
    assert ((whole[4].double() - dH).abs() <= 2 * 2.0 ** -8 * dH.abs() + 2.0 ** -12 * dH.abs().amax(1, keepdim=True)).all()
    # dW: float32 sums of the same terms in another order
    dW = sum(p[5].double() for p in parts)
    terms = sum(p[5].double().abs() for p in parts)
    assert ((whole[5].double() - dW).abs() <= 2.0 ** -16 * terms + 2.0 ** -20 * dW.abs().amax(1, keepdim=True)).all()
