"""The LM head's weighted cross-entropy and distillation where they can go wrong: lists with gaps, indices that come twice, logits of
-infinity, teachers that give more than 1, saturated caps, values that are not finite, bad indices; streams, graphs and calls that share what
they may share."""
import numpy as np
import pytest
import torch

import paper_2407_15892_amd as mst
from oracle import objective_oracle as orc
from tests.objective_gpu_harness import HALF_BF16, HALF_FP32, Problem, Run, bf16, check

pytestmark = pytest.mark.gpu

SIZES = [(20, 64, 300), (300, 72, 3000), (1500, 64, 12800)]      # tiles of 64, of 256 x 32 and of 256 x 256
TOGETHER = dict(tail=True, label_coef=0.4, temperature=2.0, weights=True)


def both(S, d, V, **o):
    return [Problem(S, d, V, K=min(40, V // 4), **{**TOGETHER, **o}), Problem(S, d, V, softcap=20.0, weights=True, z_coef=1e-3, **o)]


def run_and_check(p, grad_loss=1.0):
    r = Run(p)
    r.forward()
    r.backward(grad_loss)
    got = r.outputs()
    print(check(p, got, p.oracle(grad_loss), grad_loss))
    return r, got


@pytest.mark.parametrize("S,d,V", SIZES)
def test_an_index_that_comes_twice_counts_once(S, d, V):
    p = Problem(S, d, V, K=40, **TOGETHER)
    for s in range(0, S, 2):
        at = np.flatnonzero(p.index[s] >= 0)
        if len(at) > 6:
            p.index[s, at[-1]], p.index[s, at[3]], p.index[s, at[4]] = p.index[s, at[0]], p.index[s, at[2]], p.index[s, at[2]]
    if S < 64:
        p.index[1] = p.index[1, 0] if p.index[1, 0] >= 0 else 5      # one entry, forty times
    run_and_check(p)


@pytest.mark.parametrize("S,d,V", SIZES)
@pytest.mark.parametrize("tail", [False, True])
def test_logits_of_minus_infinity(S, d, V, tail):
    p = Problem(S, d, V, K=30, tail=tail, label_coef=0.5)
    p.logits[::2, 3:9] = -np.inf
    p.logits[::5] = -np.inf                                          # no teacher, or one that gives all to the others
    run_and_check(p)


@pytest.mark.parametrize("S,d,V", SIZES)
@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("temperature", [0.02, 1.0])
def test_masks_of_the_lowest_value_and_shares_that_are_next_to_nothing(S, d, V, tail, temperature):
    p = Problem(S, d, V, K=30, sigma=2.0 * temperature, tail=tail, temperature=temperature, empty=0)
    p.logits *= temperature                                          # so that shares are what they are at temperature 1
    if tail:
        p.lse = np.float32([orc._lse(1.5 * h @ p.W.T / temperature) for h in p.H]).astype(np.float64)
    top = p.lse if tail else (p.logits / temperature).max(1)         # exp(-95): float32 has it, but not its reciprocal
    p.logits[:, 3] = np.float32((top - 95.0) * temperature)
    p.logits[:, 4:8] = np.float32(-3.0e38)
    run = Run(p)
    run.forward()
    run.backward()
    p.logits[:, 4:8] = -np.inf                                       # what their shares come to, and the bounds count finite ones
    print(check(p, run.outputs(), p.oracle()))


@pytest.mark.parametrize("S,d,V", SIZES)
def test_what_is_not_asked_for_may_hold_anything(S, d, V):
    """Logits of missing entries, the log-sum-exp of a row without a teacher, the weight of a row without a loss."""
    for p in both(S, d, V):
        ref = p.oracle()
        nothing = p.labels == -100
        if p.K:
            p.logits[p.index < 0] = np.nan
            p.lse[(p.index < 0).all(1)] = np.inf
            nothing &= (p.index < 0).all(1)
            nothing[3], p.labels[3], p.index[3] = True, -100, -1
            ref = p.oracle()
        p.weights[nothing] = np.nan
        run = Run(p)
        run.forward()
        run.backward()
        p.weights[nothing] = 1.0
        if p.K:
            p.logits[p.index < 0], p.lse[(p.index < 0).all(1)] = 0.0, 0.0
        print(check(p, run.outputs(), ref))


@pytest.mark.parametrize("S,d,V", SIZES)
def test_labels_that_only_count(S, d, V):
    """A coefficient of 0 for the labels and no losses of theirs asked for: one log-sum-exp is enough."""
    p = Problem(S, d, V, K=30, tail=True, temperature=2.5)
    run = Run(p)
    run.nll = None
    run.forward()
    run.backward()
    print(check(p, run.outputs(), p.oracle()))


@pytest.mark.parametrize("S,d,V", SIZES)
def test_all_entries_in_one_tile(S, d, V):
    p = Problem(S, d, V, K=200, **TOGETHER)
    rng = np.random.default_rng(1)
    for s in range(S):
        p.index[s] = rng.permutation(256)[:200] + (0 if s % 3 else V - 256)
    run_and_check(p)


@pytest.mark.parametrize("S,d,V", SIZES)
def test_teacher_that_gives_more_than_1(S, d, V):
    p = Problem(S, d, V, K=30, **TOGETHER)
    p.lse = np.float32(p.lse - 3.0).astype(np.float64)              # shares of 20 in all: nothing is left for the others
    run_and_check(p)


@pytest.mark.parametrize("cap", [0.01, 0.5, 1e5])
def test_caps_that_bend_everything_and_nothing(cap):
    for o in (dict(K=30, **TOGETHER), dict(weights=True)):
        run_and_check(Problem(100, 64, 1000, softcap=cap, **o))


def test_confident_student():
    """The student gives all but 1e-10 of itself to the entries, the teacher 0.7: what is left for the others has to be formed of
    the others."""
    S, d, V = 64, 64, 600
    p = Problem(S, d, V, K=2, labels=False, short=0, empty=0, weights=False, tail=True)
    rng = np.random.default_rng(2)
    p.W[:] = 0
    p.W[:2, 0] = 4.0
    p.W[2:, 1] = rng.choice([-0.125, 0.0, 0.125], V - 2)
    p.H[:] = 0
    p.H[:, 0], p.H[:, 1] = 8.0, 1.0
    p.index[:] = [1, 0]
    p.logits[:] = [1.0, 1.5]
    p.lse = np.float32(np.full(S, np.log((np.e + np.exp(1.5)) / 0.7))).astype(np.float64)
    r, got = run_and_check(p)
    ref = p.oracle()
    assert ref["kd"].min() > 5 and np.abs(got["rows"] / ref["kd"] - 1).max() < 1e-5


@pytest.mark.parametrize("S,d,V,K", [(1, 384, 20000, 6), (30, 80, 3000, 9), (400, 128, 14144, 9), (2000, 64, 12800, 100)])
@pytest.mark.parametrize("tail", [False, True])
def test_softened_distributions_that_are_nearly_the_same(S, d, V, K, tail):
    """A divergence of shares that add up to 1 is off by (p - q) times what the logarithms of shares are off by, added up: no more than
    the largest of these times sum |p - q|, which is at most sqrt(2 kd)."""
    p = Problem(S, d, V, K=K, tail=tail, labels=False, temperature=4.0, sigma=1.5, short=0, empty=0)
    if not tail:                                                     # entries that are nearly all of the student's distribution
        p.W[:K, 0] = bf16(np.abs(p.W[:K, 0]) + 8.0)                    # as the GPU holds it
        p.H[:, 0] = 16.0
        p.index[:] = np.arange(K)
        p.logits = np.float32(p.H @ p.W[:K].T + 0.1 * np.random.default_rng(3).standard_normal((S, K))).astype(np.float64)
    run = Run(p)
    run.forward()
    run.backward()
    got, ref = run.outputs(), p.oracle()
    largest = max(np.abs(ref["Z"]).max(), np.abs(p.logits).max(), 1.0)
    arg = (8 * np.sqrt(d) * HALF_FP32 * largest + 16 * HALF_FP32 * (largest + np.log(V))) / 4 + 16 * HALF_FP32
    off = np.abs(got["rows"] - ref["kd"])
    bound = arg * np.sqrt(2 * ref["kd"]) + 16 * HALF_FP32 * ref["kd"] + arg * arg
    print(ref["kd"].min(), ref["kd"].max(), (off / ref["kd"]).max(), (off / bound).max())
    assert (off <= bound).all()
    print(check(p, got, ref))


@pytest.mark.parametrize("S,d,V", SIZES)
def test_rows_of_weight_zero(S, d, V):
    for p in both(S, d, V):
        p.weights[:] = np.where(np.arange(S) % 2, 1.0, 0.0)
        _, got = run_and_check(p)
        assert not got["dH"][::2].any()


@pytest.mark.parametrize("S,d,V", SIZES)
def test_ignore_index_that_is_an_entry_of_the_vocabulary(S, d, V):
    p = Problem(S, d, V, ignore=0.0)
    p.labels[::3] = 7
    run = Run(p)
    mst.mst_lmhead_wce_fwd(run.H, run.W, run.labels, 7, 1, run.ws, run.loss, saved=run.saved, nll=run.nll, lse=run.rows, n_valid=run.n)
    run.backward()
    got = run.outputs()
    p.labels[p.labels == 7] = -100
    print(check(p, got, p.oracle()))


@pytest.mark.parametrize("S,d,V", SIZES)
@pytest.mark.parametrize("bad", ["label", "entry", "far entry"])
def test_indices_out_of_range(S, d, V, bad):
    """Reported, not followed: NaN and -1, gradients of NaN, the other rows' outputs as they are."""
    p = Problem(S, d, V, K=20, **TOGETHER)
    good = p.oracle()
    if bad == "label":
        p.labels[3] = V
    else:
        p.index[3, 5] = V if bad == "entry" else 2**31 - 1
    run = Run(p)
    run.forward()
    run.backward()
    got = run.outputs()
    assert np.isnan(got["loss"]) and got["n"] == -1
    assert np.isnan(got["dH"]).all() and np.isnan(got["dW"]).all()
    others = np.arange(S) != 3
    np.testing.assert_allclose(got["nll"][others], good["nll"][others], rtol=1e-4, atol=1e-5)
    np.testing.assert_allclose(got["rows"][others], good["kd"][others], rtol=1e-4, atol=1e-5)


@pytest.mark.parametrize("S,d,V", SIZES)
def test_values_that_are_not_finite_stay_in_their_rows(S, d, V):
    for p in both(S, d, V):
        good = p.oracle()
        p.H[5, 3], p.H[7, 2] = np.nan, np.inf
        run = Run(p)
        run.forward(saved=False)
        got = run.outputs()
        others = ~np.isin(np.arange(S), [5, 7])
        ref = good["kd"] if p.K else good["lse"]
        np.testing.assert_allclose(got["rows"][others], ref[others], rtol=1e-4, atol=1e-5)
        assert got["n"] == good["n"]


@pytest.mark.parametrize("S,d,V", SIZES)
def test_calls_repeat_bit_by_bit_and_share_nothing(S, d, V):
    """The same bits from every call, for every M that gives the same mini-sequences, without `saved`, in a workspace that another
    call has used, from two backward calls of one forward call, and on a stream beside another call's."""
    a, b = both(S, d, V)
    ra, rb = Run(a), Run(b)
    ra.forward()
    ra.backward()
    first = {k: v.clone() for k, v in (("dH", ra.dH), ("dW", ra.dW), ("loss", ra.loss), ("rows", ra.rows), ("nll", ra.nll))}
    same = lambda r: all(torch.equal(getattr(r, k), v) for k, v in first.items())  # noqa: E731
    ra.backward(M=min(S, 7))
    assert same(ra)
    other = Run(a)
    other.ws = ra.ws
    rb.forward()
    rb.backward()
    other.forward()
    other.backward()
    assert same(other)
    side = torch.cuda.Stream()
    ra.dH.zero_(), ra.dW.zero_()
    side.wait_stream(torch.cuda.current_stream())
    for _ in range(3):
        ra.forward(stream=side)
        ra.backward(stream=side)
        rb.forward()
        rb.backward()
    torch.cuda.synchronize()
    assert same(ra)
    ra.loss.zero_(), ra.rows.zero_()
    ra.forward(saved=False)
    assert same(ra)
    ra.outputs()


@pytest.mark.parametrize("S,d,V", SIZES)
def test_a_captured_step_follows_its_inputs(S, d, V):
    for p in both(S, d, V):
        r = Run(p)
        r.forward()
        r.backward()
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            r.forward()
            r.backward()
        for k in range(3):
            q = both(S, d, V, seed=k + 1)[0 if p.K else 1]
            eager = Run(q)
            eager.forward()
            eager.backward()
            for name in ("H", "W", "labels", "weights", "index", "logits", "lse_in"):
                if getattr(r, name) is not None:
                    getattr(r, name).copy_(getattr(eager, name))
            g.replay()
            torch.cuda.synchronize()
            for name in ("loss", "n", "nll", "rows", "dH", "dW"):
                assert torch.equal(getattr(r, name), getattr(eager, name)), (k, name)


def test_scoring_weights_and_distillation_over_micro_batches():
    """As a program uses them together: a reference head scores the tokens, the scores become the tokens' weights, and a step of two
    micro-batches learns from the teacher and the labels, divided by the tokens of both."""
    S, d, V, K = 500, 136, 2000, 24
    whole = Problem(S, d, V, K=K, tail=True, label_coef=0.3, teacher_coef=0.7, temperature=2.0, softcap=30.0)
    whole.weights = np.ones(S, dtype=np.float32)
    reference = Problem(S, d, V, seed=9)
    parts = []
    dW = torch.zeros((V, d), device="cuda")
    n_all = int(((whole.labels != -100) | (whole.index >= 0).any(1)).sum())
    full = Run(whole)
    ws = torch.empty(max(mst.mst_objective_bytes(S, d, V, 4, 0)[0], *mst.mst_objective_bytes(S, d, V, 4, K)[:2]), dtype=torch.uint8, device="cuda")
    score, loss = torch.empty(S, device="cuda"), torch.empty(1, device="cuda")
    mst.mst_lmhead_wce_fwd(full.H, Run(reference).W, full.labels, -100, 4, ws, loss, nll=score)
    weights = torch.where(full.labels != -100, torch.sigmoid(score - 8.0), 1.0)
    whole.weights = weights.cpu().numpy()
    for rows in (slice(0, 200), slice(200, S)):
        n = rows.stop - rows.start
        saved = torch.empty(mst.mst_objective_bytes(n, d, V, 2, K)[2], dtype=torch.uint8, device="cuda")
        dH, dWp = torch.empty((n, d), dtype=torch.bfloat16, device="cuda"), torch.empty((V, d), device="cuda")
        part, cnt = torch.empty(1, device="cuda"), torch.empty(1, dtype=torch.int64, device="cuda")
        kd, nll = torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
        mst.mst_lmhead_distill_fwd(full.H[rows], full.W, full.index[rows], full.logits[rows], 2, ws, part, saved=saved, teacher_lse=full.lse_in[rows],
                                   labels=full.labels[rows], weights=weights[rows], divisor=n_all, nll=nll, kd=kd, n_valid=cnt, **whole.objective)
        mst.mst_lmhead_distill_bwd(full.H[rows], full.W, K, 2, 1.0, saved, ws, dH, dWp)
        dW += dWp
        parts.append((part, cnt, nll, kd, dH))
    ref = whole.oracle()
    assert sum(int(p[1]) for p in parts) == n_all == ref["n"]
    f = lambda t: t.double().cpu().numpy()  # noqa: E731
    got = {"loss": sum(float(p[0]) for p in parts), "n": n_all, "nll": f(torch.cat([p[2] for p in parts])), "rows": f(torch.cat([p[3] for p in parts])),
           "dH": f(torch.cat([p[4] for p in parts])), "dW": f(dW)}
    print(check(whole, got, ref))


def test_step_of_blocks_and_distilling_head():
    """The norm before the head, the head's distillation and the norm's gradient in a row, against the definition of each."""
    from oracle import norm_oracle as norc
    S, d, V, K = 200, 256, 1000, 20
    p = Problem(S, d, V, K=K, **TOGETHER)
    rng = np.random.default_rng(4)
    bf = torch.bfloat16
    X = torch.from_numpy(rng.standard_normal((S, d)) * 3).to("cuda", bf)
    w = torch.from_numpy(1 + 0.2 * rng.standard_normal(d)).to("cuda", bf)
    run = Run(p)
    codes, exps = torch.empty((S, d), dtype=torch.int8, device="cuda"), torch.empty((S, d // 32), dtype=torch.uint8, device="cuda")
    dX, dw = torch.empty_like(X), torch.empty(d, device="cuda")
    mst.mst_prenorm_fwd(X, w, run.H, eps=1e-5, codes=codes, exps=exps)
    p.H = run.H.double().cpu().numpy()
    run.forward()
    run.backward()
    ws = torch.empty(mst.mst_norm_workspace_bytes(S, d), dtype=torch.uint8, device="cuda")
    mst.mst_prenorm_bwd(run.dH, w, dX, dw, ws, eps=1e-5, codes=codes, exps=exps)
    got = run.outputs()
    print(check(p, got, p.oracle()))
    dx, dw_ref, _, _ = norc.norm_bwd(got["dH"], norc.restore(codes.cpu().numpy(), exps.cpu().numpy()), w.double().cpu().numpy(), 0.0, 1e-5)
    assert np.abs(dX.double().cpu().numpy() - dx).max() <= 2 * HALF_BF16 * np.abs(dx).max()
    assert np.abs(dw.double().cpu().numpy() - dw_ref).max() <= 1e-4 * np.abs(dw_ref).max()
