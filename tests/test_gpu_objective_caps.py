"""Caps of the logits from far below to far above them, on the GPU: losses, divergences and gradients under bounds that are relative to
the capped logits, and equal to the uncapped ones where the cap bends nothing."""
import numpy as np
import pytest

from tests.objective_gpu_harness import HALF_FP32, Problem, Run, bf16
from tests.objective_tight_bounds import check

pytestmark = pytest.mark.gpu

SIZES = [(20, 64, 300), (130, 72, 9000), (200, 72, 12800), (400, 72, 12800), (1500, 64, 12800)]      # tiles of 64 x 32, of 256 x 32, 64, 128 and 256
TEACHER = dict(K=30, tail=True, label_coef=0.5, temperature=2.0, weights=True)


@pytest.mark.parametrize("S,d,V", SIZES)
@pytest.mark.parametrize("cap", [0.25, 3.0, 9.0, 30.0, 100.0, 1e3, 1e4, 1e5, 1e6])
@pytest.mark.parametrize("o", [TEACHER, dict(weights=True, z_coef=1e-3)], ids=["distill", "wce"])
def test_a_cap_costs_no_precision(S, d, V, cap, o):
    p = Problem(S, d, V, softcap=cap, **o)
    run = Run(p)
    run.forward()
    run.backward()
    print(check(p, run.outputs(), p.oracle()))


@pytest.mark.parametrize("S,d,V", SIZES)
@pytest.mark.parametrize("cap", [1e3, 1e4, 1e5, 1e6])
def test_a_cap_far_above_the_logits_is_none(S, d, V, cap):
    """The same products with and without the cap: capped logits differ by z^3 / (3 c^2) at most and by their roundings, 8 half steps of
    them; log-sum-exps by as much, and by 16 half steps of the largest number that they are made of."""
    for o in (dict(K=30, label_coef=0.5), dict(z_coef=1e-3)):
        got = {}
        for c in (0.0, cap):
            p = Problem(S, d, V, softcap=c, **o)
            run = Run(p)
            run.forward(saved=False)
            got[c] = run.outputs()
        r = p.oracle()
        largest = np.abs(r["Z"]).max()
        y = largest ** 3 / (3 * cap ** 2) + 8 * HALF_FP32 * largest
        row = 2 * y + 16 * HALF_FP32 * (largest + np.log(V))
        off = {k: np.abs(got[0.0][k] - got[cap][k]).max() for k in (("nll",) if p.K else ("nll", "rows"))}
        print({k: v / row for k, v in off.items()})
        assert all(v <= row for v in off.values()), off


@pytest.mark.parametrize("S,d,V", SIZES)
def test_logits_next_to_nothing(S, d, V):
    """Logits of 1e-3 under a cap of 30: an error of some half steps of the cap would be a few per cent of what tells them apart."""
    p = Problem(S, d, V, sigma=1e-3, softcap=30.0, ignore=0.0)
    run = Run(p)
    run.forward()
    got, r = run.outputs(), p.oracle()
    # nll - log V is a difference of logits; those of one call share the log-sum-exp's error, 16 half steps of log V
    off = np.abs(got["nll"] - r["nll"])
    bound = 4 * np.sqrt(d) * HALF_FP32 * np.abs(r["Z"]).max() + 16 * HALF_FP32 * np.log(V)
    print((off / bound).max())
    assert (off <= bound).all()


@pytest.mark.parametrize("S,d,V", [(64, 64, 300), (130, 64, 9000), (400, 64, 12800), (1500, 64, 12800)])
@pytest.mark.parametrize("o", [dict(tail=True), dict(label_coef=0.5, temperature=2.0), dict(label_coef=0.5)], ids=str)
def test_slope_at_the_entries_of_a_saturated_cap(S, d, V, o):
    """Up to 13 caps from 0 the slope is 4 exp(-2 |z| / c), as at other vocabulary entries.  Row s is the s-th unit vector, so that an entry's
    gradient stands alone in dW."""
    p = Problem(S, d, V, K=30, softcap=4.0, short=0, empty=0, ignore=0, **o)
    rng = np.random.default_rng(7)
    p.H[:] = 0
    p.H[np.arange(64), np.arange(64)] = 1.0
    p.W[:30] = bf16(4.0 * rng.uniform(1.0, 13.0, (30, d)) * rng.choice([-1.0, 1.0], (30, d)))
    p.index[:64] = np.argsort(rng.random((64, 30)), axis=1)
    p.index[64:] = -1
    p.logits = np.float32(rng.standard_normal((S, 30))).astype(np.float64)
    p.labels = np.where(np.arange(S) < 64, rng.integers(0, 60, S), -100).astype(np.int32)
    if p.lse is not None:
        p.lse[:] = 5.0
    run = Run(p)
    run.forward()
    run.backward()
    print(check(p, run.outputs(), p.oracle()))
