"""Coefficients of the LM head's objectives on the GPU: the gradient of the logits is rounded to bfloat16, a factor that all of its rows share is
not, so that no coefficient makes all of a gradient a little larger or smaller; divisors of any size."""
import numpy as np
import pytest

from tests.objective_gpu_harness import Problem, Run, bf16
from tests.objective_tight_bounds import check

pytestmark = pytest.mark.gpu

SIZES = [(64, 64, 1000), (400, 64, 12800), (1500, 64, 12800)]
BETWEEN = 1 + 2.0 ** -8          # half way between two bfloat16 numbers: 2^-8 of it is lost where it is rounded


def unit_vectors(S, d, V, **o):
    """Row s < 64 is the s-th unit vector, so that its gradient stands alone in column s of dW; the other rows have no loss.  Shares of 1e-4 to
    1e-2."""
    p = Problem(S, d, V, short=0, empty=0, ignore=0, **o)
    rng = np.random.default_rng(3)
    p.H[:] = 0
    p.H[np.arange(64), np.arange(64)] = 1.0
    p.W[:] = bf16(rng.standard_normal((V, d)) * 0.5)
    if p.labels is not None:
        p.labels[:] = np.where(np.arange(S) < 64, rng.integers(0, V, S), -100)
    if p.K:
        p.index[:] = np.where(np.arange(S)[:, None] < 64, rng.integers(0, V, (S, p.K)), -1)
    return p


def gradient_of(p, at, grad_loss=1.0):
    """What the 64 rows' gradients are at one vocabulary entry each, in units of the loss's gradient by that row."""
    r = Run(p)
    r.forward()
    r.backward(grad_loss)
    got, ref = r.outputs(), p.oracle(grad_loss)
    rows = np.arange(64)
    return got["dW"][at, rows] / ref["gamma"], ref["G"][rows, at]


@pytest.mark.parametrize("S,d,V", SIZES)
@pytest.mark.parametrize("coef", [0.25 * BETWEEN, -BETWEEN, 0.3, 1.0, 1e-30 * BETWEEN, 1e30 * BETWEEN])
@pytest.mark.parametrize("kind", ["labels beside a teacher", "teacher alone"])
def test_a_coefficient_is_not_rounded(S, d, V, coef, kind):
    """At a row's label, or at the only entry of its teacher, the gradient is the coefficient times 1 - p.  Rounded by itself this is off by half
    a step of the numbers from 1/2 to 1, 2^-9, less than 2^-8 with the coefficient; 16 half steps of float32 are more than the rest takes."""
    coef = float(np.float32(coef))
    if kind == "teacher alone":
        p = unit_vectors(S, d, V, K=1, labels=False, teacher_coef=coef)
        at = p.index[:64, 0]
    else:
        p = unit_vectors(S, d, V, K=1, label_coef=coef, teacher_coef=0.0)
        at = p.labels[:64]
    got, ref = gradient_of(p, at)
    assert np.abs(ref / coef).min() > 0.5
    off = np.abs(got / coef - ref / coef)
    print(off.max() * 512)
    assert (off <= 2.0 ** -9 + 16 * 2.0 ** -24).all()


@pytest.mark.parametrize("S,d,V", SIZES)
@pytest.mark.parametrize("alpha,beta,T", [(0.3, 0.7, 4.0), (0.0, 0.7, 2.0), (0.7, 0.0, 1.0), (-0.3, 0.9, 0.5), (0.0, 0.0, 1.0), (1e-6, 1.0, 1.0), (300.0, 1e-3, 1.0)])
def test_shares_of_labels_and_teacher(S, d, V, alpha, beta, T):
    p = Problem(S, d, V, K=20, tail=True, label_coef=alpha, teacher_coef=beta, temperature=T, weights=True)
    r = Run(p)
    r.forward()
    r.backward()
    got, ref = r.outputs(), p.oracle()
    print(check(p, got, ref))
    if alpha == beta == 0.0:
        assert not got["dH"].any() and not got["dW"].any()


@pytest.mark.parametrize("o", [dict(K=20, tail=True, label_coef=0.3, teacher_coef=0.7), dict(z_coef=1e-3)], ids=["distill", "wce"])
def test_divisors_of_any_size(o):
    """2^40, 2^52 and 2^62 in place of 1, with a gradient of the loss that is larger by as much: the same bits."""
    got = {}
    for e in (0, 40, 52, 62):
        p = Problem(200, 64, 1000, divisor=2 ** e, **o)
        r = Run(p)
        r.forward()
        r.backward(grad_loss=2.0 ** e)
        got[e] = r.outputs()
        assert got[e]["loss"] == got[0]["loss"] * 2.0 ** -e
        assert (got[e]["dH"] == got[0]["dH"]).all() and (got[e]["dW"] == got[0]["dW"]).all()
