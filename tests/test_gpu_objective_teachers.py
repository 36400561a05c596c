"""Teachers' logits that are NaN, on the GPU: reported by the row's divergence and by the loss, whatever else the row holds."""
import numpy as np
import pytest

from tests.objective_gpu_harness import Problem, Run

pytestmark = pytest.mark.gpu

SIZES = [(20, 64, 300), (130, 72, 9000), (200, 72, 12800), (400, 72, 12800), (1500, 64, 12800)]      # tiles of 64 x 32, of 256 x 32, 64, 128 and 256


@pytest.mark.parametrize("S,d,V", SIZES)
@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("rest", [None, -np.inf, np.finfo(np.float32).min, 1.0], ids=["all NaN", "masks of -inf", "masks of the lowest value", "finite"])
def test_a_teacher_of_nan_is_not_a_missing_one(S, d, V, tail, rest):
    p = Problem(S, d, V, K=30, tail=tail, label_coef=0.5, empty=0, short=0)
    good = p.oracle()
    p.logits[3] = np.nan if rest is None else rest
    p.logits[3, 7] = np.nan
    run = Run(p)
    run.forward()
    run.backward()
    got = run.outputs()
    assert got["n"] == good["n"] and np.isnan(got["loss"]) and np.isnan(got["rows"][3])
    others = np.arange(S) != 3
    np.testing.assert_allclose(got["rows"][others], good["kd"][others], rtol=1e-4, atol=1e-5)
    np.testing.assert_allclose(got["nll"], good["nll"], rtol=1e-4, atol=1e-5)
    assert np.isnan(got["dH"][3]).any() and np.isnan(got["dW"]).any() and np.isfinite(got["dH"][others]).all()


@pytest.mark.parametrize("S,d,V", SIZES)
def test_a_row_of_weight_zero_may_have_one(S, d, V):
    p = Problem(S, d, V, K=30, label_coef=0.5, weights=True, empty=0)
    p.weights[3] = 0.0
    good = p.oracle()
    p.logits[3] = np.nan
    run = Run(p)
    run.forward()
    run.backward()
    got = run.outputs()
    assert got["n"] == good["n"] and np.isnan(got["rows"][3]) and abs(got["loss"] - good["loss"]) <= 1e-4 * abs(good["loss"])
    assert not got["dH"][3].any() and np.isfinite(got["dW"]).all()
