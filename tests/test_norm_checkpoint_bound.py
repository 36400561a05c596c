"""How far a checkpoint's values may be from the tensor (CPU; the kernels' codes are the oracle's bit for bit, tests/test_gpu_norm_parity.py)."""
import numpy as np
import pytest

from oracle import norm_oracle as orc


@pytest.mark.parametrize("exponent", [-149, -140, -133, -128, -127, -126, -121, -120, -119, -100, 0, 60, 120])
def test_half_a_step(exponent):
    """Blocks whose largest magnitude is 1 to 2 times a power of two: off by 1 / 127.5 of it at most, by 2^-128 with E = 0."""
    rng = np.random.default_rng(exponent + 200)
    x = rng.uniform(-1, 1, (400, 32)) * 2.0 ** exponent
    x[:, 0] = 2.0 ** exponent * rng.uniform(1, 2, 400)
    x[:4, 0] = 2.0 ** exponent * np.array([1, 127 / 64, 127.5 / 64, 2 - 2.0 ** -7])
    codes, exps = orc.checkpoint(x)
    off, top = np.abs(orc.restore(codes, exps) - x).max(1), np.abs(x).max(1)
    least = exps[:, 0] == 0
    assert (off <= np.where(least, 2.0 ** -128, top / 127.5)).all()
    assert (least == (top < 127.5 * 2.0 ** -127)).all()
    if exponent < -129:          # less than half of the smallest scale: nothing is left, and the relative bound does not hold
        assert (codes == 0).all()
