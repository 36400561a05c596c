"""Arguments of the norm binding that ctypes would hand on as something else (CPU: what is accepted gets as far as the device's check)."""
import pytest

from tests.test_norm_library_abi import ARGUMENT, NO_DEVICE, mst  # noqa: F401


@pytest.mark.parametrize("gate_rows,status", [(64, NO_DEVICE), (1 << 40, NO_DEVICE), ((1 << 63) - 1, NO_DEVICE), (1 << 63, ARGUMENT),
                                              ((1 << 64) + 1, ARGUMENT), (-1, ARGUMENT)])
def test_rows_of_the_gate_beyond_64_bits(mst, gate_rows, status):  # noqa: F811
    """Of 2^64 + 1 the C call would see 1: a gate with a row for each token, read far behind the end of this one's single row."""
    import torch
    S, d = 64, 40
    x, h, codes = torch.zeros((S, d), dtype=torch.bfloat16), torch.zeros((S, d), dtype=torch.bfloat16), torch.zeros((S, d), dtype=torch.int8)
    exps, gate = torch.zeros((S, 2), dtype=torch.uint8), torch.zeros((1, d), dtype=torch.bfloat16)
    w, sums, ws = torch.zeros(d, dtype=torch.bfloat16), torch.zeros((1, d)), torch.zeros(1 << 16, dtype=torch.uint8)
    branch = dict(gate=gate, gate_rows=gate_rows, normalize=False)
    for call in (lambda: mst.mst_residual_fwd(h, x, x, **branch),
                 lambda: mst.mst_residual_bwd(x, h, ws, dgate=sums, codes=codes, exps=exps, **branch),
                 lambda: mst.mst_residual_prenorm_fwd(h, x, x, h, w, **branch),
                 lambda: mst.mst_residual_prenorm_bwd(h, x, x, h, ws, w, sums[0], dgate=sums, codes_y=codes, exps_y=exps, codes_o=codes, exps_o=exps, **branch)):
        with pytest.raises(mst.MstError) as e:
            call()
        assert e.value.status == status
