"""Sums of the root-mean-square norm's backward pass over very many rows and very long rows: their error does not grow with the length.  Values that repeat are what a running
sum in 32 bits is worst at: every addition then errs to the same side."""
import numpy as np
import pytest

import step8_ref as R
from test_gpu_layers import column_vector, env, rng_of  # noqa: F401  (env: the fixture)

pytestmark = pytest.mark.gpu
U, U16 = R.U32, R.U16


@pytest.mark.parametrize("cols", [8193, 100003, 3000001])
@pytest.mark.parametrize("bf16", [False, True])
def test_mean_along_a_long_row(env, cols, bf16):  # noqa: F811
    """dz of rows whose two terms nearly cancel, so that the mean's own error is what is left."""
    torch, B = env
    z = np.ones((2, cols), np.float32)
    z[1] = 1.0 + 0.25 * rng_of(cols).random(cols)
    z = R.rounded(z, bf16)
    dy = R.rounded(z * np.float32(1.5), bf16)
    gamma, rstd = np.ones(cols, np.float32), np.float32(R.rms(z, np.ones(cols), 1e-5)[1])
    dt = torch.bfloat16 if bf16 else torch.float32
    D, Z = column_vector(torch, dy).to(dt), column_vector(torch, z).to(dt)
    dz = torch.empty_like(Z)
    B.conef_rms_backward(D, Z, column_vector(torch, gamma), column_vector(torch, rstd), None, dz, None, None, B.Model.stream_handle())
    want, _, hat, a = R.rms_back(dy, z, gamma, rstd)
    # roundings of hat and of a in the sum's terms, of their product, of the mean; of the row's own hat, its product with the mean, the difference, and the product with rstd
    s = rstd.astype(np.float64)[:, None]
    err = s * (2 * U * np.abs(a) + 7 * U * np.abs(hat) * np.abs(a * hat).mean(1, keepdims=True)) + 2 * U * np.abs(want)
    err = err * 1.01 + (np.abs(want) * U16 * 1.01 if bf16 else 0)
    assert (np.abs(dz.float().cpu().numpy() - want) <= err).all()


MOST_ROWS = 128               # that a lane adds in 32 bits; then a few across a wave and a workgroup


@pytest.mark.parametrize("rows,cols", [(20_000_000, 5), (5_000_000, 100), (2_000_000, 300), (1_000_000, 700), (300_000, 1500), (300_000, 2304), (150_000, 4500), (100_000, 7000),
                                       (200_000, 8200)])
def test_sums_over_very_many_rows(env, rows, cols):  # noqa: F811
    torch, B = env
    g = torch.Generator(device="cuda:0").manual_seed(cols)
    row = (torch.rand(cols, device="cuda:0", generator=g) + 1.0).bfloat16()
    z = row[None, :].repeat(rows, 1)
    dy = torch.full_like(z, 1.7)
    rstd, gamma = torch.full((rows,), 0.7, device="cuda:0"), torch.ones(cols, device="cuda:0")
    dgamma = torch.empty(cols, device="cuda:0")
    ws = torch.full((B.conef_rms_workspace(rows, cols),), 0xFF, dtype=torch.uint8, device="cuda:0")
    B.conef_rms_backward(dy, z, gamma, rstd, None, None, dgamma, ws, B.Model.stream_handle())
    want = rows * dy[0].double() * (row.double() * rstd[0].double())
    # hat's rounding, the lane's sums, six across a wave and four across a workgroup, the result's
    assert bool(((dgamma.double() - want).abs() <= (MOST_ROWS + 12) * U * 1.01 * want).all())
