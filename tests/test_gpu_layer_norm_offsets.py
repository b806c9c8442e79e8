"""Layer norm of constant rows: where fp32 holds the row's sums exactly, the mean is the constant, the variance 0 and y beta.

bf16 constants have 8 significant bits and rows at most 14 bits of length, so every partial sum is exact; fp32 constants
with at most 10 significant bits likewise.  sum / M is then the constant itself, and x - mean is 0."""
import pytest
import torch

import test_gpu_layer_norm as N

pytestmark = pytest.mark.gpu

# rows of a warp with 8, 16 and 32 values per lane, of a block, few rows and many
SIZES = [(3, 96), (5, 1000), (9, 1022), (40, 341), (2500, 96), (1300, 1000), (1201, 341), (1300, 513), (1300, 600), (1300, 1024), (6, 2050),
         (900, 2050), (700, 3000), (3, 9000), (640, 9000), (2, 16383), (700, 8200)]
VALUES = (1000.0, -1000.0, 12288.0, 1e6, 0.1, -77.5, 3e-3, 1e30, 0.0, 1e-30)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("n,M", SIZES)
def test_constant_rows_give_beta(n, M, dtype):
    t = N._make(n, M, dtype)
    c = torch.tensor(VALUES, device="cuda").bfloat16()[torch.arange(n, device="cuda") % len(VALUES)]
    t["x"] = c[:, None].expand(n, M).to(dtype).contiguous()
    y, mean, rstd = N._forward(t)
    assert torch.equal(mean, c.float())
    assert torch.equal(y, t["beta"].to(dtype).expand(n, M))
    # 1 / sqrt(eps): the rounding of eps, the root and the division
    assert torch.allclose(rstd, torch.full_like(rstd, N.EPS ** -0.5), rtol=4 * N.U32, atol=0)


def test_mean_of_rows_with_an_infinity_or_nan():
    """The mean of such a row is what its sum is; its neighbours keep theirs."""
    t = N._make(1300, 1000, torch.float32)
    _, mean0, _ = N._forward(t)
    t["x"][5, 3], t["x"][700, 999], t["x"][9, 0] = float("inf"), float("-inf"), float("nan")
    y, mean, _ = N._forward(t)
    assert mean[5] == float("inf") and mean[700] == float("-inf") and torch.isnan(mean[9])
    assert torch.isnan(y[[5, 700, 9]]).all()
    keep = torch.ones(1300, dtype=torch.bool, device="cuda")
    keep[[5, 9, 700]] = False
    assert torch.equal(mean[keep], mean0[keep])
