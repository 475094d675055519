"""Layer norm on blocks whose rows or whose values lie far apart, on the GPU against the plain form in 64 bits, columns by columns.

Bounds as in test_gpu_layernorm_paths: a result is rounded once (2^-24 of itself), 64 bits lose less than 1e-12 of the terms that it is
made of.  Sums along rows of B values: 2^-53 of the terms' absolute values for every rounding on a value's way, which are B / 1024 (the tiles' sums, four at a
time) and some hundred."""
import pytest
import torch

from paper_2104_11805_amd import sdnn
from tests.blocks import HALF
from tests.test_gpu_layernorm_paths import DEV, close, random

pytestmark = pytest.mark.gpu
PIECE = 1 << 24  # columns that are compared at a time


@pytest.mark.parametrize("n,b", [(2, (1 << 29) + 2), (3, 600000001), (1, 1 << 30)])
def test_more_columns_than_two_rows_of_them_have_offsets_in_32_bits(n, b):
    """Rows of 2 GiB and more."""
    x, dy = random((n, b), n).mul_(2).add_(0.5), random((n, b), n + 1)
    gamma, beta = random((n,), 3), random((n,), 4)
    y, stats = sdnn.sdnn_layernorm(x, gamma, beta)
    dx, dgamma, dbeta = sdnn.sdnn_layernorm_backward(dy, x, stats, gamma)
    g = gamma.double()[:, None]
    sums = torch.zeros(4, n, dtype=torch.float64, device=DEV)
    for c in range(0, b, PIECE):
        part = slice(c, min(b, c + PIECE))
        xd, dyd = x[:, part].double(), dy[:, part].double()
        mean = xd.mean(0)
        rstd = ((xd - mean).square().mean(0) + 1e-5).rsqrt()
        close(stats[0, part], mean, 1e-12 * xd.abs().amax(0), ("mean", c))
        close(stats[1, part], rstd, 1e-12 * rstd, ("rstd", c))
        want = (xd - mean) * rstd * g + beta.double()[:, None]
        size = (xd.abs() + mean.abs()) * rstd * g.abs()
        close(y[:, part], want, HALF * want.abs() + 1e-12 * (size + want.abs()), ("y", c))
        mean, rstd = stats[:, part]
        h, d, most = (xd - mean) * rstd, g * dyd, (xd.abs() + mean.abs()) * rstd
        want = rstd * (d - d.mean(0) - h * (d * h).mean(0))
        bound = rstd * (d.abs() + d.abs().mean(0) + most * (d.abs() * most).mean(0))
        close(dx[:, part], want, HALF * want.abs() + 1e-12 * bound, ("dx", c))
        for k, v in enumerate((dyd * h, dyd.abs() * most, dyd, dyd.abs())):
            sums[k] += v.sum(1)
    lost = 2.0 ** -53 * (b / 1024 + 1000)
    close(dgamma, sums[0], HALF * sums[0].abs() + lost * sums[1], "dgamma")
    close(dbeta, sums[2], HALF * sums[2].abs() + lost * sums[3], "dbeta")


def test_dx_over_dy_from_8_bits_behind_32_bits_of_offset():
    """More than 2^31 values: dX written over dY and formed from the packed block, whole columns of it, at every row."""
    n, b = 140000, 16384
    x, y = random((n, b), 5), random((n, b), 6)
    gamma = random((n,), 7)
    cols = torch.tensor([0, 5, 255, 256, 8191, 16383], device=DEV)
    stats = sdnn.sdnn_layernorm(x, gamma)[1]
    packed = sdnn.sdnn_pack8(x)
    xd, dyd = sdnn.sdnn_unpack8(packed, x=x)[:, cols].double(), y[:, cols].double()  # (what the bytes stand for: test_gpu_pack8)
    dx, dgamma, dbeta = sdnn.sdnn_layernorm_backward(y, packed, stats, gamma, dx=y)
    mean, rstd = stats[:, cols]
    h, d, most = (xd - mean) * rstd, gamma.double()[:, None] * dyd, (xd.abs() + mean.abs()) * rstd
    want = rstd * (d - d.mean(0) - h * (d * h).mean(0))
    bound = rstd * (d.abs() + d.abs().mean(0) + most * (d.abs() * most).mean(0))
    close(dx[:, cols], want, HALF * want.abs() + 1e-12 * bound, "dx")
