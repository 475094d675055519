"""Layer norm at the sizes where another kernel, split or width of tile is taken, against the plain form in 64 bits on the GPU.

Bounds as in test_gpu_layernorm: a result is rounded once (2^-24 of itself); what 64 bits lose, here and in the plain form, is below 1e-12 of
the terms that a result is made of."""
import pytest
import torch

from paper_2104_11805_amd import sdnn
from tests.blocks import HALF

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
# one launch and two: rows 1024 | 1025 and 2048 | 2049, columns 3 | 4 and 4095 | 4096, 2^24 values, 200 MB
BORDERS = [(1024, 3), (1024, 4), (1024, 5), (1023, 17), (1025, 4), (1025, 19), (2048, 9), (2049, 9), (1024, 4095), (1000, 4096), (1024, 4099), (1, 4097), (2, 8191),
           (127, 8192), (127, 8193), (128, 8193), (2048, 8192), (2047, 8203), (2047, 8193), (1000, 20001), (960, 52430)]
# the ranges' sums by a launch of their own, with a last tile that is not whole, tiles of each width, and their neighbours without that launch
SPLITS = [(70001, 61), (140003, 30), (65536, 64), (65535, 64), (32771, 129), (8192, 1030), (8111, 1037), (2100, 4099), (2500, 4095), (2049, 4096), (524289, 16), (300001, 3), (57344, 128), (57343, 128),
          (24001, 306), (2100, 2101), (4001, 161), (4001, 160), (2047, 500), (200000, 40),
          (1 << 20, 2), (5000001, 1), (40001, 7)]
FAR = [(2101, 24001), (50331648, 1), (786433, 64)]  # 200 MB and more
BEHIND = 1 << 16


def random(shape, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    return torch.randn(shape, generator=gen, device=DEV)


def close(got, want, bound, what):
    off = ((got.double() - want).abs() - bound).max().item()
    assert off <= 0.0, (what, off)


def check(n, b, packed=False, affine=True):
    x, dy = random((n, b), n + 3 * b) * 2 + 0.5, random((n, b), n + 3 * b + 1)
    gamma, beta = (random((n,), n), random((n,), b)) if affine else (None, None)
    nbytes = sdnn.sdnn_layernorm_workspace_bytes(n, b)
    work = torch.full((nbytes + BEHIND,), 255, dtype=torch.uint8, device=DEV)  # NaN wherever it is read unwritten
    y, stats = sdnn.sdnn_layernorm(x, gamma, beta, work=work[:nbytes])
    xd = x.double()
    mean, g = xd.mean(0), torch.ones(n, 1, dtype=torch.float64, device=DEV) if gamma is None else gamma.double()[:, None]
    rstd = ((xd - mean).square().mean(0) + 1e-5).rsqrt()
    want = (xd - mean) * rstd * g
    size = (xd.abs() + mean.abs()) * rstd * g.abs()
    if beta is not None:
        want += beta.double()[:, None]
    close(y, want, HALF * want.abs() + 1e-12 * (size + want.abs()), "y")
    close(stats[0], mean, 1e-12 * xd.abs().amax(0), "mean")
    close(stats[1], rstd, 1e-12 * rstd, "rstd")
    del y, want, size
    source = x
    if packed:
        source = sdnn.sdnn_pack8(x)
        xd = sdnn.sdnn_unpack8(source).double()
    work[:nbytes].fill_(255)
    dx, dgamma, dbeta = sdnn.sdnn_layernorm_backward(dy, source, stats, gamma, work=work[:nbytes])
    assert bool((work[nbytes:] == 255).all())
    mean, rstd = stats
    h, d = (xd - mean) * rstd, g * dy.double()
    most = (xd.abs() + mean.abs()) * rstd
    close(dgamma, (dy.double() * h).sum(1), HALF * (dy.double() * h).sum(1).abs() + 1e-12 * (dy.double().abs() * most).sum(1), "dgamma")
    close(dbeta, dy.double().sum(1), HALF * dy.double().sum(1).abs() + 1e-12 * dy.double().abs().sum(1), "dbeta")
    want = rstd * (d - d.mean(0) - h * (d * h).mean(0))
    bound = rstd * (d.abs() + d.abs().mean(0) + most * (d.abs() * most).mean(0))
    close(dx, want, HALF * want.abs() + 1e-12 * bound, "dx")


@pytest.mark.parametrize("n,b", BORDERS + SPLITS)
def test_where_the_way_changes(n, b):
    check(n, b)


@pytest.mark.parametrize("n,b", SPLITS + [(1025, 19), (1024, 4099)])
def test_where_the_way_changes_from_8_bits(n, b):
    check(n, b, packed=True, affine=b % 2 == 0)


@pytest.mark.parametrize("n,b", FAR)
def test_blocks_that_the_caches_do_not_hold(n, b):
    check(n, b, affine=b > 1)


@pytest.mark.parametrize("n,b", [(1024, 64), (2100, 4099), (70001, 61)])
def test_in_place_where_the_way_changes(n, b):
    x, dy, gamma, beta = random((n, b), 1), random((n, b), 2), random((n,), 3), random((n,), 4)
    y, stats = sdnn.sdnn_layernorm(x, gamma, beta)
    over = x.clone()
    sdnn.sdnn_layernorm(over, gamma, beta, y=over)
    assert torch.equal(over, y)
    dx = sdnn.sdnn_layernorm_backward(dy, x, stats, gamma)[0]
    for source in (dy.clone(), x.clone()):
        first = (source, x) if torch.equal(source, dy) else (dy, source)
        sdnn.sdnn_layernorm_backward(*first, stats, gamma, dx=source)
        assert torch.equal(source, dx)


def test_two_at_once_with_workspaces_of_their_own():
    """Calls on two streams, neither waiting for the other: each has the bits that it has alone."""
    sizes = [(65536, 64), (8192, 1030)]
    streams = [torch.cuda.Stream() for _ in sizes]
    data = [(random((n, b), 5), random((n, b), 6), random((n,), 7), random((n,), 8)) for n, b in sizes]
    works = [torch.empty(sdnn.sdnn_layernorm_workspace_bytes(n, b), dtype=torch.uint8, device=DEV) for n, b in sizes]
    alone = []
    for x, dy, gamma, beta in data:
        y, stats = sdnn.sdnn_layernorm(x, gamma, beta)
        alone.append((y, stats, *sdnn.sdnn_layernorm_backward(dy, sdnn.sdnn_pack8(x), stats, gamma)))
    outs = [[[torch.empty_like(t) for t in one] for one in alone] for _ in range(4)]
    kept = [sdnn.sdnn_pack8(x) for x, *_ in data]
    torch.cuda.synchronize()
    for turn in outs:
        for (x, dy, gamma, beta), (y, stats, dx, dgamma, dbeta), stream, work, packed in zip(data, turn, streams, works, kept):
            sdnn.sdnn_layernorm(x, gamma, beta, y=y, stats=stats, work=work, stream=stream)
            sdnn.sdnn_pack8(x, packed=packed.data, stream=stream)
            sdnn.sdnn_layernorm_backward(dy, packed, stats, gamma, dx=dx, dgamma=dgamma, dbeta=dbeta, work=work, stream=stream)
    torch.cuda.synchronize()
    for turn in outs:
        for one, ref in zip(turn, alone):
            assert all(torch.equal(u, v) for u, v in zip(one, ref))
