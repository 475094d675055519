"""Layer norm forward and backward on the GPU against the plain form in 64 bits.

Bounds: sums are taken in 64 bits and a result is rounded to fp32 once, which moves it by at most 2^-24 of itself; what 64 bits
lose is below 1e-12 of the terms that a result is made of (2^-53 times some hundred roundings; a variance whose shift, the sample's
first value, lies k standard deviations off loses k^2 2^-53)."""
import numpy as np
import pytest
import torch

from paper_2104_11805_amd import sdnn
from tests import blocks
from tests.blocks import HALF, TINY, close

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
SIZES = [(1, 1), (1, 300), (2, 1), (5, 3), (64, 4), (33, 64), (127, 2), (257, 63), (1024, 64), (1000, 1), (100000, 1), (129, 65), (1025, 99), (4097, 128),
         (300, 1030), (40, 4100), (20000, 36), (9, 2048), (3001, 777), (65536, 16)]


def dev(a):
    return None if a is None else torch.from_numpy(np.ascontiguousarray(a)).to(DEV)


def case(n, b, seed, affine=True, offset=0.0):
    rng = np.random.default_rng(seed)
    x = (rng.normal(size=(n, b)) * (1 + rng.random((1, b))) + offset * (1 + rng.random((1, b)))).astype(np.float32)
    gamma, beta = (rng.normal(size=n).astype(np.float32), rng.normal(size=n).astype(np.float32)) if affine else (None, None)
    return x, gamma, beta, rng.normal(size=(n, b)).astype(np.float32)


def check_forward(y, stats, x, gamma, beta, eps):
    want, (mean, rstd) = blocks.norm(x, gamma, beta, eps)
    g = np.ones(len(x)) if gamma is None else np.abs(gamma.astype(np.float64))
    x0 = x[0].astype(np.float64)
    size = (np.abs(x) + np.abs(mean)) * rstd * g[:, None] + np.abs(want)
    lost = 1e-12 * (1 + ((x0 - mean) * rstd) ** 2)
    close(y.cpu().numpy(), want, HALF * np.abs(want) + lost * size + TINY, "y")
    close(stats[0].cpu().numpy(), mean, 1e-13 * (np.abs(x0) + np.abs(x - x0).max(axis=0)), "mean")
    close(stats[1].cpu().numpy(), rstd, lost * rstd, "rstd")


def check_backward(got, dy, x, stats, gamma):
    want = blocks.norm_backward(dy, x, stats, gamma)
    dy, x = dy.astype(np.float64), np.asarray(x, np.float64)
    g = np.ones(len(x)) if gamma is None else gamma.astype(np.float64)
    mean, rstd = stats
    h, d = (np.abs(x) + np.abs(mean)) * rstd, np.abs(g[:, None] * dy)
    close(got[0].cpu().numpy(), want[0], HALF * np.abs(want[0]) + 1e-12 * rstd * (d + d.mean(0) + h * (d * h).mean(0)) + TINY, "dx")
    close(got[1].cpu().numpy(), want[1], HALF * np.abs(want[1]) + 1e-12 * (np.abs(dy) * h).sum(1) + TINY, "dgamma")
    close(got[2].cpu().numpy(), want[2], HALF * np.abs(want[2]) + 1e-12 * np.abs(dy).sum(1) + TINY, "dbeta")


@pytest.mark.parametrize("n,b", SIZES)
def test_forward_and_backward(n, b):
    for affine, eps in ((True, 1e-5), (False, 0.1)):
        x, gamma, beta, dy = case(n, b, 100 * n + b, affine)
        y, stats = sdnn.sdnn_layernorm(dev(x), dev(gamma), dev(beta), eps=eps)
        check_forward(y, stats, x, gamma, beta, eps)
        got = sdnn.sdnn_layernorm_backward(dev(dy), dev(x), stats, dev(gamma))
        check_backward(got, dy, x, stats.cpu().numpy(), gamma)


@pytest.mark.parametrize("cap", [0.0, 2.0, float("inf")])
@pytest.mark.parametrize("n,b", SIZES)
def test_backward_from_8_bits(n, b, cap):
    x, gamma, _, dy = case(n, b, 7 * n + b)
    stats = blocks.norm(x, None, None, 1e-5)[1]
    packed = sdnn.sdnn_pack8(dev(x), cap)
    kept = blocks.pack8(x, cap)[2]
    got = sdnn.sdnn_layernorm_backward(dev(dy), packed, dev(stats), dev(gamma))
    check_backward(got, dy, kept, stats, gamma)


@pytest.mark.parametrize("n,b", [(500, 7), (1024, 64), (3000, 130), (66000, 8)])
def test_a_large_mean_and_samples_without_variance(n, b):
    """Values whose spread is a few steps of fp32 around their mean; one sample of one value (y = beta, rstd = 1/sqrt(eps)); one whose
    first value lies far off; a smallest and a largest one."""
    x, gamma, beta, dy = case(n, b, 3, offset=3e5)
    x[:, 1] = 7.25
    x[:, 2] *= np.float32(1e-30)
    x[:, 3] *= np.float32(1e31)
    x[0, 4] += np.float32(1e7)
    y, stats = sdnn.sdnn_layernorm(dev(x), dev(gamma), dev(beta))
    check_forward(y, stats, x, gamma, beta, 1e-5)
    assert np.array_equal(y[:, 1].cpu().numpy(), beta)
    check_backward(sdnn.sdnn_layernorm_backward(dev(dy), dev(x), stats, dev(gamma)), dy, x, stats.cpu().numpy(), gamma)


@pytest.mark.parametrize("eps", [1e-5, 1e-20])
@pytest.mark.parametrize("n,b", [(1, 5), (500, 7), (1024, 64), (3000, 130), (66000, 130)])
def test_samples_without_variance_whatever_their_size(n, b, eps):
    """Every sample is one value n times: h is 0, however large 1/sqrt(eps) is, so that Y is beta, dgamma 0, and dX of a single row 0."""
    x, gamma, beta, dy = case(n, b, 4)
    x[:] = (10.0 ** np.linspace(-6, 9, b)).astype(np.float32)
    y, stats = sdnn.sdnn_layernorm(dev(x), dev(gamma), dev(beta), eps=eps)
    assert np.array_equal(y.cpu().numpy(), np.broadcast_to(beta[:, None], y.shape))
    dx, dgamma, dbeta = sdnn.sdnn_layernorm_backward(dev(dy), dev(x), stats, dev(gamma))
    assert bool((dgamma == 0).all())
    d = gamma.astype(np.float64)[:, None] * dy
    want = (d - d.mean(0)) / np.sqrt(eps)
    close(dx.cpu().numpy(), want, HALF * np.abs(want) + 1e-12 * (np.abs(d) + np.abs(d).mean(0)) / np.sqrt(eps) * (n > 1) + TINY, "dx")


@pytest.mark.parametrize("n,b", [(5, 3), (1024, 64), (700, 129), (70000, 12), (64, 2050)])
@pytest.mark.parametrize("bad", [np.nan, np.inf, -np.inf])
def test_nonfinite_samples_stay_by_themselves(n, b, bad):
    x, gamma, beta, dy = case(n, b, 5)
    ok = np.ones(b, bool)
    for s, i in ((0, 0), (b // 2, n - 1)):
        x[i, s], ok[s] = bad, False
    y, stats = sdnn.sdnn_layernorm(dev(x), dev(gamma), dev(beta))
    assert bool(y[:, ~ok].isnan().all()) and bool(stats[1, ~ok].isnan().all())
    check_forward(y[:, ok], stats[:, ok], x[:, ok], gamma, beta, 1e-5)
    dx, dgamma, dbeta = sdnn.sdnn_layernorm_backward(dev(dy), dev(x), stats, dev(gamma))
    assert bool(dx[:, ~ok].isnan().all()) and bool(dgamma.isnan().all()) and bool(dbeta.isfinite().all())
    want = blocks.norm_backward(dy[:, ok], x[:, ok], stats[:, ok].cpu().numpy(), gamma)[0]
    np.testing.assert_allclose(dx[:, ok].cpu().numpy(), want, rtol=2 * HALF, atol=1e-9)  # values of size 1


@pytest.mark.parametrize("n,b", [(33, 64), (200, 4), (1025, 99), (5000, 512)])
def test_in_place_unaligned_and_nothing_beside(n, b):
    """Results over their inputs, blocks at addresses that are multiples of 4 bytes only, guards around every result: the same bits."""
    x, gamma, beta, dy = (dev(t) for t in case(n, b, 11))
    y, stats = sdnn.sdnn_layernorm(x, gamma, beta)
    dx, dgamma, dbeta = sdnn.sdnn_layernorm_backward(dy, x, stats, gamma)
    packed = sdnn.sdnn_pack8(x)
    from_8 = sdnn.sdnn_layernorm_backward(dy, packed, stats, gamma)

    def guarded(shape, dtype=torch.float32, shift=1):
        whole = torch.full((int(np.prod(shape)) + 8,), 777.0, dtype=dtype, device=DEV)
        return whole, whole[shift:shift + int(np.prod(shape))].view(shape)

    def untouched(whole, inner):
        at = (inner.data_ptr() - whole.data_ptr()) // whole.element_size()
        assert bool((whole[:at] == 777).all()) and bool((whole[at + inner.numel():] == 777).all())

    for shift in (1, 4):
        wy, y2 = guarded((n, b), shift=shift)
        ws, s2 = guarded((2, b), torch.float64, shift)
        y2.copy_(x)
        assert sdnn.sdnn_layernorm(y2, gamma, beta, y=y2, stats=s2)[0] is y2
        wd, d2 = guarded((n, b), shift=shift)
        wg, g2 = guarded((n,), shift=shift)
        wb, b2 = guarded((n,), shift=shift)
        _, x2 = guarded((n, b), shift=shift)
        x2.copy_(x)
        _, gamma2 = guarded((n,), shift=shift)
        gamma2.copy_(gamma)
        for source, want in ((x2, (dx, dgamma, dbeta)), (packed, from_8)):
            d2.copy_(dy)
            sdnn.sdnn_layernorm_backward(d2, source, s2, gamma2, dx=d2, dgamma=g2, dbeta=b2)
            for got, ref in zip((d2, g2, b2), want):  # another way through the sums may be taken: the last bit of 64
                torch.testing.assert_close(got, ref, rtol=2 * HALF, atol=1e-9)
            for whole, inner in ((wd, d2), (wg, g2), (wb, b2)):
                untouched(whole, inner)
        torch.testing.assert_close(y2, y, rtol=2 * HALF, atol=1e-9)
        untouched(wy, y2)
        untouched(ws, s2)
    x3 = x.clone()
    sdnn.sdnn_layernorm_backward(dy, x3, stats, gamma, dx=x3)
    assert torch.equal(x3, dx)


def test_results_that_are_not_wanted_and_a_workspace_that_was_used():
    n, b = 900, 72
    x, gamma, beta, dy = (dev(t) for t in case(n, b, 12))
    work = torch.full((sdnn.sdnn_layernorm_workspace_bytes(n, b),), 255, dtype=torch.uint8, device=DEV)  # NaN wherever it is read unwritten
    y, stats = sdnn.sdnn_layernorm(x, gamma, beta, work=work)
    ref = sdnn.sdnn_layernorm(x, gamma, beta)
    assert torch.equal(y, ref[0]) and torch.equal(stats, ref[1])
    full = sdnn.sdnn_layernorm_backward(dy, x, stats, gamma, work=work.fill_(255))
    ptr = lambda t: None if t is None else t.data_ptr()
    for wanted in ((1, 0, 0), (0, 1, 0), (0, 0, 1), (1, 1, 0), (0, 1, 1)):
        outs = [torch.full_like(t, 5.0) if w else None for t, w in zip(full, wanted)]
        work.fill_(255)
        rc = sdnn.lib().sdnn_layernorm_backward(ptr(dy), ptr(x), ptr(stats), ptr(gamma), n, b, *[ptr(t) for t in outs], ptr(work), work.numel(),
                                                torch.cuda.current_stream().cuda_stream)
        assert rc == 0
        assert all(o is None or torch.equal(o, t) for o, t in zip(outs, full))


def test_the_same_bits_each_time_and_on_another_stream():
    n, b = 5003, 60
    x, gamma, beta, dy = (dev(t) for t in case(n, b, 13))
    first = sdnn.sdnn_layernorm(x, gamma, beta)
    first += sdnn.sdnn_layernorm_backward(dy, x, first[1], gamma)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for stream in (None, side, side):
        again = sdnn.sdnn_layernorm(x, gamma, beta, stream=stream)
        again += sdnn.sdnn_layernorm_backward(dy, x, again[1], gamma, stream=stream)
        torch.cuda.synchronize()
        assert all(torch.equal(u, v) for u, v in zip(first, again))


@pytest.mark.parametrize("n,b", [(1024, 64), (6000, 33), (40000, 64)])
def test_captured_and_replayed(n, b):
    x, gamma, beta, dy = (dev(t) for t in case(n, b, 14))
    y, stats, work = torch.empty_like(x), torch.empty(2, b, dtype=torch.float64, device=DEV), torch.empty(
        sdnn.sdnn_layernorm_workspace_bytes(n, b), dtype=torch.uint8, device=DEV)
    packed = torch.empty(sdnn.sdnn_pack8_bytes(n, b), dtype=torch.uint8, device=DEV)
    out = [torch.empty_like(x), torch.empty(n, device=DEV), torch.empty(n, device=DEV)]

    def step():
        sdnn.sdnn_layernorm(x, gamma, beta, y=y, stats=stats, work=work)
        p = sdnn.sdnn_pack8(x, packed=packed)
        sdnn.sdnn_layernorm_backward(dy, p, stats, gamma, *out, work=work)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for k in range(4):
        x.mul_(0.9).add_(0.01 * k)
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (y, stats, *out)]
        step()
        torch.cuda.synchronize()
        assert all(torch.equal(u, v) for u, v in zip(got, (y, stats, *out)))


def test_a_block_past_32_bits_of_offset():
    """More than 2^31 values, 9 GB: the rows behind that offset, and sums that run over all of them."""
    n, b = 140000, 16384
    gen = torch.Generator(device=DEV)
    gen.manual_seed(5)
    x = torch.randn(n, b, generator=gen, device=DEV)
    x[-1, 5] = 1000.0
    gamma, beta = torch.randn(n, generator=gen, device=DEV), torch.randn(n, generator=gen, device=DEV)
    y, stats = sdnn.sdnn_layernorm(x, gamma, beta)
    cols = torch.tensor([0, 5, 8191, 16383], device=DEV)
    xs = x[:, cols].double()
    mean = xs.mean(0)
    rstd = (xs.var(0, unbiased=False) + 1e-5).rsqrt()
    want = (xs - mean) * rstd * gamma.double()[:, None] + beta.double()[:, None]
    torch.testing.assert_close(y[:, cols].double(), want, rtol=2 * HALF, atol=1e-9)
    packed = sdnn.sdnn_pack8(x)
    rows = torch.tensor([0, 70000, n - 1], device=DEV)
    kept = np.concatenate([blocks.pack8(x[r:r + 1].cpu().numpy(), 0.0)[2] for r in rows.tolist()])  # rows of whole groups
    dx, dgamma, dbeta = sdnn.sdnn_layernorm_backward(y, packed, stats, gamma, dx=y)
    h = (torch.from_numpy(kept).to(DEV) - stats[0]) * stats[1]
    again = sdnn.sdnn_layernorm(x, gamma, beta)[0][rows].double()
    torch.testing.assert_close(dgamma[rows].double(), (again * h).sum(1), rtol=2 * HALF, atol=1e-7)  # 16384 terms of size 1 in 64 bits
    torch.testing.assert_close(dbeta[rows].double(), again.sum(1), rtol=2 * HALF, atol=1e-7)
    assert bool(dx[:, cols].isfinite().all())
