"""Blocks in 8 bits on the GPU: every byte, every scale and every value that comes back as the plain form's."""
import numpy as np
import pytest
import torch

from paper_2104_11805_amd import sdnn
from tests import blocks

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def check(x, cap, shift=0):
    n, b = x.shape
    codes, scales, value = blocks.pack8(x, cap)
    whole = torch.full((n * b + 8,), 777.0, device=DEV)
    xd = whole[shift:shift + n * b].view(n, b)
    xd.copy_(torch.from_numpy(x))
    room = torch.full((blocks.packed_bytes(n, b) + 512,), 99, dtype=torch.uint8, device=DEV)
    packed = sdnn.sdnn_pack8(xd, cap, packed=room[256:-256])
    got = room.cpu().numpy()
    c, s = blocks.split_packed(got[256:], n, b)
    np.testing.assert_array_equal(c, codes)
    np.testing.assert_array_equal(s, scales)
    assert (got[:256] == 99).all() and (got[-256:] == 99).all()
    back = torch.full((n * b + 8,), 777.0, device=DEV)
    out = sdnn.sdnn_unpack8(packed, x=back[shift:shift + n * b].view(n, b))
    np.testing.assert_array_equal(out.cpu().numpy().astype(np.float64), value)
    assert bool((back[:shift] == 777).all()) and bool((back[shift + n * b:] == 777).all())


@pytest.mark.parametrize("cap", [0.0, 1.0, 32.0, 0.1, float("inf")])
@pytest.mark.parametrize("n,b", [(1, 1), (1, 127), (127, 1), (128, 1), (129, 1), (3, 43), (16, 8), (1000, 64), (777, 99), (2, 70001), (4096, 260)])
def test_bytes_scales_and_values(n, b, cap):
    rng = np.random.default_rng(n * b)
    x = (rng.normal(size=(n, b)) * np.exp(3 * rng.normal(size=(n, 1)))).astype(np.float32)
    if cap > 0:
        x = np.where(rng.random(x.shape) < 0.05, np.float32(min(cap, 1e30)), np.clip(x, 0, cap)).astype(np.float32)
    for shift in (0, 1):
        check(x, cap, shift)


@pytest.mark.parametrize("cap", [0.0, 1.0, 32.0, float("inf")])
def test_halves_and_values_next_to_them(cap):
    """Multiples and halves of a scale, and the fp32 values on both sides of each: the border of every rounding."""
    most = 253 if cap > 0 else 127
    for t in (2.0 ** -6, 129 * 2.0 ** -12, 255 * 2.0 ** -11, 171 * 2.0 ** -40, 2.0 ** -130):
        t = np.float32(t)
        if cap > 0 and most * float(t) >= cap:
            t = np.float32(t / 256)
        halves = (np.arange(0, 2 * most, dtype=np.float64) / 2 * float(t)).astype(np.float32)
        v = np.concatenate([halves, np.nextafter(halves, np.float32(1e30)), np.nextafter(halves, np.float32(0))])
        v = np.concatenate([v, -v]) if cap == 0 else v
        top = np.float32(most * float(t))
        rows = np.pad(v, (0, -v.size % 127)).reshape(-1, 127)
        check(np.concatenate([np.full((len(rows), 1), top, np.float32), rows], axis=1), cap)


@pytest.mark.parametrize("cap", [0.0, 1.0, 32.0, float("inf")])
def test_special_values(cap):
    rng = np.random.default_rng(4)
    x = rng.normal(size=(40, 128)).astype(np.float32)
    x[0] = 0
    x[1, 3] = np.nan
    x[2, :] = np.nan
    x[3, 5], x[3, 6] = np.inf, -np.inf
    x[4, :] = 0; x[4, 9] = 2.0 ** -149
    x[5, :] = np.float32(1e-44)
    x[6, 1], x[6, 2] = 3.4e38, -3.4e38
    x[7, :] = 32
    x[8, ::2] = np.nextafter(np.float32(32), np.float32(0))
    x[9, :] = -0.0
    x[10, 0] = 1e-20
    x[11, :] = 1
    x[12, ::3] = np.nextafter(np.float32(1), np.float32(0))
    check(x, cap)


def test_an_empty_block_and_another_stream():
    assert sdnn.sdnn_unpack8(sdnn.sdnn_pack8(torch.empty(0, 5, device=DEV))).shape == (0, 5)
    x = torch.randn(3000, 77, device=DEV)
    want = sdnn.sdnn_unpack8(sdnn.sdnn_pack8(x))
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = sdnn.sdnn_unpack8(sdnn.sdnn_pack8(x, stream=side), stream=side)
    torch.cuda.synchronize()
    assert torch.equal(got, want)


def test_a_block_past_32_bits_of_offset():
    n, b = 140001, 16384
    gen = torch.Generator(device=DEV)
    gen.manual_seed(6)
    x = torch.randn(n, b, generator=gen, device=DEV)
    packed = sdnn.sdnn_pack8(x)
    back = sdnn.sdnn_unpack8(packed)
    for r in (0, 65536, 131072, n - 1):  # rows of whole groups
        codes, scales, value = blocks.pack8(x[r:r + 1].cpu().numpy(), 0.0)
        at = r * b
        np.testing.assert_array_equal(packed.data[at:at + b].cpu().numpy(), codes)
        at = n * b + 2 * (r * b // 128)
        np.testing.assert_array_equal(packed.data[at:at + 2 * (b // 128)].cpu().numpy().view(np.uint16), scales)
        np.testing.assert_array_equal(back[r:r + 1].cpu().numpy().astype(np.float64), value)
    x.sub_(back).abs_()
    assert float(x.max()) <= 0.5 * 7.0 / 127 * 1.01  # half a scale of a group with a value of 7, which 2e9 normal ones do not pass by much
