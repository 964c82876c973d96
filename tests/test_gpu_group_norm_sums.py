"""Sums of group norms whose maps a workgroup holds: a wavefront's are binary32, and what is added behind them is added in binary64.
The inputs' sums over a wavefront are exact; 2^24 of one of them and 1 of each other add up to what binary32 additions in a row lose."""
import pytest
import torch

import paper_2206_11357_amd as gact

pytestmark = pytest.mark.gpu

BIG = 2.0 ** 24


def spread(P, rows, per_wave, C, dtype, B=1):
    """2^24 in channel 0 of the first pixel, 1 in one pixel of each other wavefront; and how many of these there are."""
    x = torch.zeros(B, P, C, dtype=dtype, device="cuda")
    others = range(per_wave, min(rows, P), per_wave)
    for p in others:
        x[:, p, 0] = 1.0
    x[:, 0, 0] = BIG
    return x, len(others)


# one column of eight channels: thread t has the pixels t, t + threads, ..
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("P,threads", [(1000, 256), (4096, 512), (8192, 1024)])
def test_wavefronts(P, threads, dtype):
    x, others = spread(P, threads, 64, 8, dtype)
    assert others == threads // 64 - 1
    context = gact.make_group_norm_context(x, 1)
    gact.gact_group_norm(x, 1, context=context)
    want = torch.tensor((BIG + others) / (P * 8), dtype=torch.float64)
    # the product with 1 / (P 8) in binary64 and one rounding
    assert abs(float(context.mean) - want) <= 2.0 ** -24 * want * (1 + 2.0 ** -20)
    # a gradient with the same values: db is its sum, rounded once
    w = torch.ones(8, device="cuda")
    dx, dw, db = gact.gact_group_norm_backward(x, 1, w, w, context=context, x=torch.zeros_like(x))
    assert float(db[0]) == float(torch.tensor(BIG + others, dtype=torch.float64).float()) and (db[1:] == 0).all()


@pytest.mark.parametrize("bits,dtype", [(1, torch.bfloat16), (2, torch.float32), (8, torch.bfloat16), (8, torch.float32)])
def test_wavefronts_of_larger_maps(bits, dtype):
    """Maps whose gradient is held as it came, 512 threads: four columns of bf16, a wavefront has 16 rows of them; two of fp32, 32 rows."""
    B, P, C, H = 128, 3000, 64, 8
    rows, per_wave = (128, 16) if dtype == torch.bfloat16 else (256, 32)
    if dtype == torch.float32:
        P = 6000
    dy, others = spread(P, rows, per_wave, C, dtype, B)
    assert others == 7
    x = torch.randn(B, P, C, device="cuda").to(dtype)
    context = gact.make_group_norm_context(x, H, bits, 64, 1)
    gact.gact_group_norm(x, H, context=context)
    w = torch.ones(C, device="cuda")
    dx, dw, db = gact.gact_group_norm_backward(dy, H, w, w, context=context)
    want = B * (BIG + others)
    # a rounding of a sample's sum and one of theirs
    assert abs(float(db[0]) - want) <= 2 * 2.0 ** -24 * want


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("P,C,H", [(100, 24, 2), (300, 72, 2), (40, 56, 1)])
def test_channels_of_a_group(P, C, H, dtype):
    """Groups of 12, 36 and 56 channels, whose sums add up from channels' or columns'."""
    D = C // H
    x = torch.zeros(1, P, C, dtype=dtype, device="cuda")
    x[:, 0, :D] = 1.0
    x[:, 0, 0] = BIG
    if D % 8 == 0:
        x[:, 0, 1:8] = 0.0                              # (a lane adds its eight channels)
        x[:, 0, 8:16] = 0.0
    context = gact.make_group_norm_context(x, H)
    gact.gact_group_norm(x, H, context=context)
    if D % 8:
        want = (BIG + D - 1) / (P * D)
        assert abs(float(context.mean[0, 0]) - want) <= 2.0 ** -24 * want * (1 + 2.0 ** -20)
    # g n of a constant map is zero: dx = r (dy - mean dy), and mean dy holds the ones
    flat = gact.make_group_norm_context(torch.zeros_like(x), H)
    gact.gact_group_norm(torch.zeros_like(x), H, eps=1.0, context=flat)
    dx, _, _ = gact.gact_group_norm_backward(x, H, context=flat, x=torch.zeros_like(x))
    mean = x[0, :, :D].double().sum() / (P * D)
    off = 2.0 ** -24 if dtype == torch.float32 else 2.0 ** -8
    assert abs(float(dx[0, 1, 0]) + float(mean)) <= (2.0 ** -24 + off) * float(mean) * (1 + 2.0 ** -7)


@pytest.mark.parametrize("C,H", [(2048, 256), (1024, 256)])
def test_inverse_deviations_are_rounded_once(C, H):
    """Groups of values a and -a, a of eight bits: the mean is 0 and the variance a a, both exactly."""
    D = C // H
    a = torch.arange(1, H + 1, device="cuda", dtype=torch.float64) % 255 + 1.0
    sign = 1.0 - 2.0 * (torch.arange(16, device="cuda", dtype=torch.float64) % 2)
    x = (sign[:, None, None] * a[None, :, None] * 2.0 ** -6).expand(16, H, D).reshape(1, 16, C).float()
    context = gact.make_group_norm_context(x, H)
    gact.gact_group_norm(x, H, eps=1e-5, context=context)
    assert (context.mean == 0).all()
    eps = torch.tensor(1e-5, dtype=torch.float32).double().cuda()
    v = (a * 2.0 ** -6).square() + eps
    # (D = 4: 1 / (16 D) is a power of two, so that the variance is a a itself; the root and the quotient in binary64)
    assert torch.equal(context.rstd[0], v.rsqrt().float())
