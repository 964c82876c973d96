"""The weight gradient where values of its context are not finite: they reach the columns that hold them, and nothing else."""
import pytest
import torch

import paper_2206_11357_amd as gact

pytestmark = pytest.mark.gpu

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}

# every form of tiles, groups of whole chunks and others; the last group is short, and the last chunk has tokens that there are none of,
# some of whose elements would fall into that group
SHAPES = [(3, 200, 200, 96), (1, 130, 72, 64), (17, 40, 72, 64), (2001, 24, 200, 64), (2001, 24, 200, 96), (2002, 200, 24, 32),
          (3001, 130, 104, 64), (3001, 130, 104, 96), (19001, 512, 520, 256), (19001, 510, 501, 96)]


def inputs(T, N, K, G, bits, dtype):
    gen = torch.Generator(device="cuda").manual_seed(T + 31 * N + 7 * K)
    x = (torch.randn(T, K, generator=gen, device="cuda") + 0.3).to(dtype)
    dy = (torch.rand(T, N, generator=gen, device="cuda") + 0.5).to(dtype)          # no zeros
    return x, dy, gact.gact_compress(x, G, bits, 5)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("bits", [1, 4, 8])
@pytest.mark.parametrize("T,N,K,G", SHAPES)
def test_the_last_group_stays_in_its_columns(T, N, K, G, bits, dtype):
    x, dy, context = inputs(T, N, K, G, bits, DTYPES[dtype])
    first = T * K // G * G
    assert 0 < T * K - first < K and T * K % G != 0
    clean, clean_b = gact.gact_linear_weight_grad(dy, *context, K, G, bits, w_dtype=torch.float32, bias=True)
    held = torch.zeros(K, dtype=torch.bool, device="cuda")
    held[torch.arange(first, T * K, device="cuda") % K] = True
    for which, value in ((1, float("inf")), (1, float("nan")), (2, float("inf")), (2, float("nan"))):
        poisoned = [t.clone() for t in context]
        poisoned[which][-1] = value
        dw, db = gact.gact_linear_weight_grad(dy, *poisoned, K, G, bits, w_dtype=torch.float32, bias=True)
        assert torch.equal(dw[:, ~held], clean[:, ~held]) and torch.equal(db, clean_b)
        if value != value or which == 1:            # (an infinite step times code 0 is no number, times another one an infinity)
            assert not torch.isfinite(dw[:, held]).any()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,N,K,G", SHAPES)
def test_an_infinity_that_was_compressed(T, N, K, G, dtype):
    """From the compressor on: an infinity among the last elements, and what gact_decompress makes of it."""
    x, dy, context = inputs(T, N, K, G, 4, DTYPES[dtype])
    x.view(-1)[-1] = float("inf")
    poisoned = gact.gact_compress(x, G, 4, 5)
    back = gact.gact_decompress(*poisoned, T * K, G, 4, dtype=x.dtype).view(T, K)
    bad = ~torch.isfinite(back).all(0)
    assert bad.any() and not bad.all()
    clean, _ = gact.gact_linear_weight_grad(dy, *context, K, G, 4, w_dtype=torch.float32)
    dw, _ = gact.gact_linear_weight_grad(dy, *poisoned, K, G, 4, w_dtype=torch.float32)
    assert torch.equal(dw[:, ~bad], clean[:, ~bad]) and not torch.isfinite(dw[:, bad]).any()


# every form again
FORMS = [(1, 130, 72), (64, 100, 100), (2000, 24, 200), (2000, 200, 24), (3001, 130, 104), (19000, 512, 512), (19001, 510, 501)]


@pytest.mark.parametrize("w_dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,N,K", FORMS)
def test_binary32_sums_as_binary32_has_them(T, N, K, w_dtype):
    """Infinities keep their sign where no infinity is against them, zeros and infinities make NaN, and elements that bfloat16 has
    no number for (from 2^128 - 2^119 on) count as they are."""
    G, bits = 64, 2
    gen = torch.Generator(device="cuda").manual_seed(T + N)
    x = torch.rand(T, K, generator=gen, device="cuda") * 0.5 + 0.25
    x.view(-1)[torch.arange(0, T * K, G, device="cuda")] = 0.0                    # minima: code 0 is zero
    context = gact.gact_compress(x, G, bits, 3)
    if T > 1:
        context[1][-1] = -float("inf")
    dy = torch.randn(T, N, generator=gen, device="cuda")
    dy[T // 2, 3], dy[T // 3, 9], dy[T - 1, 11] = float("nan"), float("inf"), -float("inf")
    dy[0, 15], dy[T // 2, 17], dy[T - 1, 17] = 3.4e38, -3.4e38, float("inf") if T > 1 else -3.4e38
    dw, db = gact.gact_linear_weight_grad(dy, *context, K, G, bits, w_dtype=DTYPES[w_dtype], bias=True)
    back = gact.gact_decompress(*context, T * K, G, bits).view(T, K).cpu().double()
    d = dy.cpu().double()
    bad = ~torch.isfinite(back).all(0)
    size = d.abs().t() @ back.abs()
    want = d.t() @ back
    got = dw.cpu().double()
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    # a bfloat16 dW has no number for sums within half a step of 2^128
    sure = torch.isinf(want)
    assert torch.equal(got[sure], want[sure])
    # T products and additions of binary32, each off by 2^-23 of the terms' sizes at most (in matrix products that cut), and the output's half step
    half = 2.0 ** -24 if w_dtype == "f32" else 2.0 ** -8
    fine = torch.isfinite(want) & (size < 3.38e38)
    bound = half * want.abs() + (T + 2) * 2.0 ** -23 * size * (1 + half) + 2.0 ** -126
    assert ((got - want).abs() <= bound)[fine].all()
    assert torch.isnan(want[3]).all()
    if not bad.all():                                   # (24 columns are all in the last group)
        assert fine[15].sum() >= (K - bad.sum()) // 2 and torch.isinf(want[9]).any()


@pytest.mark.parametrize("T,N,K", FORMS)
def test_small_elements_in_binary32(T, N, K):
    """Elements that bfloat16's least number, 2^-133, cuts the parts of: x^ is 1, and dW is dy's one row up to 2^-134 and the roundings of
    test_each_product_is_exact_to_a_rounding."""
    context = gact.gact_compress(torch.ones(T, K, device="cuda"), 32, 4, 1)
    gen = torch.Generator(device="cuda").manual_seed(N)
    dy = torch.zeros(T, N, device="cuda")
    exponents = -100.0 - (torch.arange(N, device="cuda") % 27)
    dy[T // 2] = (1.0 + torch.rand(N, generator=gen, device="cuda")) * 2.0 ** exponents
    dw, db = gact.gact_linear_weight_grad(dy, *context, K, 32, 4, bias=True)
    want = dy[T // 2].double()[:, None]
    off = (dw.double() - want).abs() - (2.0 ** -24 + 7 * 2.0 ** -23) * want - 2.0 ** -134
    assert off.max() <= 0 and torch.equal(db, dy[T // 2])
