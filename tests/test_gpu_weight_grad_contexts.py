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
