"""How many bits of a softmax numerator reach the result of the paged attention.

Scores are exact in fp32 and every value is a power of two, so that nothing but the numerators' splitting into 16-bit terms and the
sums round. All numerators but each block's largest, which is 1, are chosen so that two bf16 terms would be short of them, by
three quarters of the most they can be: a result of two terms is off by more than the limit, which the test says of the plain
sums before it looks at the kernel's."""
import numpy as np
import pytest
import torch

from paged_util import build, rows

pytestmark = pytest.mark.gpu

SCALE = float(np.float32(0.6931472))                                 # times log2(e), in fp32, is 1: scores are powers of two's exponents


def _bf16(x):
    return torch.from_numpy(np.ascontiguousarray(x)).float().bfloat16().double().numpy()


def _short_of_two_terms():
    """Exponents -i / 2^14 of numerators in [1/2, 1) whose third bf16 term is 0.75 to 0.95 of its largest, 2^-18, and positive."""
    x = -np.arange(1, 1 << 14) / 2.0 ** 14
    e = np.exp2(x)
    first = _bf16(e)
    rest = e - first - _bf16(e - first)
    return x[(rest > 0.75 * 2.0 ** -18) & (rest < 0.95 * 2.0 ** -18)]


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("D,G", [(64, 8), (128, 1), (128, 4), (256, 7), (64, 12), (128, 16)])
@pytest.mark.parametrize("n", [10, 16, 33, 47, 60])
def test_numerators_keep_their_bits(dtype, D, G, n):
    """The limit, in units of 2^-24 of the result. Normaliser: 3 additions in a lane, 1 with the running sum, 3 between lanes, 4 between
    warps. Weighted values: an MMA adds 16 exact products to its accumulator, off by at most 2^-22 of their magnitudes, 4 units; a
    block of 16 rows takes three of them, with more than eight heads two blocks are chained; 1 with the running
    sum, 2 between warps. What three terms leave: 1. Reciprocal and product: 2."""
    cache, gen = build([n], H=1, G=G, D=D, page_size=16, dtype=dtype)
    x = np.random.default_rng(n).choice(_short_of_two_terms(), n)
    x[::16] = 0.0                                                    # the largest of 16 rows, and of 32
    e = np.exp2(x)
    terms = _bf16(e) + _bf16(e - _bf16(e))
    limit = (11 + 12 * (1 if G <= 8 else 2) + 3 + 1 + 2) * 2.0 ** -24
    assert abs(terms.sum() / e.sum() - 1) > limit
    # <q, k> = high + low / 128: seven bits each
    high = np.floor(x * 128) / 128
    low = (x - high) * 128
    page, off = rows(cache, 0, n)
    cache.k_pages[page, 0, off] = 0.0
    cache.k_pages[page, 0, off, 3] = torch.from_numpy(high).to("cuda", cache.k_pages.dtype)
    cache.k_pages[page, 0, off, D - 7] = torch.from_numpy(low).to("cuda", cache.k_pages.dtype)
    value = torch.exp2((torch.arange(D, device="cuda") % 5 - 2).double())
    cache.v_pages[page, 0, off] = value.to(cache.v_pages.dtype)
    q = torch.zeros(1, G, D, dtype=cache.k_pages.dtype, device="cuda")
    q[..., 3], q[..., D - 7] = 1.0, 1 / 128
    assert (torch.einsum("gd,ld->gl", q[0].double(), cache.k_pages[page, 0, off].double()).cpu().numpy() == x).all()
    out = cache.laser_kv_paged_attention(q, softmax_scale=SCALE).double() / value
    assert (out - 1).abs().max().item() <= limit
