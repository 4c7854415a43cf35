"""Sums of a code word's blocks, the gradient of a code book, against float64.

A piece of 256 float32 values is off by at most 255 2^-24 of the sum of their
sizes, the pieces' float64 sum by less than 2^-50 of it, the result's rounding by
2^-24: 256 2^-24 of the sizes with a hundredth added.
"""

import pytest
import torch

from paper_2609_21137_amd import fit


def _check(device, n, K, d, kind):
    g = torch.Generator().manual_seed(n + K)
    codes = torch.randint(0, K, (n,), generator=g)
    if kind == "uneven":
        codes = torch.where(torch.rand(n, generator=g) < 0.9, 1 % K, codes)      # most blocks one word's
        codes[codes == K - 1] = 0                                               # and one word's none
    blocks = torch.rand((n, d), generator=g) * 0.1 + 0.3 if kind != "signed" else torch.randn((n, d), generator=g)
    want = torch.zeros(K, d, dtype=torch.float64).index_add_(0, codes, blocks.double())
    size = torch.zeros(K, d, dtype=torch.float64).index_add_(0, codes, blocks.double().abs())
    codes, blocks = codes.to(device), blocks.to(device)
    sums = fit._WordSums(codes, K)
    got = sums(blocks)
    assert got.dtype == torch.float32 and got.shape == (K, d)
    assert ((got.double().cpu() - want).abs() <= 1.01 * 256 * 2.0 ** -24 * size).all()
    assert torch.equal(got, sums(blocks))


CASES = [(1, 1, 4), (7, 16, 2), (255, 1, 4), (256, 1, 4), (257, 1, 8), (1000, 256, 4), (50000, 16, 4)]


@pytest.mark.parametrize("kind", ["level", "uneven", "signed"])
@pytest.mark.parametrize("n,K,d", CASES)
def test_on_the_host(n, K, d, kind):
    _check("cpu", n, K, d, kind)


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["level", "uneven", "signed"])
@pytest.mark.parametrize("n,K,d", CASES + [(600000, 4, 4), (3000000, 16, 2)])
def test_on_the_gpu(n, K, d, kind):
    print(f"[word sums] n={n} K={K} d={d} {kind}", flush=True)
    _check("cuda", n, K, d, kind)
