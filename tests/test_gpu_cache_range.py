"""The cache in 8 bits at the ends of its range: rows of zeros out of blocks with large scales.  Oracle as in test_gpu_cache_quant.py.
"""
import numpy as np
import pytest
import torch

import paper_2506_11498_amd as lrsa
from oracle import lrsa_cache_ops as ops
from test_gpu_cache_quant import CODES, host, i32
from test_gpu_cache_weights import DEV, params

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("d", [128, 64])
@pytest.mark.parametrize("n,budget", [(96, 60), (9000, 1300)])
def test_rows_of_zeros_stay_zero_whatever_the_scale_that_they_leave(fmt, d, n, budget):
    """Every block has one row that is not zero, which goes; the scales reach to the largest.  A block of zeros alone has the least scale: the
    ratio of the two is beyond the numbers of 32 bits.  One launch and two."""
    block, nb = 16, -(-n // 16)
    raw = torch.zeros((1, 1, n, d), dtype=torch.uint8)
    raw[:, :, ::block] = 0x31
    raw[:, :, 5::block, ::3] = 0x80 if fmt == "e4m3" else 0                       # minus zero
    scales = torch.exp2(torch.tensor([119, 20, 8, 7, 6, 0, -100, -120])[torch.arange(nb) % 8].float()).view(1, 1, nb)
    acc = torch.ones((1, 1, n))
    acc[:, :, ::block] = 0
    one = 7 * n // 8 // block * block + 1                                          # not zero, and stays, in a block with zeros
    raw[:, :, one], acc[:, :, one] = 0x32, 2
    cache = lrsa.QuantCache(*(raw.to(DEV).view(CODES[fmt]) for _ in range(2)), *(scales.to(DEV) for _ in range(2)), block)
    out = lrsa.QuantCache.empty(1, 1, n, d, CODES[fmt], block, DEV)
    p = params(1, 1, 1, n, d, (n * d, n * d, d, 1), torch.float32)
    ao, lo = torch.empty((1, 1, n), device=DEV), i32([0])
    lrsa.lrsa_cache_evict_quant(p, cache, None, acc.to(DEV), i32([n]), n, budget, 0, out, None, ao, lo)
    rows = ops.evict_rows(acc[0, 0].numpy(), n, 0, 0, budget)
    codes, want = ops.evict_blocks(ops.values(raw[0, 0].numpy(), scales[0, 0].numpy(), block, fmt)[rows], block, fmt)
    got = host(out)
    for z in range(2):
        assert np.array_equal(got[2 + z][0, 0, :len(want)].astype(np.float64), want)
        assert np.array_equal(ops.decode(got[z][0, 0, :budget], fmt), ops.decode(codes, fmt))
