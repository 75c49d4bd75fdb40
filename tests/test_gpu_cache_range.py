"""The cache in 8 bits at the ends of its range: rows of zeros out of blocks with large scales, the largest numbers.  Oracle as in test_gpu_cache_quant.py.
"""
import numpy as np
import pytest
import torch

import paper_2506_11498_amd as lrsa
from oracle import lrsa_cache_ops as ops
from test_gpu_cache_quant import CODES, host, i32
from test_gpu_cache_weights import DEV, DT, params

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


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("dtype,block", [("f32", 16), ("bf16", 32)])
def test_finite_values_stay_finite(fmt, dtype, block):
    """Rows up to the largest finite number: codes and scales of the definition, and every value that is read back is finite and off by at
    most half a step of its scale, or is the largest one where the row's is beyond it.  The same after a move to another cache, and in attention over one row."""
    T, d, big, least = DT[dtype], 64, ops.LARGEST[fmt], 2.0 ** 118
    most = torch.finfo(T).max
    x = torch.linspace(0, 1, block * d).view(block, d).double() * (most - least) + least
    x[::2] *= -1
    x[-1, -1] = most
    x = torch.cat([x, x.clamp(-big, big), x * 2.0 ** -1]).to(T).clamp(-most, most)[None, None]      # the first block above the largest value, the second just below
    n = x.shape[2]
    cache, other = (lrsa.QuantCache.empty(1, 1, n, d, CODES[fmt], block, DEV) for _ in range(2))
    p = params(1, 1, 1, n, d, x.stride(), T)
    lrsa.lrsa_cache_append_quant(p, cache, x.to(DEV), x.to(DEV), i32([0]))
    codes, scales = ops.append(np.zeros((n, d), np.uint8), np.ones(3), block, fmt, 0, x[0, 0].double().numpy())
    got = host(cache)
    assert np.array_equal(got[2][0, 0].astype(np.float64), scales)
    assert np.array_equal(ops.decode(got[0][0, 0], fmt), ops.decode(codes, fmt))
    Kr, Vr = lrsa.lrsa_cache_read_quant(p, cache, i32([n]), n)
    r, want = Kr[0, 0].double().cpu().numpy(), x[0, 0].double().numpy()
    assert np.all(np.isfinite(r)) and torch.equal(Kr, Vr)
    step = scales.repeat(block)[:, None] * (1.0 if fmt == "int8" else 2.0 ** -9)
    kept = np.clip(want, -big, big)
    assert np.all(np.abs(r - kept) <= step / 2 + (0.0 if fmt == "int8" else 2.0 ** -4) * np.abs(kept))
    ao, lo = torch.empty((1, 1, n), device=DEV), i32([0])
    lrsa.lrsa_cache_evict_quant(p, cache, None, torch.ones((1, 1, n), device=DEV), i32([n]), n, n, 0, other, None, ao, lo)
    assert torch.equal(other.K.view(torch.uint8), cache.K.view(torch.uint8)) and torch.equal(other.V_scale, cache.V_scale)
    # a cache of one row has a weight of one: V's values, whatever the logit
    O, _ = lrsa.lrsa_decode_attn_quant(p, torch.zeros((1, 1, 1, d), dtype=T, device=DEV), cache, i32([1]), 1)
    assert torch.equal(O[0, 0, 0], Vr[0, 0, 0])
