"""The cache in 8 bits at the ends of its range: rows of zeros out of blocks with large scales, the largest numbers, small
values in attention.  Oracle as in test_gpu_cache_quant.py.
"""
import numpy as np
import pytest
import torch

import paper_2506_11498_amd as lrsa
from oracle import lrsa_cache_ops as ops
from test_gpu_cache_quant import CODES, host, i32
from test_gpu_cache_weights import DEV, DT, close_attention, params

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


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("dtype,d,B,Hkv,G,T,n", [
    ("f32", 128, 1, 1, 4, 1, 5), ("f32", 64, 2, 2, 2, 3, 700), ("bf16", 128, 1, 2, 4, 1, 3000), ("f32", 128, 1, 1, 20, 1, 2500), ("f32", 64, 4, 8, 4, 5, 21000),
    ("bf16", 128, 4, 8, 4, 5, 21000),
])
def test_attention_keeps_its_bits_where_values_are_small(fmt, dtype, d, B, Hkv, G, T, n):
    """Scales of V that are 2^-k of others (powers of two, different ones along the cache) give outputs that are 2^-k of theirs, bit for bit: no
    product, weight or sum has fewer bits there, as long as the outputs themselves are normal numbers."""
    block = 16
    g = torch.Generator(device=DEV).manual_seed(n + G)
    raw = [torch.randint(0, 256, (B, Hkv, n, d), generator=g, device=DEV, dtype=torch.uint8) for _ in range(2)]
    for r in raw:
        r.bitwise_and_(0xbf if fmt == "e4m3" else 0xff)                          # e4m3: magnitudes below 2
    nb = -(-n // block)
    Ks = torch.exp2(torch.randint(-9, -5, (B, Hkv, nb), generator=g, device=DEV).float()) * (64 if fmt == "e4m3" else 1)
    Vs = torch.exp2(torch.randint(0, 5, (B, Hkv, nb), generator=g, device=DEV).float())
    q = torch.randn((B, Hkv * G, T, d), generator=g, device=DEV).to(DT[dtype])
    p, lens = params(B, Hkv * G, Hkv, n, d, (Hkv * n * d, n * d, d, 1), DT[dtype]), i32([n - 3 * b for b in range(B)])
    outs = []
    for k in (8, 40, 104, 113):
        cache = lrsa.QuantCache(*(r.view(CODES[fmt]) for r in raw), Ks, Vs * 2.0 ** -k, block)
        outs.append(lrsa.lrsa_decode_attn_quant(p, q, cache, lens, n))
        want = torch.ldexp(outs[0][0].double(), torch.tensor(8.0 - k, device=DEV)).to(DT[dtype])
        normal = want.abs() >= torch.finfo(DT[dtype]).tiny
        assert torch.equal(outs[-1][1], outs[0][1]) and bool((outs[-1][0] == want)[normal].all()) and float(normal.float().mean()) > 0.9


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_small_and_large_values_in_one_cache(fmt):
    """V scales from the least to 2^60 in one cache; tokens that see the small ones alone, the large ones among them or first."""
    d, block, n, G = 128, 16, 160, 4
    g = torch.Generator().manual_seed(12)
    raw = [torch.randint(0, 256, (1, 1, n, d), generator=g, dtype=torch.uint8) & (0xbf if fmt == "e4m3" else 0xff) for _ in range(2)]
    q = torch.randn((1, G, 1, d), generator=g)
    p = params(1, G, 1, n, d, (n * d, n * d, d, 1), torch.float32)
    Ks = torch.full((1, 1, n // block), 2.0 ** -8 if fmt == "int8" else 0.5)
    for order in ([-120, -118, -100, -80, -40, -20, 0, 3, 30, 60], [60, 30, 3, 0, -20, -40, -80, -100, -118, -120]):
        Vs = torch.exp2(torch.tensor(order).float()).view(1, 1, -1)
        cache = lrsa.QuantCache(*(r.to(DEV).view(CODES[fmt]) for r in raw), Ks.to(DEV), Vs.to(DEV), block)
        for m in (1, 16, 20, 33, 100, 111, 160):
            O, lse = lrsa.lrsa_decode_attn_quant(p, q.to(DEV), cache, i32([m]), n)
            k, v = (ops.values(r[0, 0].numpy(), s[0, 0].numpy(), block, fmt)[:m] for r, s in zip(raw, (Ks, Vs)))
            qs = q[0].double().numpy()
            O_ref, lse_ref, _ = ops.attend(qs, k, v)
            close_attention(O[0].double().cpu().numpy(), lse[0].double().cpu().numpy(), qs, k, v, O_ref, lse_ref, d ** -0.5, 2.0 ** -24)
