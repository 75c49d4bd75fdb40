"""The inference-cache calls in forms that other tests leave out: 17 to 32 columns over caches larger than the GPU's.
Oracle and tolerances as in test_gpu_cache_weights.py.
"""
import numpy as np
import pytest
import torch

import paper_2506_11498_amd as lrsa
from oracle import lrsa_cache_ops as ops
from test_gpu_cache_quant import CODES, i32
from test_gpu_cache_weights import DEV, DT, close_attention, params

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt,dtype,d,n", [("int8", "bf16", 128, 33000), ("e4m3", "f32", 64, 66000), ("e4m3", "bf16", 64, 17000)])
def test_two_groups_of_columns(fmt, dtype, d, n):
    """20 columns on both sides of 256 MB, with weights and without (the same bits); two units are compared."""
    B, Hkv, G, T, block = 8, 8, 4, 5, 64
    cap, lens = n + 9, [n - 17 * b for b in range(B)]
    g = torch.Generator(device=DEV).manual_seed(n)
    raw = [torch.randint(0, 256, (B, Hkv, cap, d), generator=g, device=DEV, dtype=torch.uint8) for _ in range(2)]
    if fmt == "e4m3":
        raw = [r.bitwise_and_(0xbf) for r in raw]                               # magnitudes below 2
    scales = [torch.exp2(torch.randint(-9, -5, (B, Hkv, -(-cap // block)), generator=g, device=DEV).float()) * (64 if fmt == "e4m3" else 1) for _ in range(2)]
    cache = lrsa.QuantCache(*(r.view(CODES[fmt]) for r in raw), *scales, block)
    q = torch.randn((B, Hkv * G, T, d), generator=g, device=DEV).to(DT[dtype])
    p = params(B, Hkv * G, Hkv, cap, d, (Hkv * cap * d, cap * d, d, 1), DT[dtype])
    out = torch.full((B, Hkv, cap), -7.0, device=DEV)
    O, lse = lrsa.lrsa_decode_attn_quant(p, q, cache, i32(lens), n, None, out)
    O1, lse1 = lrsa.lrsa_decode_attn_quant(p, q, cache, i32(lens), n)
    assert torch.equal(O, O1) and torch.equal(lse, lse1)
    assert all(bool((out[b, :, m:] == -7.0).all()) for b, m in enumerate(lens))
    for b, h in ((0, 7), (5, 2)):
        hs, m = slice(h * G, (h + 1) * G), lens[b]
        K, V = (ops.values(r[b, h, :m].cpu().numpy(), s[b, h, :-(-m // block)].cpu().numpy(), block, fmt) for r, s in zip(raw, scales))
        qs = q[b, hs].double().cpu().numpy()
        O_ref, lse_ref, w = ops.attend(qs, K, V)
        eps = close_attention(O[b, hs].double().cpu().numpy(), lse[b, hs].double().cpu().numpy(), qs, K, V, O_ref, lse_ref, d ** -0.5,
                              2.0 ** -8 if dtype == "bf16" else 2.0 ** -24)
        assert np.all(np.abs(out[b, h, :m].double().cpu().numpy() - w) <= 2 * eps * w + 1e-37)
