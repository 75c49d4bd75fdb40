"""Attention over the inference-time caches and eviction where their work is divided in other ways: short caches in one launch and their
limits, long walks of many columns, more sequences than a wave has lanes, many heads, rows far apart.  Oracle and tolerances as in test_gpu_cache_weights.py.
"""
import numpy as np
import pytest
import torch

import paper_2506_11498_amd as lrsa
from oracle import lrsa_cache_ops as ops
from test_gpu_cache_quant import CODES, check_attention, host, i32, make_cache
from test_gpu_cache_weights import DEV, DT, close_attention, params

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt,dtype,d", [("int8", "bf16", 128), ("e4m3", "bf16", 64), ("e4m3", "f32", 128), ("int8", "f32", 64)])
@pytest.mark.parametrize("G,T,lens,max_len", [
    (1, 1, [512, 1, 0], 512), (16, 1, [513, 32], 513), (5, 3, [1024, 2, 1023, 257], 1024), (4, 4, [1025, 1000], 1025), (2, 1, [5000, 700], 1024),
    (4, 1, [(37 * i) % 1025 for i in range(64)], 1024),
])
def test_short_caches(fmt, dtype, d, G, T, lens, max_len):
    """On both sides of the lengths and of the number of heads at which the work is divided otherwise; some sequences far shorter than
    the bound, some without rows, one longer than it."""
    B, Hkv, cap = len(lens), 2, max(max(lens), max_len) + 7
    g = torch.Generator().manual_seed(max_len + G)
    cache, _, _ = make_cache(B, Hkv, cap, d, fmt, 32, g, lens)
    q = torch.randn((B, Hkv * G, T, d), generator=g).to(DT[dtype])
    p = params(B, Hkv * G, Hkv, cap, d, (Hkv * cap * d, cap * d, d, 1), DT[dtype])
    check_attention(p, cache, q, lens, max_len, torch.rand((B, Hkv, cap), generator=g), 0.5, fmt, dtype)


@pytest.mark.parametrize("fmt,dtype,d,G,T", [
    ("int8", "bf16", 128, 4, 5), ("e4m3", "bf16", 128, 4, 12), ("int8", "bf16", 64, 5, 16), ("e4m3", "bf16", 128, 10, 16), ("int8", "f32", 128, 4, 5),
    ("e4m3", "f32", 64, 9, 4),
])
def test_long_walks_of_many_columns(fmt, dtype, d, G, T):
    """20 to 160 columns over 32 units of 21000 rows, so that a workgroup walks 40 tiles and more; two units are compared."""
    B, Hkv, n, block = 4, 8, 21000, 64
    cap, lens = n + 9, [21000, 20999, 20480, 20970]
    g = torch.Generator(device=DEV).manual_seed(G * T)
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
    # every unit's weights sum to the number of its columns: in each the relative error is that of a weight, at most 2^-14 here
    sums = torch.stack([out[b, :, :m].double().sum(-1) for b, m in enumerate(lens)])
    assert bool(((sums - G * T).abs() <= 2.0 ** -13 * G * T).all())
    for b, h in ((0, 7), (2, 3)):
        hs, m = slice(h * G, (h + 1) * G), lens[b]
        K, V = (ops.values(r[b, h, :m].cpu().numpy(), s[b, h, :-(-m // block)].cpu().numpy(), block, fmt) for r, s in zip(raw, scales))
        qs = q[b, hs].double().cpu().numpy()
        O_ref, lse_ref, w = ops.attend(qs, K, V)
        eps = close_attention(O[b, hs].double().cpu().numpy(), lse[b, hs].double().cpu().numpy(), qs, K, V, O_ref, lse_ref, d ** -0.5,
                              2.0 ** -8 if dtype == "bf16" else 2.0 ** -24)
        assert 2 * eps <= 2.0 ** -13
        assert np.all(np.abs(out[b, h, :m].double().cpu().numpy() - w) <= 2 * eps * w + 1e-37)


@pytest.mark.parametrize("fmt,dtype,d,B,Hkv,G,T,most", [
    ("int8", "bf16", 128, 70, 4, 2, 1, 1500), ("e4m3", "f32", 64, 130, 1, 3, 1, 1100), ("int8", "bf16", 64, 130, 5, 18, 1, 300), ("e4m3", "bf16", 128, 64, 2, 1, 1, 2000),
])
def test_many_sequences(fmt, dtype, d, B, Hkv, G, T, most):
    """More sequences than a wave has lanes, more units than run at once; every fifth sequence is empty."""
    lens = [0 if b % 5 == 3 else 1 + (997 * b) % most for b in range(B)]
    lens[-1] = most
    g = torch.Generator().manual_seed(B + most)
    cache, _, _ = make_cache(B, Hkv, most, d, fmt, 16, g, lens, strided=False)
    q = torch.randn((B, Hkv * G, T, d), generator=g).to(DT[dtype])
    p = params(B, Hkv * G, Hkv, most, d, (Hkv * most * d, most * d, d, 1), DT[dtype])
    check_attention(p, cache, q, lens, most, torch.rand((B, Hkv, most), generator=g), 2.0, fmt, dtype)


def test_many_sequences_without_any_row():
    g = torch.Generator().manual_seed(1)
    cache, _, _ = make_cache(70, 4, 1500, 128, "int8", 64, g, [0] * 70, strided=False)
    q = torch.randn((70, 8, 1, 128), generator=g).to(torch.bfloat16)
    p = params(70, 8, 4, 1500, 128, (4 * 1500 * 128, 1500 * 128, 128, 1), torch.bfloat16)
    check_attention(p, cache, q, [0] * 70, 1500, torch.rand((70, 4, 1500), generator=g))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_far_apart(dtype):
    """Single-query attention with and without weights, and eviction, over caches whose rows are 16 MiB and more apart: the bits of the
    packed cache."""
    B, Hkv, G, d, cap, n, T = 1, 2, 4, 128, 100, 97, DT[dtype]
    g = torch.Generator(device=DEV).manual_seed(8)
    near = [torch.randn((B, Hkv, cap, d), generator=g, device=DEV).to(T) for _ in range(2)]
    st = (cap << 23, d, 1 << 23, 1)
    far = [torch.empty((cap - 1 << 23) + Hkv * d, dtype=T, device=DEV).as_strided(x.shape, st) for x in near]
    for a, b in zip(far, near):
        a.copy_(b)
    q = torch.randn((B, Hkv * G, d), generator=g, device=DEV).to(T)
    got = []
    for K, V in (near, far):
        p = params(B, Hkv * G, Hkv, cap, d, K.stride(), T, sink=3)
        acc = torch.ones((B, Hkv, cap), device=DEV)
        O, lse, _ = lrsa.lrsa_decode_attn_acc(p, q, K, V, n, acc, acc)
        O1, lse1 = lrsa.lrsa_decode_attn(p, q, K, V, n)
        Ko, Vo = (torch.zeros(x.untyped_storage().nbytes() // x.element_size(), dtype=T, device=DEV).as_strided(x.shape, x.stride()) for x in (K, V))
        acc_o = torch.empty_like(acc)
        lrsa.lrsa_cache_evict(p, K, V, None, acc, n, 50, 10, Ko, Vo, None, acc_o)
        got.append((O, lse, O1, lse1, acc, Ko[:, :, :50].clone(), Vo[:, :, :50].clone(), acc_o))
    assert all(torch.equal(a, b) for a, b in zip(*got))


@pytest.mark.parametrize("dtype,d,B,Hkv,length,budget", [("bf16", 64, 40, 8, 300, 120), ("f32", 64, 64, 1, 5000, 2100), ("bf16", 128, 16, 8, 1000, 999), ("f32", 128, 3, 1, 8192, 8191),
                                                         ("bf16", 128, 1, 2, 8193, 100), ("bf16", 64, 300, 1, 0, 5), ("f32", 128, 2, 2, 200, 100)])
def test_evictions_of_many_heads_and_at_the_limits(dtype, d, B, Hkv, length, budget):
    """One launch and two: on both sides of the length and of the number of workgroups; positions, weights and rows of all heads."""
    cap = max(length, budget) + 3
    g = torch.Generator(device=DEV).manual_seed(length + B)
    K, V = (torch.randn((B, cap, Hkv, d), generator=g, device=DEV).to(DT[dtype]).permute(0, 2, 1, 3) for _ in range(2))
    acc = torch.randint(0, 50, (B, Hkv, cap), generator=g, device=DEV).float()
    pos = torch.arange(cap, dtype=torch.int32, device=DEV).expand(B, Hkv, cap).contiguous()
    p = params(B, Hkv, Hkv, cap, d, K.stride(), DT[dtype], sink=2)
    Ko, Vo, po, ao = torch.full_like(K, 3), torch.full_like(V, 3), torch.full_like(pos, -5), torch.full_like(acc, -5)
    new = lrsa.lrsa_cache_evict(p, K, V, pos, acc, length, budget, 3, Ko, Vo, po, ao)
    assert new == min(length, budget)
    want = torch.tensor(np.stack([ops.evict_rows(a, length, 2, 3, budget) for a in acc.reshape(-1, cap).cpu().numpy()]), device=DEV).reshape(B, Hkv, new).long()
    assert torch.equal(po[:, :, :new].long(), want) and torch.equal(ao[:, :, :new], acc.gather(2, want))
    at = want[..., None].expand(B, Hkv, new, d)
    assert torch.equal(Ko[:, :, :new], K.gather(2, at)) and torch.equal(Vo[:, :, :new], V.gather(2, at))
    for t, fill in ((Ko, 3), (Vo, 3), (po, -5), (ao, 0)):
        assert bool((t[:, :, new:] == fill).all())


@pytest.mark.parametrize("fmt,d,B,Hkv,block,n,budget", [("int8", 128, 40, 8, 64, 300, 130), ("e4m3", 64, 64, 1, 128, 5000, 700), ("int8", 64, 16, 8, 16, 1000, 256), ("e4m3", 128, 3, 1, 128, 8192, 8100),
                                                        ("int8", 128, 2, 1, 32, 8193, 100), ("e4m3", 64, 130, 2, 16, 90, 50)])
def test_evictions_of_many_heads_in_eight_bits(fmt, d, B, Hkv, block, n, budget):
    """The same of ragged sequences.  Every second one is compared."""
    cap = n + 3
    lens = [n - (29 * b) % n for b in range(B)]
    lens[-1] = 0
    g = torch.Generator().manual_seed(B + n)
    cache, raw, scales = make_cache(B, Hkv, cap, d, fmt, block, g, lens, strided=False)
    out, _, _ = make_cache(B, Hkv, cap, d, fmt, block, g)
    acc = torch.randint(0, 1 << 20, (B, Hkv, cap), generator=g).float()
    p = params(B, Hkv, Hkv, cap, d, (Hkv * cap * d, cap * d, d, 1), torch.bfloat16, sink=2)
    ao, lo = torch.full((B, Hkv, cap), -3.0, device=DEV), i32([-3] * B)
    lrsa.lrsa_cache_evict_quant(p, cache, None, acc.to(DEV), i32(lens), n, budget, 3, out, None, ao, lo)
    assert lo.cpu().tolist() == [min(x, budget) for x in lens]
    got = host(out)
    for b in range(0, B, 2):
        new = min(lens[b], budget)
        for h in range(Hkv):
            rows = ops.evict_rows(acc[b, h].double().numpy(), lens[b], 2, 3, budget)
            assert torch.equal(ao[b, h, :new].cpu(), acc[b, h][torch.from_numpy(rows)]) and bool((ao[b, h, new:] == 0).all())
            for z in range(2):
                x = ops.values(raw[z][b, h].numpy()[:lens[b]], scales[z][b, h].numpy(), block, fmt)[rows] if lens[b] else np.zeros((0, d))
                codes, s = ops.evict_blocks(x, block, fmt)
                assert np.array_equal(ops.decode(got[z][b, h, :new], fmt), ops.decode(codes, fmt))
                assert np.array_equal(got[2 + z][b, h, :len(s)].astype(np.float64), s)


@pytest.mark.parametrize("d,B,n", [(128, 9, 10300), (64, 17, 10301)])
def test_large_bf16_caches(d, B, n):
    """Caches of more than 320 MiB, read past the GPU's caches; two units are compared, and the bits with and without weights."""
    Hkv, G, T, cap = 8, 5, torch.bfloat16, n + 3
    g = torch.Generator(device=DEV).manual_seed(n)
    K, V = (torch.randn((B, Hkv, cap, d), generator=g, device=DEV, dtype=torch.float32).to(T) for _ in range(2))
    K[:, :, n:], V[:, :, n:] = float("nan"), float("inf")
    q = torch.randn((B, Hkv * G, d), generator=g, device=DEV).to(T)
    p = params(B, Hkv * G, Hkv, cap, d, K.stride(), T)
    acc = torch.full((B, Hkv, cap), -7.0, device=DEV)
    O, lse, _ = lrsa.lrsa_decode_attn_acc(p, q, K, V, n, None, acc)
    O1, lse1 = lrsa.lrsa_decode_attn(p, q, K, V, n)
    assert torch.equal(O, O1) and torch.equal(lse, lse1) and bool((acc[:, :, n:] == -7.0).all())
    for b, h in ((0, 3), (B - 1, 7)):
        hs = slice(h * G, (h + 1) * G)
        Kh, Vh, qs = (x.double().cpu().numpy() for x in (K[b, h, :n], V[b, h, :n], q[b, hs][:, None]))
        O_ref, lse_ref, w = ops.attend(qs, Kh, Vh)
        eps = close_attention(O[b, hs][:, None].double().cpu().numpy(), lse[b, hs][:, None].double().cpu().numpy(), qs, Kh, Vh, O_ref, lse_ref, d ** -0.5, 2.0 ** -8)
        assert np.all(np.abs(acc[b, h, :n].double().cpu().numpy() - w) <= 2 * eps * w + 1e-37)


@pytest.mark.parametrize("fmt,dtype,d,B,n,T", [("int8", "bf16", 128, 8, 16500, 1), ("e4m3", "f32", 64, 17, 16400, 2)])
def test_large_caches_in_eight_bits(fmt, dtype, d, B, n, T):
    """The same of more than 256 MiB of codes, sequences of unequal length."""
    Hkv, G, block, cap = 8, 4, 64, n + 5
    lens = [n - 11 * b for b in range(B)]
    lens[2] = 0
    g = torch.Generator(device=DEV).manual_seed(n)
    raw = [torch.randint(0, 256, (B, Hkv, cap, d), generator=g, device=DEV, dtype=torch.uint8) for _ in range(2)]
    if fmt == "e4m3":
        raw = [r.bitwise_and_(0xbf) for r in raw]
        for r in raw:
            r[(r & 0x7f) == 0x7f] = 0x31
    scales = [torch.exp2(torch.randint(-9, -5, (B, Hkv, -(-cap // block)), generator=g, device=DEV).float()) * (64 if fmt == "e4m3" else 1) for _ in range(2)]
    cache = lrsa.QuantCache(*(r.view(CODES[fmt]) for r in raw), *scales, block)
    q = torch.randn((B, Hkv * G, T, d), generator=g, device=DEV).to(DT[dtype])
    p = params(B, Hkv * G, Hkv, cap, d, (Hkv * cap * d, cap * d, d, 1), DT[dtype])
    out = torch.full((B, Hkv, cap), -7.0, device=DEV)
    O, lse = lrsa.lrsa_decode_attn_quant(p, q, cache, i32(lens), n, None, out)
    O1, lse1 = lrsa.lrsa_decode_attn_quant(p, q, cache, i32(lens), n)
    assert torch.equal(O, O1) and torch.equal(lse, lse1)
    assert all(bool((out[b, :, m:] == -7.0).all()) for b, m in enumerate(lens)) and bool((O[2] == 0).all()) and bool(torch.isneginf(lse[2]).all())
    for b, h in ((1, 0), (B - 1, 6)):
        hs, m = slice(h * G, (h + 1) * G), lens[b]
        K, V = (ops.values(r[b, h, :m].cpu().numpy(), s[b, h, :-(-m // block)].cpu().numpy(), block, fmt) for r, s in zip(raw, scales))
        qs = q[b, hs].double().cpu().numpy()
        O_ref, lse_ref, w = ops.attend(qs, K, V)
        eps = close_attention(O[b, hs].double().cpu().numpy(), lse[b, hs].double().cpu().numpy(), qs, K, V, O_ref, lse_ref, d ** -0.5, 2.0 ** -8 if dtype == "bf16" else 2.0 ** -24)
        assert np.all(np.abs(out[b, h, :m].double().cpu().numpy() - w) <= 2 * eps * w + 1e-37)
