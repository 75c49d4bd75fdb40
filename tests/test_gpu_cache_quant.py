"""The inference-time cache in 8 bits on the GPU against the oracle in 64 bits: appending and reading (codes and scales bit for bit),
attention (tolerances as derived in test_gpu_cache_weights.py; the values of the cache are exact), eviction (bit for bit).
"""
import numpy as np
import pytest
import torch

import paper_2506_11498_amd as lrsa
from oracle import lrsa_cache_ops as ops
from test_gpu_cache_weights import DEV, DT, close_attention, make_lists, params

pytestmark = pytest.mark.gpu
CODES = {"int8": torch.int8, "e4m3": torch.float8_e4m3fn}


def make_cache(B, Hkv, cap, d, fmt, block, g, lens=None, strided=True):
    """A cache of random codes and scales; behind lens, codes that are no numbers (or the largest) and scales that are none."""
    raw = [torch.randint(0, 256, (B, cap, Hkv, d) if strided else (B, Hkv, cap, d), generator=g, dtype=torch.uint8) for _ in range(2)]
    nb = -(-cap // block)
    scales = [torch.exp2(torch.randint(-9, -5, (B, Hkv, nb), generator=g).float()) for _ in range(2)]
    for i in range(2):
        if fmt == "e4m3":
            raw[i][(raw[i] & 0x7f) == 0x7f] = 0x31
            raw[i] &= 0xbf                                   # magnitudes below 2
            scales[i] *= 2.0 ** 6
        if strided:
            raw[i] = raw[i].permute(0, 2, 1, 3)
        if lens is not None:
            for b, n in enumerate(lens):
                raw[i][b, :, n:] = 0x7f
                scales[i][b, :, -(-n // block):] = float("nan")
    return lrsa.QuantCache(*(r.to(DEV).view(CODES[fmt]) for r in raw), *(s.to(DEV) for s in scales), block), raw, scales


def host(cache):
    return [t.view(torch.uint8).cpu().numpy().copy() if t.dtype != torch.float32 else t.cpu().numpy().copy() for t in (cache.K, cache.V, cache.K_scale, cache.V_scale)]


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


# ------------------------------------------------------------------------------------------------ appending and reading
@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("dtype,d,block", [("bf16", 128, 64), ("bf16", 64, 16), ("f32", 128, 128), ("f32", 64, 32)])
@pytest.mark.parametrize("tokens,lens,counts", [
    (1, [0, 1, 15, 16, 63, 64, 199], None), (200, [0, 3, 130], None), (7, [0, 5, 12, 60, 124, 190], [7, 0, 3, 1, 7, 7]), (33, [16, 100, 230], [33, 40, -2]),
    (129, [64, 1], None), (3, [199, 198, 200, 500, -4], None), (1000, [0, 37], None),
])
def test_append_and_read(fmt, dtype, d, block, tokens, lens, counts):
    """Into caches with older rows; block boundaries; rows beyond the cap (200, of no whole block) dropped; counts and lengths out of
    range; nothing else touched."""
    B, Hkv, cap, T = len(lens), 2, 200, DT[dtype]
    g = torch.Generator().manual_seed(tokens + d)
    cache, _, _ = make_cache(B, Hkv, cap, d, fmt, block, g)
    before = host(cache)
    # rows of growing size, so that scales grow within a block and between blocks; a row of zeros
    rows = [(torch.randn((B, tokens, Hkv, d), generator=g) * torch.exp2(torch.randint(-6, 5, (B, tokens, Hkv, 1), generator=g).float())).to(T) for _ in range(2)]
    rows[0][:, tokens // 2] = 0
    K, V = (x.permute(0, 2, 1, 3) for x in rows)
    p = params(B, 4, Hkv, cap, d, K.to(DEV).stride(), T)
    lrsa.lrsa_cache_append_quant(p, cache, K.to(DEV), V.to(DEV), i32(lens), None if counts is None else i32(counts))
    after = host(cache)
    n0 = [max(0, min(x, cap)) for x in lens]
    cnt = [tokens if counts is None else max(0, min(c, tokens)) for c in counts or lens]
    for z, x in ((0, K), (1, V)):
        for b in range(B):
            for h in range(Hkv):
                codes, scales = ops.append(before[z][b, h], before[2 + z][b, h].astype(np.float64), block, fmt, n0[b], x[b, h, :cnt[b]].double().numpy())
                assert np.array_equal(after[2 + z][b, h].astype(np.float64), scales)
                assert np.array_equal(after[z][b, h], codes)
    n1 = [min(a + c, cap) for a, c in zip(n0, cnt)]
    first, take = [a - 20 for a in n0], 70                    # from before the first row to behind the last
    q = params(B, 4, Hkv, cap, d, (Hkv * take * d, take * d, d, 1), T)
    Kr, Vr = lrsa.lrsa_cache_read_quant(q, cache, i32(n1), take, i32(first))
    for z, got in ((0, Kr), (1, Vr)):
        for b in range(B):
            for h in range(Hkv):
                v = ops.values(after[z][b, h], after[2 + z][b, h], block, fmt)
                want = np.array([v[r] if 0 <= r < n1[b] else np.zeros(d) for r in range(first[b], first[b] + take)])
                assert np.array_equal(got[b, h].double().cpu().numpy(), want)
    K0, _ = lrsa.lrsa_cache_read_quant(q, cache, i32([10 ** 9] * B), take)
    assert np.array_equal(K0[0, 0].double().cpu().numpy(), ops.values(after[0][0, 0], after[2][0, 0], block, fmt)[:take])


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_every_value_of_sixteen_bits_gets_the_nearest_code(fmt):
    """All bf16 numbers up to the largest code, ties and subnormals among them, in blocks whose scale is one (or, past the first
    rows, smaller powers of two: each block's own)."""
    x = torch.arange(0, 65536, dtype=torch.int32).to(torch.int16).view(torch.bfloat16)
    x = x[(x.float().abs() <= ops.TOP[fmt])]
    d, n = 128, -(-len(x) // 128)
    rows = torch.zeros(n * d, dtype=torch.bfloat16)
    rows[:len(x)] = x[torch.randperm(len(x), generator=torch.Generator().manual_seed(3))]
    rows = rows.view(1, 1, n, d)
    cap = n + 5
    cache = lrsa.QuantCache.empty(1, 1, cap, d, CODES[fmt], 64, DEV)
    p = params(1, 1, 1, cap, d, rows.stride(), torch.bfloat16)
    lrsa.lrsa_cache_append_quant(p, cache, rows.to(DEV), rows.to(DEV), i32([0]))
    codes, scales = ops.append(np.zeros((cap, d), np.uint8), np.ones(-(-cap // 64)), 64, fmt, 0, rows[0, 0].double().numpy())
    got = host(cache)
    assert np.array_equal(got[2][0, 0], scales) and np.array_equal(got[0][0, 0], codes) and np.array_equal(got[1][0, 0], codes)


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_extreme_magnitudes(fmt):
    """fp32 rows of the largest finite and the smallest normal and subnormal numbers, one block each."""
    d, block = 64, 16
    tops = [3.4028234e38, 1e-30, 2.0 ** -113, 1.2e-38, 1e-44, 0.0]
    g = torch.Generator().manual_seed(5)
    x = torch.cat([(torch.rand((block, d), generator=g) * 2 - 1) * t for t in tops])[None, None]
    cap = x.shape[2]
    cache = lrsa.QuantCache.empty(1, 1, cap, d, CODES[fmt], block, DEV)
    p = params(1, 1, 1, cap, d, x.stride(), torch.float32)
    lrsa.lrsa_cache_append_quant(p, cache, x.to(DEV), x.to(DEV), i32([0]))
    codes, scales = ops.append(np.zeros((cap, d), np.uint8), np.ones(len(tops)), block, fmt, 0, x[0, 0].double().numpy())
    got = host(cache)
    assert np.array_equal(got[2][0, 0].astype(np.float64), scales)
    # a code whose value rounds to zero keeps the sign of it or not
    assert np.array_equal(ops.decode(got[0][0, 0], fmt), ops.decode(codes, fmt))


def test_rows_that_are_no_numbers_leave_the_other_blocks_alone():
    cache = lrsa.QuantCache.empty(1, 1, 64, 64, torch.int8, 16, DEV)
    g = torch.Generator().manual_seed(6)
    x = torch.randn((1, 1, 64, 64), generator=g)
    clean = lrsa.QuantCache.empty(1, 1, 64, 64, torch.int8, 16, DEV)
    p = params(1, 1, 1, 64, 64, x.stride(), torch.float32)
    lrsa.lrsa_cache_append_quant(p, clean, x.to(DEV), x.to(DEV), i32([0]))
    x[0, 0, 20, 3], x[0, 0, 21], x[0, 0, 22, 7] = float("nan"), float("inf"), -float("inf")
    lrsa.lrsa_cache_append_quant(p, cache, x.to(DEV), x.to(DEV), i32([0]))
    a, b = host(cache), host(clean)
    for r in (slice(0, 16), slice(32, 64)):
        assert np.array_equal(a[0][0, 0, r], b[0][0, 0, r])
    assert np.array_equal(a[2][0, 0, [0, 2, 3]], b[2][0, 0, [0, 2, 3]])


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,block", [(64, 16), (2048, 64)])
def test_tokens_do_not_see_later_rows_that_are_no_numbers(fmt, dtype, n, block):
    """The last of three tokens has rows of NaN and infinities, in a block of its own: the others' outputs keep their bits, and no
    code or scale becomes one that is no number."""
    d, T = 128, DT[dtype]
    g = torch.Generator().manual_seed(n)
    x, q = torch.randn((1, 1, n + 1, d), generator=g).to(T), torch.randn((1, 4, 3, d), generator=g).to(T).to(DEV)
    outs = []
    for bad in (False, True):
        cache = lrsa.QuantCache.empty(1, 1, n + 70, d, CODES[fmt], block, DEV)
        if bad:
            x[0, 0, n, ::3], x[0, 0, n, 1::3], x[0, 0, n, 2::7] = float("nan"), float("inf"), -float("inf")
        p = params(1, 4, 1, n + 70, d, x.stride(), T)
        lrsa.lrsa_cache_append_quant(p, cache, x.to(DEV), x.to(DEV), i32([0]))
        O, lse = lrsa.lrsa_decode_attn_quant(p, q, cache, i32([n + 1]), n + 70)
        K, V, Ks, Vs = host(cache)
        j = n // block
        assert np.all(np.isfinite(ops.values(V[0, 0, :n + 1], Vs[0, 0, :j + 1], block, fmt) / Vs[0, 0, j])) and np.isfinite(Ks[0, 0, j])
        outs.append((O[:, :, :2].clone(), lse[:, :, :2].clone()))
    assert all(torch.equal(a, b) for a, b in zip(*outs))


# ------------------------------------------------------------------------------------------------ attention
def check_attention(p, cache, q, lens, max_len, acc=None, decay=1.0, fmt="int8", dtype="bf16", scale=None):
    B, Hq, T, d = q.shape
    Hkv, cap = cache.K.shape[1:3]
    G = Hq // Hkv
    out = torch.full((B, Hkv, cap), -7.0, device=DEV)
    a = None if acc is None else acc.to(DEV)
    O, lse = lrsa.lrsa_decode_attn_quant(p, q.to(DEV), cache, i32(lens), max_len, a, out, decay)
    O1, lse1 = lrsa.lrsa_decode_attn_quant(p, q.to(DEV), cache, i32(lens), max_len)
    assert torch.equal(O, O1) and torch.equal(lse, lse1)
    O, lse, out = (t.double().cpu().numpy() for t in (O, lse, out))
    K, V, Ks, Vs = host(cache)
    scale = d ** -0.5 if scale is None else scale
    for b in range(B):
        n = max(0, min(lens[b], max_len))
        assert np.all(out[b, :, n:] == -7.0)
        for h in range(Hkv):
            hs = slice(h * G, (h + 1) * G)
            k, v = (ops.values(c[b, h, :n], s[b, h, :-(-n // cache.block)], cache.block, fmt) if n else np.zeros((0, d)) for c, s in ((K, Ks), (V, Vs)))
            qs = q[b, hs].double().numpy()
            O_ref, lse_ref, w = ops.attend(qs, k, v, scale)
            eps = close_attention(O[b, hs], lse[b, hs], qs, k, v, O_ref, lse_ref, scale, 2.0 ** -8 if dtype == "bf16" else 2.0 ** -24)
            want = w if acc is None else decay * acc[b, h, :n].double().numpy() + w
            assert np.all(np.abs(out[b, h, :n] - want) <= 2 * eps * w + 2.0 ** -23 * np.abs(want) + 1e-37)


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)])
@pytest.mark.parametrize("block,G,T,lens", [
    (64, 1, 1, [1, 0, 15, 16]), (16, 4, 1, [17, 31, 32, 33]), (32, 16, 1, [127, 128]), (128, 17, 1, [129, 1000]), (64, 4, 5, [0, 1, 4, 5, 6, 40]),
    (64, 3, 16, [1, 16, 17, 300]), (128, 1, 2, [513, 2500]), (64, 33, 2, [70, 0]),
])
def test_attention(fmt, dtype, d, block, G, T, lens):
    """Lengths around tiles, blocks and slices, sequences without rows, tokens that see none, groups and tokens around the 16 columns
    of a tile; behind the lengths the codes and scales are no numbers."""
    B, Hkv, cap = len(lens), 2, max(lens) + 39
    g = torch.Generator().manual_seed(sum(lens) + G)
    cache, _, _ = make_cache(B, Hkv, cap, d, fmt, block, g, lens)
    q = torch.randn((B, Hkv * G, T, d), generator=g).to(DT[dtype])
    p = params(B, Hkv * G, Hkv, cap, d, (Hkv * cap * d, cap * d, d, 1), DT[dtype])
    check_attention(p, cache, q, lens, max(lens), torch.rand((B, Hkv, cap), generator=g), 0.5, fmt, dtype)


@pytest.mark.parametrize("fmt,dtype,d,B,Hkv,G,T,lens,max_len", [
    ("int8", "bf16", 128, 1, 1, 4, 1, [33000], 33000), ("e4m3", "bf16", 128, 2, 2, 4, 1, [20001, 555], 20011), ("int8", "f32", 64, 1, 2, 8, 3, [9999], 9999),
    ("e4m3", "f32", 128, 3, 4, 2, 2, [4000, 0, 1200], 4100), ("int8", "bf16", 64, 33, 4, 3, 1, [1100 - 7 * i for i in range(33)], 1100),
    ("int8", "bf16", 128, 2, 1, 1, 1, [900, 5000], 1000),                    # a length above the bound counts as the bound
])
def test_attention_over_many_slices(fmt, dtype, d, B, Hkv, G, T, lens, max_len):
    cap = max(*lens, max_len) + 5
    g = torch.Generator().manual_seed(max_len)
    cache, _, _ = make_cache(B, Hkv, cap, d, fmt, 64, g, lens, strided=False)
    # logits that grow along the cache: the slices' maxima differ
    cache.K_scale.mul_(torch.linspace(0.5, 1.5, cache.K_scale.shape[-1], device=DEV))
    q = torch.randn((B, Hkv * G, T, d), generator=g).to(DT[dtype])
    p = params(B, Hkv * G, Hkv, cap, d, (Hkv * cap * d, cap * d, d, 1), DT[dtype], scale=0.11)
    check_attention(p, cache, q, lens, max_len, None, 1.0, fmt, dtype, scale=float(np.float32(0.11)))


def test_attention_with_offsets_beyond_32_bits():
    """Rows a mebibyte apart and sequences more than 4 GiB apart."""
    d, cap, block, T = 128, 4200, 64, torch.bfloat16
    g = torch.Generator(device=DEV).manual_seed(4)
    st = (cap * (1 << 20) + 4096, 256, 1 << 20, 1)
    size = st[0] + (cap - 1) * st[2] + 2 * 256
    K, V = (torch.empty(size, dtype=torch.int8, device=DEV).as_strided((2, 2, cap, d), st) for _ in range(2))
    for t in (K, V):
        t.copy_(torch.randint(-127, 128, (2, 2, cap, d), generator=g, device=DEV, dtype=torch.int8))
    scales = [torch.exp2(torch.randint(-8, -5, (2, 2, -(-cap // block)), generator=g, device=DEV).float()) for _ in range(2)]
    far, near = lrsa.QuantCache(K, V, *scales, block), lrsa.QuantCache(K.contiguous(), V.contiguous(), *(t.clone() for t in scales), block)
    q = torch.randn((2, 4, 1, d), generator=g, device=DEV).to(T)
    p = params(2, 4, 2, cap, d, (2 * cap * d, cap * d, d, 1), T)
    lens = i32([4101, 4150])
    for a, b in zip(lrsa.lrsa_decode_attn_quant(p, q, far, lens, cap), lrsa.lrsa_decode_attn_quant(p, q, near, lens, cap)):
        assert torch.equal(a, b)
    rows = torch.randn((2, 2, 40, d), generator=g, device=DEV).to(T)
    pr = params(2, 4, 2, cap, d, rows.stride(), T)
    for c in (far, near):
        lrsa.lrsa_cache_append_quant(pr, c, rows, rows.neg(), lens)
    assert torch.equal(far.K, near.K) and torch.equal(far.V, near.V)
    for a, b in zip(*(lrsa.lrsa_cache_read_quant(pr, c, lens + 40, 40, lens - 3) for c in (far, near))):
        assert torch.equal(a, b)
    acc = torch.rand((2, 2, cap), generator=g, device=DEV)
    outs = []
    for c in (far, near):
        o, acc_o, lens_o = lrsa.QuantCache.empty(2, 2, cap, d, torch.int8, block, DEV), torch.empty_like(acc), torch.empty_like(lens)
        lrsa.lrsa_cache_evict_quant(p, c, None, acc, lens, cap, 2000, 50, o, None, acc_o, lens_o)
        outs.append((o.K, o.V, o.K_scale, acc_o, lens_o))
    assert all(torch.equal(a, b) for a, b in zip(*outs))


# ------------------------------------------------------------------------------------------------ eviction
@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("d,block,lens,budget,sink,recent,ties", [
    (128, 64, [200, 0, 64, 65, 199], 65, 3, 10, "none"), (64, 16, [100, 33], 40, 0, 0, "few values"), (128, 128, [1000, 300, 301], 300, 5, 100, "all equal"),
    (64, 32, [5000], 1111, 64, 200, "none"), (128, 64, [20000, 9000], 8200, 4, 1000, "signs"), (128, 16, [17], 1, 0, 1, "none"),
])
def test_eviction(fmt, d, block, lens, budget, sink, recent, ties):
    B, Hkv, cap = len(lens), 2, max(max(lens), budget) + 11
    g = torch.Generator().manual_seed(budget)
    cache, _, _ = make_cache(B, Hkv, cap, d, fmt, block, g, lens)
    acc, pos = make_lists(B, Hkv, cap, g, ties)
    out, _, _ = make_cache(B, Hkv, cap, d, fmt, block, g, strided=False)
    stale, before = host(out), host(cache)
    p = params(B, Hkv, Hkv, cap, d, (Hkv * cap * d, cap * d, d, 1), torch.bfloat16, sink=sink)
    ad, pd = acc.to(DEV), pos.to(DEV)
    ao, po, lo = torch.full_like(ad, -3.0), torch.full_like(pd, -3), i32([-3] * B)
    lrsa.lrsa_cache_evict_quant(p, cache, pd, ad, i32(lens), max(lens), budget, recent, out, po, ao, lo)
    assert lo.cpu().tolist() == [min(n, budget) for n in lens]
    assert all(np.array_equal(a, b, equal_nan=True) for a, b in zip(host(cache), before))
    got = host(out)
    for b, n in enumerate(lens):
        new = min(n, budget)
        for h in range(Hkv):
            rows = ops.evict_rows(acc[b, h].double().numpy(), n, sink, recent, budget)
            assert po[b, h, :new].cpu().tolist() == pos[b, h][torch.from_numpy(rows)].tolist() and bool((po[b, h, new:] == -3).all())
            assert torch.equal(ao[b, h, :new].cpu(), acc[b, h][torch.from_numpy(rows)]) and bool((ao[b, h, new:] == 0).all())
            for z in range(2):
                x = ops.values(before[z][b, h], before[2 + z][b, h], block, fmt)[rows]
                codes, scales = ops.evict_blocks(x, block, fmt)
                assert np.array_equal(ops.decode(got[z][b, h, :new], fmt), ops.decode(codes, fmt))      # zero has two codes
                assert np.array_equal(got[2 + z][b, h, :len(scales)].astype(np.float64), scales)
                assert np.array_equal(got[z][b, h, new:], stale[z][b, h, new:]) and np.array_equal(got[2 + z][b, h, len(scales):], stale[2 + z][b, h, len(scales):])


# ------------------------------------------------------------------------------------------------ together
def _generate(steps, use_graph, fmt="int8", T=torch.bfloat16):
    """A prompt, then tokens that are appended, attend and credit rows, and an eviction whenever the longest sequence reaches the limit."""
    B, Hkv, G, d, cap, block, sink, recent, budget = 3, 2, 2, 128, 192, 32, 4, 16, 96
    g = torch.Generator().manual_seed(11)
    prompt, counts = [torch.randn((B, Hkv, 150, d), generator=g).to(T).to(DEV) for _ in range(2)], [150, 90, 1]
    new = [torch.randn((steps, B, Hkv, 1, d), generator=g).to(T).to(DEV) for _ in range(2)]
    q = torch.randn((steps, B, Hkv * G, 1, d), generator=g).to(T).to(DEV)
    caches = [lrsa.QuantCache.empty(B, Hkv, cap, d, CODES[fmt], block, DEV) for _ in range(2)]
    acc, pos = [torch.zeros((B, Hkv, cap), device=DEV) for _ in range(2)], [torch.zeros((B, Hkv, cap), dtype=torch.int32, device=DEV) for _ in range(2)]
    lens = [torch.zeros(B, dtype=torch.int32, device=DEV) for _ in range(2)]
    p0, p1 = (params(B, Hkv * G, Hkv, cap, d, (Hkv * n * d, n * d, d, 1), T, sink=sink) for n in (150, 1))
    lrsa.lrsa_cache_append_quant(p0, caches[0], *prompt, lens[0], i32(counts))
    lens[0].add_(i32(counts))
    pos[0].copy_(torch.arange(cap, dtype=torch.int32, device=DEV).expand(B, Hkv, cap))
    k, v, x, O, lse = torch.empty_like(new[0][0]), torch.empty_like(new[1][0]), torch.empty_like(q[0]), torch.empty_like(q[0]), torch.empty((B, Hkv * G, 1), device=DEV)
    ws = torch.empty(max(lrsa.decode_attn_quant_ws_bytes(p1, 1, cap, True), lrsa.cache_evict_ws_bytes(p1, cap, budget)), dtype=torch.uint8, device=DEV)

    def step(i):
        lrsa.lrsa_cache_append_quant(p1, caches[i], k, v, lens[i])
        lens[i].add_(1)
        lrsa.lrsa_decode_attn_quant(p1, x, caches[i], lens[i], cap, acc[i], acc[i], 1.0, O, lse, ws)

    def evict(i):
        lrsa.lrsa_cache_evict_quant(p1, caches[i], pos[i], acc[i], lens[i], cap, budget, recent, caches[1 - i], pos[1 - i], acc[1 - i], lens[1 - i], ws)

    graphs = None
    if use_graph:
        state = [t.clone() for c in caches for t in (c.K, c.V, c.K_scale, c.V_scale)] + [t.clone() for t in (*acc, *pos, *lens)]
        live = [t for c in caches for t in (c.K, c.V, c.K_scale, c.V_scale)] + [*acc, *pos, *lens]
        for i in range(2):
            step(i), evict(i)                              # everything is loaded before the capture
        torch.cuda.synchronize()
        graphs = {}
        for name, f in (("step", step), ("evict", evict)):
            for i in range(2):
                graphs[name, i] = torch.cuda.CUDAGraph()
                with torch.cuda.graph(graphs[name, i]):
                    f(i)
        for a, b in zip(live, state):
            a.copy_(b)
    at, longest, history = 0, 150, []
    for t in range(steps):
        if longest == cap:
            graphs["evict", at].replay() if use_graph else evict(at)
            at, longest = 1 - at, budget
        k.copy_(new[0][t]), v.copy_(new[1][t]), x.copy_(q[t])
        graphs["step", at].replay() if use_graph else step(at)
        torch.empty(1 << 18, device=DEV).normal_()
        longest += 1
        history.append((O.clone(), lse.clone()))
        if t % 17 == 0:
            torch.cuda.synchronize()
    torch.cuda.synchronize()
    return history, caches[at], acc[at], pos[at], lens[at], (prompt, counts, new, q, (B, Hkv, G, d, cap, block, sink, recent, budget))


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_a_generation_in_eight_bits(fmt):
    """The whole course against the oracle, which replays every append and eviction in codes: attention at every step, then lengths,
    weights and the cache.  (The weights agree to about 1e-6 and the evictions choose among some hundred of them: no close call is near.)"""
    steps = 210
    history, cache, acc, pos, lens, (prompt, counts, new, q, (B, Hkv, G, d, cap, block, sink, recent, budget)) = _generate(steps, False, fmt)
    got = host(cache)
    for b in range(B):
        for h in range(Hkv):
            ref = [(np.zeros((cap, d), np.uint8), np.ones(cap // block)) for _ in range(2)]
            w, n = np.zeros(cap), counts[b]
            for z in range(2):
                ref[z] = ops.append(*ref[z], block, fmt, 0, prompt[z][b, h, :n].double().cpu().numpy())
            longest = max(counts)
            for t in range(steps):
                if longest == cap:
                    rows = ops.evict_rows(w.astype(np.float32), n, sink, recent, budget)
                    for z in range(2):
                        codes, scales = ops.evict_blocks(ops.values(*ref[z], block, fmt)[rows], block, fmt)
                        full = (np.zeros((cap, d), np.uint8), np.ones(cap // block))
                        full[0][:len(codes)], full[1][:len(scales)] = codes, scales
                        ref[z] = full
                    w, n, longest = np.concatenate([w[rows], np.zeros(cap - len(rows))]), len(rows), budget
                for z in range(2):
                    ref[z] = ops.append(*ref[z], block, fmt, n, new[z][t, b, h].double().cpu().numpy())
                n, longest = n + 1, longest + 1
                K, V = (ops.values(*ref[z], block, fmt)[:n] for z in range(2))
                hs = slice(h * G, (h + 1) * G)
                qs = q[t, b, hs].double().cpu().numpy()
                O_ref, lse_ref, w_t = ops.attend(qs, K, V)
                w[:n] += w_t
                O, lse = (x[b, hs].double().cpu().numpy() for x in history[t])
                close_attention(O, lse, qs, K, V, O_ref, lse_ref, d ** -0.5, 2.0 ** -8)
            assert n == int(lens[b])
            for z in range(2):
                have = ops.values(got[z][b, h, :n], got[2 + z][b, h, :-(-n // block)], block, fmt)
                assert np.array_equal(have, ops.values(*ref[z], block, fmt)[:n])
            # sums of up to 210 weights, each as derived, and as many roundings
            assert np.allclose(acc[b, h, :n].double().cpu().numpy(), w[:n], rtol=2.0 ** -15, atol=0) and bool((acc[b, h, n:] == 0).all())


def test_a_generation_replayed_from_graphs_gives_the_same_bits():
    eager, graph = _generate(130, False), _generate(130, True)
    for a, b in zip(eager[0], graph[0]):
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    for a, b in ((eager[1].K, graph[1].K), (eager[1].V, graph[1].V), (eager[2], graph[2]), (eager[3], graph[3]), (eager[4], graph[4])):
        assert torch.equal(a, b)


def test_on_another_stream():
    B, Hkv, G, d, cap = 2, 2, 4, 128, 700
    g = torch.Generator().manual_seed(2)
    cache, _, _ = make_cache(B, Hkv, cap, d, "int8", 64, g)
    q, acc, lens = torch.randn((B, Hkv * G, 1, d), generator=g).to(torch.bfloat16).to(DEV), torch.rand((B, Hkv, cap), generator=g).to(DEV), i32([650, 333])
    p = params(B, Hkv * G, Hkv, cap, d, (Hkv * cap * d, cap * d, d, 1), torch.bfloat16, sink=4)

    def all_calls():
        out = torch.zeros_like(acc)
        O, lse = lrsa.lrsa_decode_attn_quant(p, q, cache, lens, cap, acc, out)
        o, ao, lo = lrsa.QuantCache.empty(B, Hkv, cap, d, torch.int8, 64, DEV), torch.zeros_like(acc), torch.zeros_like(lens)
        lrsa.lrsa_cache_evict_quant(p, cache, None, out, lens, cap, 200, 30, o, None, ao, lo)
        return O, lse, out, o.K, o.V, o.K_scale, ao, lo
    want = all_calls()
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = all_calls()
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))


def test_tensors_elsewhere_are_refused():
    cache = lrsa.QuantCache.empty(1, 1, 64, 64, torch.int8, 16, DEV)
    p = params(1, 1, 1, 64, 64, (64, 64, 64, 1), torch.float32)
    x, lens = torch.zeros((1, 1, 1, 64), device=DEV), i32([0])
    for bad in ((x.cpu(), x.cpu(), lens), (x, x.cpu(), lens), (x, x, lens.cpu()), (x, x, lens.long()), (x, x.to(torch.bfloat16), lens), (x, x, i32([0, 0]))):
        with pytest.raises(ValueError):
            lrsa.lrsa_cache_append_quant(p, cache, *bad)
    with pytest.raises(ValueError):
        lrsa.lrsa_decode_attn_quant(params(1, 1, 1, 65, 64, (64, 64, 64, 1), torch.float32), x, cache, lens, 64)
