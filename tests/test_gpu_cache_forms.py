"""The inference-cache calls in forms that other tests leave out: 17 to 32 columns over caches larger than the GPU's, weights that are followed through
evictions, all calls captured without a workspace.
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


@pytest.mark.parametrize("dtype,d,decay", [("bf16", 64, 1.0), ("f32", 128, 1.0), ("bf16", 128, 0.9)])
def test_weights_through_evictions(dtype, d, decay):
    """Tokens are appended, attend and credit the rows in place; the lightest rows go whenever the cache is full.  Beside it the weights
    are added up in 64 bits for every row that is kept.  A step's weight is off by at most 2 eps of itself (see test_gpu_cache_weights.py),
    and each sum by a rounding: the bounds are added up alike.  The choice of the rows is the oracle's from the device's weights."""
    B, Hkv, G, cap, sink, recent, budget, n, T = 2, 2, 3, 80, 3, 10, 40, 190, DT[dtype]
    g = torch.Generator().manual_seed(d)
    K, V = (torch.randn((B, Hkv, n, d), generator=g).to(T).to(DEV) for _ in range(2))
    q = torch.randn((n, B, Hkv * G, d), generator=g).to(T).to(DEV)
    caches = [[torch.zeros((B, Hkv, cap, d), dtype=T, device=DEV) for _ in range(2)] + [torch.zeros((B, Hkv, cap), dtype=torch.int32, device=DEV),
               torch.zeros((B, Hkv, cap), device=DEV)] for _ in range(2)]
    p = params(B, Hkv * G, Hkv, cap, d, caches[0][0].stride(), T, sink=sink)
    K64, V64, q64 = (x.double().cpu().numpy() for x in (K, V, q))
    units = [(b, h) for b in range(B) for h in range(Hkv)]
    kept = {u: np.zeros(0, np.int64) for u in units}             # tokens whose rows are there, their weights and how far these may be off
    sums, off = {u: np.zeros(0) for u in units}, {u: np.zeros(0) for u in units}
    length, evictions = 0, 0
    for t in range(n):
        Kc, Vc, pos, acc = caches[0]
        if length == cap:
            old = acc.double().cpu().numpy()
            Ko, Vo, po, ao = caches[1]
            length = lrsa.lrsa_cache_evict(p, Kc, Vc, pos, acc, length, budget, recent, Ko, Vo, po, ao)
            for b, h in units:
                rows = ops.evict_rows(old[b, h], cap, sink, recent, budget)
                kept[b, h], sums[b, h], off[b, h] = kept[b, h][rows], sums[b, h][rows], off[b, h][rows]
                assert np.array_equal(po[b, h, :length].cpu().numpy(), kept[b, h]) and bool((ao[b, h, length:] == 0).all())
            caches.reverse()
            Kc, Vc, pos, acc = caches[0]
            evictions += 1
        Kc[:, :, length], Vc[:, :, length], pos[:, :, length] = K[:, :, t], V[:, :, t], t
        length += 1
        lrsa.lrsa_decode_attn_acc(p, q[t], Kc, Vc, length, acc, acc, decay)
        got = acc.double().cpu().numpy()
        for b, h in units:
            rows = kept[b, h] = np.append(kept[b, h], t)
            qs = q64[t, b, h * G:(h + 1) * G][:, None]
            _, _, w = ops.attend(qs, K64[b, h, rows], V64[b, h, rows])
            eps = 2.0 ** -20 * max(8.0, d ** -0.5 * (np.abs(qs[:, 0]) @ np.abs(K64[b, h, rows]).T).max())
            f = float(np.float32(decay))
            sums[b, h] = f * np.append(sums[b, h], 0.0) + w
            off[b, h] = f * np.append(off[b, h], 0.0) + 2 * eps * w + 2.0 ** -23 * sums[b, h]
            assert np.all(np.abs(got[b, h, :length] - sums[b, h]) <= off[b, h] + 1e-37) and np.all(got[b, h, length:] == 0)
    assert evictions >= 3 and max((o / s).max() for o, s in zip(off.values(), sums.values())) < 2.0 ** -10


def test_captured_without_a_workspace():
    """All calls in one graph, outputs and workspaces allocated while it is captured; replayed with other inputs and eager work between."""
    B, Hkv, G, d, cap, n, T = 2, 2, 4, 128, 2200, 2050, torch.bfloat16
    g = torch.Generator(device=DEV).manual_seed(3)
    K, V, q = (torch.empty(s, dtype=T, device=DEV) for s in ((B, Hkv, cap, d), (B, Hkv, cap, d), (B, Hkv * G, d)))
    new, lens = [torch.empty((B, Hkv, 1500, d), dtype=T, device=DEV) for _ in range(2)], i32([0, 0])
    cache, other = (lrsa.QuantCache.empty(B, Hkv, cap, d, torch.int8, 64, DEV) for _ in range(2))
    Ko, Vo, acc, ao, aq, lo = torch.zeros_like(K), torch.zeros_like(V), *(torch.zeros((B, Hkv, cap), device=DEV) for _ in range(3)), i32([0, 0])
    p = params(B, Hkv * G, Hkv, cap, d, K.stride(), T, sink=4)
    pn = params(B, Hkv * G, Hkv, cap, d, new[0].stride(), T, sink=4)

    def calls():
        O, lse, _ = lrsa.lrsa_decode_attn_acc(p, q, K, V, n, None, acc)
        lrsa.lrsa_cache_evict(p, K, V, None, acc, n, 700, 50, Ko, Vo, None, ao)
        lrsa.lrsa_cache_append_quant(pn, cache, *new, lens)
        end = lens + 1500
        Oq, lseq = lrsa.lrsa_decode_attn_quant(pn, q, cache, end, cap, None, aq)
        lrsa.lrsa_cache_evict_quant(pn, cache, None, aq, end, cap, 600, 50, other, None, ao, lo)
        Kr, Vr = lrsa.lrsa_cache_read_quant(pn, other, lo, 600)
        return [O, lse, Oq, lseq, Kr, Vr, acc, aq, Ko[:, :, :700], Vo[:, :, :700], lo]

    def fill(k):
        g.manual_seed(k)
        for t in (K, V, q, *new):
            t.copy_(torch.randn(t.shape, generator=g, device=DEV))
        lens.copy_(i32([k, 600]))
        for t in (cache.K, cache.V, other.K, other.V, cache.K_scale, cache.V_scale):
            t.zero_()
        for t in (acc, aq, Ko, Vo):
            t.zero_()
    fill(0)
    calls()                                                      # everything is loaded before the capture
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = calls()
    for k in (1, 17, 300):
        fill(k)
        want = [t.clone() for t in calls()]
        fill(k)
        junk = [torch.empty(1 << 22, device=DEV).normal_() for _ in range(4)]
        graph.replay()
        got = [t.clone() for t in out]
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, got)), k
        del junk
