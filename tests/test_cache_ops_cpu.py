"""The oracle of the cache calls pinned to independent statements, and what the C ABI refuses before any GPU work: no GPU needed."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2506_11498_amd as lrsa
from paper_2506_11498_amd import binding
from oracle import lrsa_cache_ops as ops


def test_e4m3_codes_are_those_of_torch():
    codes = torch.arange(256, dtype=torch.uint8)
    want = codes.view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(ops.E4M3, want, equal_nan=True)
    # every number of 16 bits in range, ties among them
    x = torch.arange(-32768, 32768, dtype=torch.int16).view(torch.bfloat16)
    x = x[x.float().abs() <= 448]
    assert np.array_equal(ops.encode(x.double().numpy(), "e4m3"), x.float().to(torch.float8_e4m3fn).view(torch.uint8).numpy())
    mid = (ops.E4M3[:126] + ops.E4M3[1:127]) / 2
    assert np.array_equal(ops.encode(mid, "e4m3") % 2, np.zeros(126))
    assert np.array_equal(ops.encode(np.array([0.5, 1.5, 2.5, -0.5, 127, -127]), "int8").view(np.int8), [0, 2, 2, 0, 127, -127])


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_scales_are_the_least_powers_of_two(fmt):
    for top in (0.0, 1e-40, 2.0 ** -113, 1.0, 126.99, 127.0, 127.5, 447.9, 448.0, 449.0, 3e38):
        s = ops.scale_for(top, fmt)
        assert np.log2(s) == np.rint(np.log2(s)) and top <= ops.TOP[fmt] * s
        assert s == 2.0 ** -120 or top > ops.TOP[fmt] * s / 2


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_appending_one_by_one_keeps_every_value_within_its_step(fmt):
    """Rows that come one by one end with the scale of all rows at once, and every value is off by at most the half steps of the scales
    that its block has had (a block's scale doubles at least each time it grows: their sum is below twice the last one's)."""
    g = np.random.default_rng(1)
    x = g.standard_normal((40, 64)) * np.exp2(np.linspace(-6, 3, 40))[:, None]
    codes, scales = np.zeros((64, 64), np.uint8), np.ones(4)
    for t in range(40):
        codes, scales = ops.append(codes, scales, 16, fmt, t, x[t:t + 1])
    whole, at_once = ops.append(np.zeros((64, 64), np.uint8), np.ones(4), 16, fmt, 0, x)
    assert np.array_equal(scales, at_once)
    step = np.repeat(scales, 16)[:40, None] * (1.0 if fmt == "int8" else 2.0 ** -9)
    rel = 0.0 if fmt == "int8" else 2.0 ** -4
    for c, times in ((codes, 2), (whole, 1)):
        assert np.all(np.abs(ops.values(c, scales, 16, fmt)[:40] - x) <= times * (step / 2 + rel * np.abs(x)))


def test_attention_and_eviction_oracles():
    g = np.random.default_rng(2)
    q, K, V = g.standard_normal((3, 4, 64)), g.standard_normal((9, 64)), g.standard_normal((9, 64))
    O, lse, w = ops.attend(q, K, V)
    Q = torch.from_numpy(q)
    mask = torch.ones(4, 9, dtype=torch.bool).tril(5)
    ref = torch.nn.functional.scaled_dot_product_attention(Q, torch.from_numpy(K).expand(3, 9, 64), torch.from_numpy(V).expand(3, 9, 64), attn_mask=mask)
    assert np.allclose(O, ref.numpy(), atol=1e-12) and abs(w.sum() - 12) < 1e-12
    O, lse, w = ops.attend(q, K[:2], V[:2])          # the first two of four tokens see nothing
    assert np.all(O[:, :2] == 0) and np.all(np.isneginf(lse[:, :2])) and abs(w.sum() - 6) < 1e-12
    assert ops.evict_rows(np.array([9, 0, 5, 1, 5, 5, 0, 0]), 8, 1, 2, 5).tolist() == [0, 2, 4, 6, 7]
    assert ops.evict_rows(np.zeros(8), 8, 0, 0, 3).tolist() == [0, 1, 2] and ops.evict_rows(np.zeros(8), 3, 1, 1, 4).tolist() == [0, 1, 2]


# ------------------------------------------------------------------------------------------------ refusals
FAKE = ctypes.c_void_p(1 << 16)        # never dereferenced
FAKE2, FAKE3, FAKE4 = (ctypes.c_void_p((1 << 16) * i) for i in (2, 3, 4))
ODD = ctypes.c_void_p((1 << 16) + 8)


def _p(B=2, Hq=4, Hkv=2, cap=100, d=128, sink=4, dtype=torch.bfloat16):
    return lrsa.make_params((B, Hq, cap, d), (B, Hkv, cap, d), (Hq * cap * d, cap * d, d, 1), (Hkv * cap * d, cap * d, d, 1), dtype=dtype, sink=sink,
                            lag=16, topk=4)


def _c(K=FAKE, V=FAKE2, Ks=FAKE3, Vs=FAKE4, fmt=0, block=64, stride=(25600, 12800, 128)):
    v = lambda x: x.value if x is not None else None
    return binding.LrsaQuantCache(fmt, block, (ctypes.c_int64 * 3)(*stride), v(K), v(V), v(Ks), v(Vs))


def _refused(rc, code, text):
    assert rc == code and text in lrsa.lib().lrsa_last_error().decode(), (rc, lrsa.lib().lrsa_last_error())


def test_decode_attn_acc_refuses():
    L, p = lrsa.lib(), _p()
    nan, need = float("nan"), lrsa.decode_attn_acc_ws_bytes(p, 100)
    r = ctypes.byref(p)

    def call(q=FAKE, K=FAKE, V=FAKE, length=100, a=FAKE, b=FAKE, decay=1.0, O=FAKE, ws=FAKE, nb=need):
        return L.lrsa_decode_attn_acc(r, q, K, V, length, a, b, decay, O, None, ws, nb, None)
    for kw in (dict(q=None), dict(K=None), dict(V=None), dict(b=None), dict(O=None), dict(a=None, b=None)):
        _refused(call(**kw), -1, "NULL")
    for n in (0, -1, 101):
        _refused(call(length=n), -1, "outside")
        assert lrsa.decode_attn_acc_ws_bytes(p, n) == 0
    for d in (nan, float("inf")):
        _refused(call(decay=d), -1, "decay")
    _refused(call(q=ODD), -1, "aligned")
    for kw in (dict(ws=None), dict(nb=need - 1), dict(ws=ctypes.c_void_p((1 << 16) + 64))):
        _refused(call(**kw), -1, "workspace")


def test_cache_evict_refuses():
    L, p = lrsa.lib(), _p()
    r, out, need = ctypes.byref(p), ctypes.c_int32(-7), lrsa.cache_evict_ws_bytes(p, 100, 50)
    assert need >= 2 * 2 * 50 * 4

    def call(K=FAKE, V=FAKE, pos=FAKE, acc=FAKE, length=100, budget=50, recent=10, Ko=FAKE2, Vo=FAKE3, pos_o=FAKE2, acc_o=FAKE2, n=out, ws=FAKE, nb=need):
        return L.lrsa_cache_evict(r, K, V, pos, acc, length, budget, recent, Ko, Vo, pos_o, acc_o, ctypes.byref(n) if n else None, ws, nb, None)
    for kw in (dict(K=None), dict(V=None), dict(Ko=None), dict(Vo=None), dict(acc=None), dict(acc_o=None), dict(n=None)):
        _refused(call(**kw), -1, "NULL")
    for kw in (dict(pos=None), dict(pos_o=None)):
        _refused(call(**kw), -1, "go together")
    for kw in (dict(length=-1), dict(length=101)):
        _refused(call(**kw), -1, "outside")
    for kw in (dict(budget=0, recent=0), dict(budget=101), dict(recent=-1), dict(budget=13, recent=10), dict(recent=2 ** 31 - 1)):
        _refused(call(**kw), -1, "budget")
    for kw in (dict(Ko=FAKE), dict(Vo=FAKE), dict(Ko=FAKE3)):
        _refused(call(**kw), -1, "must not be the old one")
    for kw in (dict(pos_o=FAKE), dict(acc_o=FAKE)):
        _refused(call(**kw), -1, "lists")
    _refused(call(Ko=ODD), -1, "aligned")
    for kw in (dict(ws=None), dict(nb=need - 1), dict(ws=ctypes.c_void_p((1 << 16) + 64))):
        _refused(call(**kw), -1, "workspace")
    assert out.value == -7


def test_quant_calls_refuse():
    L, p = lrsa.lib(), _p()
    r = ctypes.byref(p)

    def each(c, code, text):
        ref = ctypes.byref(c) if c is not None else None
        _refused(L.lrsa_cache_append_quant(r, ref, FAKE, FAKE, 1, FAKE, None, None), code, text)
        _refused(L.lrsa_cache_read_quant(r, ref, FAKE, 1, None, FAKE, FAKE, None), code, text)
        _refused(L.lrsa_decode_attn_quant(r, ref, FAKE, 1, FAKE, 100, None, None, 1.0, FAKE, None, FAKE, 1 << 30, None), code, text)
        good = _c(FAKE4, FAKE3, FAKE2, FAKE)
        _refused(L.lrsa_cache_evict_quant(r, ref, None, FAKE, FAKE, 100, 50, 1, ctypes.byref(good), None, FAKE2, FAKE2, FAKE, 1 << 30, None), code, text)
        _refused(L.lrsa_cache_evict_quant(r, ctypes.byref(good), None, FAKE, FAKE, 100, 50, 1, ref, None, FAKE2, FAKE2, FAKE, 1 << 30, None), code, text)
    each(None, -1, "NULL")
    for kw in (dict(K=None), dict(V=None), dict(Ks=None), dict(Vs=None)):
        each(_c(**kw), -1, "NULL")
    each(_c(fmt=2), -2, "format")
    for b in (0, 8, 48, 256, -64):
        each(_c(block=b), -2, "blocks")
    each(_c(K=ODD), -1, "16-byte")
    each(_c(Vs=ctypes.c_void_p((1 << 16) + 2)), -1, "4-byte")
    for st in ((25600, 12800, 64), (25600, 12800, 136), (25608, 12800, 128), (-25600, 12800, 128)):
        each(_c(stride=st), -1, "stride")
    each(_c(stride=(1 << 34, 128, 1 << 24)), -2, "apart")

    c = ctypes.byref(_c())
    for kw in ((None, FAKE, 1, FAKE), (FAKE, None, 1, FAKE), (FAKE, FAKE, 1, None)):
        _refused(L.lrsa_cache_append_quant(r, c, *kw, None, None), -1, "NULL")
    _refused(L.lrsa_cache_append_quant(r, c, FAKE, FAKE, 0, FAKE, None, None), -1, "tokens")
    _refused(L.lrsa_cache_append_quant(r, c, ODD, FAKE, 1, FAKE, None, None), -1, "aligned")
    for kw in ((None, 1, None, FAKE, FAKE), (FAKE, 1, None, None, FAKE), (FAKE, 1, None, FAKE, None)):
        _refused(L.lrsa_cache_read_quant(r, c, *kw, None), -1, "NULL")
    _refused(L.lrsa_cache_read_quant(r, c, FAKE, 0, None, FAKE, FAKE, None), -1, "rows")

    need = lrsa.decode_attn_quant_ws_bytes(p, 3, 100, True)

    def attend(q=FAKE, tokens=3, lens=FAKE, most=100, a=FAKE, b=FAKE, decay=1.0, O=FAKE, ws=FAKE, nb=need):
        return L.lrsa_decode_attn_quant(r, c, q, tokens, lens, most, a, b, decay, O, None, ws, nb, None)
    for kw in (dict(q=None), dict(lens=None), dict(O=None)):
        _refused(attend(**kw), -1, "NULL")
    for t in (0, 17, -1):
        _refused(attend(tokens=t), -1, "tokens")
    for m in (0, 101):
        _refused(attend(most=m), -1, "max_len")
    _refused(attend(b=None), -1, "acc_in without acc_out")
    _refused(attend(decay=float("nan")), -1, "decay")
    _refused(attend(q=ODD), -1, "aligned")
    for kw in (dict(ws=None), dict(nb=need - 1), dict(ws=ctypes.c_void_p((1 << 16) + 64))):
        _refused(attend(**kw), -1, "workspace")

    def evict(o=_c(FAKE4, FAKE3, FAKE2, FAKE), pos=None, acc=FAKE, lens=FAKE, most=100, budget=50, recent=5, pos_o=None, acc_o=FAKE2, lens_o=FAKE2, ws=FAKE,
              nb=1 << 30):
        return L.lrsa_cache_evict_quant(r, c, pos, acc, lens, most, budget, recent, ctypes.byref(o), pos_o, acc_o, lens_o, ws, nb, None)
    for kw in (dict(acc=None), dict(acc_o=None)):
        _refused(evict(**kw), -1, "NULL")
    for kw in (dict(lens=None), dict(lens_o=None), dict(lens_o=FAKE)):
        _refused(evict(**kw), -1, "two arrays")
    _refused(evict(o=_c(FAKE4, FAKE3, FAKE2, FAKE, block=32)), -1, "format and block")
    _refused(evict(o=_c(FAKE4, FAKE3, FAKE2, FAKE, fmt=1)), -1, "format and block")
    for o in (_c(), _c(V=FAKE3), _c(FAKE2, FAKE3), _c(FAKE4, FAKE3, FAKE3, FAKE), _c(FAKE4, FAKE3, FAKE, FAKE4)):
        _refused(evict(o=o), -1, "must not be the old one")
    _refused(evict(pos=FAKE), -1, "go together")
    _refused(evict(acc_o=FAKE), -1, "lists")
    _refused(evict(budget=8), -1, "budget")
    _refused(evict(most=101), -1, "outside")
    _refused(evict(nb=16), -1, "workspace")


def test_rows_that_are_written_must_not_be_shared():
    """Broadcast caches may be read, not written; K and V of a cache that is written are two."""
    L, p = lrsa.lib(), _p()
    r, out = ctypes.byref(p), ctypes.c_int32(-7)
    shared = _p()
    good = ctypes.byref(_c())
    for st in ((0, 12800, 128), (25600, 0, 128)):
        c = ctypes.byref(_c(stride=st))
        _refused(L.lrsa_cache_append_quant(r, c, FAKE, FAKE, 1, FAKE, None, None), -1, "share")
        c = ctypes.byref(_c(FAKE4, FAKE3, FAKE2, FAKE, stride=st))
        _refused(L.lrsa_cache_evict_quant(r, good, None, FAKE, FAKE, 100, 50, 1, c, None, FAKE2, FAKE2, FAKE, 1 << 30, None), -1, "share")
        shared.kv_stride[:] = st
        s = ctypes.byref(shared)
        _refused(L.lrsa_cache_read_quant(s, good, FAKE, 1, None, FAKE, FAKE2, None), -1, "share")
        _refused(L.lrsa_cache_evict(s, FAKE, FAKE, None, FAKE, 100, 50, 10, FAKE2, FAKE3, None, FAKE2, ctypes.byref(out), FAKE, 1 << 30, None), -1, "share")
    _refused(L.lrsa_cache_append_quant(r, ctypes.byref(_c(V=FAKE)), FAKE, FAKE, 1, FAKE, None, None), -1, "must be two")
    _refused(L.lrsa_cache_append_quant(r, ctypes.byref(_c(Vs=FAKE3)), FAKE, FAKE, 1, FAKE, None, None), -1, "must be two")
    _refused(L.lrsa_cache_read_quant(r, good, FAKE, 1, None, FAKE, FAKE, None), -1, "must be two")
    assert out.value == -7


def test_workspaces_for_a_longer_cache_are_enough_for_a_shorter_one():
    for kw in (dict(B=1, Hq=12, Hkv=2), dict(B=16, Hq=32, Hkv=8), dict(B=1, Hq=1, Hkv=1), dict(B=20, Hq=64, Hkv=8, dtype=torch.float32), dict(B=8, Hq=32, Hkv=8, d=64)):
        p = _p(cap=50000, **kw)
        for f in (lambda n: lrsa.decode_attn_acc_ws_bytes(p, n), lambda n: lrsa.decode_attn_quant_ws_bytes(p, 5, n, False),
                  lambda n: lrsa.decode_attn_quant_ws_bytes(p, 1, n, True)):
            sizes = [f(n) for n in list(range(1, 3000, 37)) + list(range(3000, 50001, 1237))]
            assert all(a <= b for a, b in zip(sizes, sizes[1:])) and sizes[0] > 0


def test_the_binding_refuses_other_layouts():
    codes = lambda dt=torch.int8, cap=64: torch.zeros((2, 2, cap, 128), dtype=torch.uint8).view(dt)
    scales = lambda n=1: torch.ones((2, 2, n))
    c = lrsa.QuantCache(codes(), codes(), scales(), scales(), 64)
    assert (c.struct.format, c.struct.block, list(c.struct.stride)) == (0, 64, [2 * 64 * 128, 64 * 128, 128]) and ctypes.sizeof(c.struct) == 64
    assert lrsa.QuantCache.empty(2, 2, 65, 64, torch.float8_e4m3fn, 16, "cpu").K_scale.shape == (2, 2, 5)
    for bad in ((codes(torch.uint8), codes(torch.uint8), scales(), scales(), 64), (codes(), codes(torch.float8_e4m3fn), scales(), scales(), 64),
                (codes(), codes(), scales(2), scales(), 64), (codes(), codes(), scales(), scales().double(), 64), (codes(), codes(), scales(), scales(), 48),
                (codes().transpose(2, 3), codes().transpose(2, 3), scales(), scales(), 64), (codes(), codes(cap=32), scales(), scales(), 64)):
        with pytest.raises(ValueError):
            lrsa.QuantCache(*bad)
    p = _p(cap=64)
    with pytest.raises((ValueError, RuntimeError, AssertionError)):       # tensors of the CPU
        lrsa.lrsa_cache_append_quant(p, c, torch.zeros((2, 2, 1, 128), dtype=torch.bfloat16), torch.zeros((2, 2, 1, 128), dtype=torch.bfloat16), torch.zeros(2, dtype=torch.int32))


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_the_largest_values_are_finite_and_the_nearest_there_are(fmt):
    """At the end of the range: the codes of the largest scale whose values are numbers of 32 bits and of bf16, the nearest one of them each."""
    big, scale = ops.LARGEST[fmt], 2.0 ** (121 if fmt == "int8" else 120)
    assert big == float(np.float32(big)) == float(torch.tensor(big).bfloat16()) and ops.scale_for(3.4028234663852886e38, fmt) == scale
    numbers = np.array([v * scale for v in ops.decode(np.arange(256, dtype=np.uint8), fmt) if abs(v * scale) <= big])
    x = np.linspace(0.95 * 2.0 ** 127, 3.4028234663852886e38, 640).reshape(10, 64) * np.where(np.arange(64) % 3, 1, -1)
    codes, scales = ops.append(np.zeros((16, 64), np.uint8), np.ones(1), 16, fmt, 0, x)
    got = ops.values(codes, scales, 16, fmt)[:10]
    assert np.array_equal(np.abs(got - x), np.abs(x[..., None] - numbers).min(-1)) and scales[0] == scale and np.abs(got).max() == big


def test_rows_that_overlap_by_their_strides_are_not_written():
    """Strides that were made for fewer rows, or heads less than a row apart; layouts whose axes come in another order are written."""
    L, p = lrsa.lib(), _p()
    r, out = ctypes.byref(p), ctypes.c_int32(-7)
    good, other = ctypes.byref(_c()), _p()

    def read(rows, st):
        other.kv_stride[:] = st
        return L.lrsa_cache_read_quant(ctypes.byref(other), good, FAKE, rows, None, FAKE, FAKE2, None)

    def evict(st, budget=50):
        other.kv_stride[:] = st
        return L.lrsa_cache_evict(ctypes.byref(other), FAKE, FAKE, None, FAKE, 100, budget, 10, FAKE2, FAKE3, None, FAKE2, ctypes.byref(out), FAKE, 16, None)
    # one row per head, taken for a call of more (the second head's first row is the first one's second)
    for rows, st in ((2, (256, 128, 128)), (64, (256, 128, 128)), (9, (2048, 1024, 128)), (2, (128, 1024, 128)), (5, (512, 128, 256)), (3, (1024, 8, 128)),
                     (3, (128, 4096, 248))):
        _refused(read(rows, st), -1, "share")
    for st in ((12800, 6272, 128), (6400, 6400, 128), (12672, 128, 256), (25600, 64, 128)):
        _refused(evict(st), -1, "share")
        _refused(L.lrsa_cache_append_quant(r, ctypes.byref(_c(stride=st)), FAKE, FAKE, 1, FAKE, None, None), -1, "share")
        _refused(L.lrsa_cache_evict_quant(r, good, None, FAKE, FAKE, 100, 50, 1, ctypes.byref(_c(FAKE4, FAKE3, FAKE2, FAKE, stride=st)), None, FAKE2, FAKE2, FAKE,
                                          1 << 30, None), -1, "share")
    # layouts that are: refused for another reason, which is looked for later
    for st in ((50 * 256, 128, 256), (50 * 128, 50 * 256, 128), (128, 50 * 256, 256), (128, 256, 512), (2 ** 50, 2 ** 40, 2 ** 20), (2 ** 60, 128, 2 ** 50)):
        _refused(evict(st), -1, "workspace")
    for st in ((2 ** 50, 2 ** 42, 128), (128, 256, 512), (2 ** 60, 128, 256), (128, 2 ** 42, 264)):
        _refused(read(2 ** 31 - 1, st), -2, "grid")
    # axes of length one have any stride
    other = _p(B=1, Hkv=1)
    _refused(read(2 ** 31 - 1, (0, 0, 128)), -2, "grid")
    _refused(evict((0, 8, 128)), -1, "workspace")
    assert out.value == -7
