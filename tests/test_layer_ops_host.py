"""The operators around the projections, without a GPU: refusals, the page size, the argument conversion, and the oracle itself
against hand-made values."""
import ctypes

import numpy as np
import pytest

from oracle import layer_ops as O
from paper_2607_21985_b200 import build, spdp

F, ODD = 1 << 20, (1 << 20) + 1          # addresses that are never touched: every call here is refused first
INVALID, SHAPE = spdp.SPDP_ERR_INVALID_ARG, spdp.SPDP_ERR_UNSUPPORTED_SHAPE


@pytest.fixture(scope="module")
def L():
    build.build()
    return spdp.lib()


LORA = dict(X=F, N=4, K=64, ldx=64, adapter=F, A=F, lda=64, stride_a=512, B=F, ldb=8, stride_b=768, count=3, rank=8, ranks=F, scales=F, base=F, ldbase=96,
            Y=2 * F, M=96, ldy=96, ydt=0, stream=None)


@pytest.mark.parametrize("change,status", [
    (dict(X=None), INVALID), (dict(adapter=None), INVALID), (dict(A=None), INVALID), (dict(B=None), INVALID), (dict(base=None), INVALID), (dict(Y=None), INVALID),
    (dict(N=0), INVALID), (dict(N=(1 << 24) + 1), INVALID), (dict(K=0), SHAPE), (dict(M=0), SHAPE), (dict(rank=0), SHAPE), (dict(rank=257, ldb=300), SHAPE),
    (dict(count=0), INVALID), (dict(ldx=63), INVALID), (dict(lda=63), INVALID), (dict(ldb=7), INVALID), (dict(ldbase=95), INVALID), (dict(ldy=95), INVALID),
    (dict(stride_a=511), INVALID), (dict(stride_b=767), INVALID), (dict(ldx=1 << 50), INVALID), (dict(ydt=2), INVALID), (dict(base=2 * F, ldbase=97), INVALID),
    (dict(X=ODD), INVALID), (dict(A=ODD), INVALID), (dict(B=ODD), INVALID), (dict(Y=ODD), INVALID), (dict(ydt=1, base=F + 2), INVALID), (dict(adapter=F + 2), INVALID),
    (dict(ranks=F + 1), INVALID), (dict(scales=F + 2), INVALID)])
def test_lora_refuses(L, change, status):
    assert L.spdp_lora(*dict(LORA, **change).values()) == status


HEADS = dict(q=F, ldq=512, k=F, ldk=256, dt=0, N=3, q_heads=4, kv_heads=2, dim=128, qw=F, kw=F, eps=1e-6, pos=F, pos_stride=3, axes=2, sections=(40, 24), freq=F,
             pairs=64, adjacent=0, q_out=2 * F, ldq_out=512, k_out=2 * F, ldk_out=256, stream=None)


@pytest.mark.parametrize("change,status", [
    (dict(dim=127), SHAPE), (dict(dim=0), SHAPE), (dict(dim=258), SHAPE), (dict(q_heads=1 << 17), SHAPE), (dict(N=0), INVALID), (dict(N=(1 << 24) + 1), INVALID),
    (dict(q_heads=-1), INVALID), (dict(kv_heads=-1), INVALID), (dict(q_heads=0, kv_heads=0), INVALID), (dict(dt=2), INVALID), (dict(pairs=65), INVALID),
    (dict(pairs=-1), INVALID), (dict(adjacent=2), INVALID), (dict(eps=-1.0), INVALID), (dict(eps=float("nan")), INVALID), (dict(q=None), INVALID), (dict(k=None), INVALID),
    (dict(q_out=None), INVALID), (dict(k_out=None), INVALID), (dict(ldq=511), INVALID), (dict(ldk=255), INVALID), (dict(ldq_out=511), INVALID),
    (dict(ldk_out=255), INVALID), (dict(q=ODD), INVALID), (dict(dt=1, q=F + 2), INVALID), (dict(qw=ODD), INVALID), (dict(kw=ODD), INVALID),
    (dict(q_out=F, ldq_out=513), INVALID), (dict(dt=1, q_out=F), INVALID), (dict(k_out=F, ldk_out=300), INVALID), (dict(pos=None), INVALID),
    (dict(pos=F + 2), INVALID), (dict(pos_stride=2), INVALID), (dict(axes=0), INVALID), (dict(axes=5), INVALID), (dict(sections=None), INVALID),
    (dict(sections=(40, 25)), INVALID), (dict(sections=(65, -1)), INVALID), (dict(freq=None), INVALID), (dict(freq=F + 2), INVALID)])
def test_qk_norm_rope_refuses(L, change, status):
    a = dict(HEADS, **change)
    if a["sections"] is not None:
        a["sections"] = (ctypes.c_int * 8)(*a["sections"], 0, 0, 0)
    assert L.spdp_qk_norm_rope(*a.values()) == status


STORE = dict(k=F, ldk=256, v=F, ldv=256, vdt=0, N=3, heads=2, dim=128, slot=F, cache=F, pages=5, page=16, ko=F, ldko=256, vo=F, ldvo=256, stream=None)


@pytest.mark.parametrize("change,status", [
    (dict(k=None), INVALID), (dict(v=None), INVALID), (dict(slot=None), INVALID), (dict(cache=None), INVALID), (dict(heads=0), SHAPE), (dict(heads=4097), SHAPE),
    (dict(dim=96), SHAPE), (dict(page=8), SHAPE), (dict(page=24), SHAPE), (dict(page=512), SHAPE), (dict(N=0), INVALID), (dict(pages=0), INVALID),
    (dict(ldk=255), INVALID), (dict(ldv=255), INVALID), (dict(vdt=3), INVALID), (dict(ldko=255), INVALID), (dict(ldvo=255), INVALID), (dict(k=ODD), INVALID),
    (dict(vdt=1, v=F + 2), INVALID), (dict(slot=F + 4), INVALID), (dict(cache=F + 8), INVALID), (dict(ko=ODD), INVALID), (dict(vo=ODD), INVALID)])
def test_kv4_store_refuses(L, change, status):
    assert L.spdp_kv4_store(*dict(STORE, **change).values()) == status


ATTN = dict(q=F, ldq=1024, B=2, q_heads=8, kv_heads=2, dim=128, cache=F, pages=9, page=16, table=F, table_stride=4, table_pages=4, length=F, scale=0.1, cap=0.0,
            window=0, thr=0.0, y=2 * F, ldy=1024, mask=F, mask_stride=32, stream=None)


@pytest.mark.parametrize("change,status", [
    (dict(q=None), INVALID), (dict(cache=None), INVALID), (dict(table=None), INVALID), (dict(length=None), INVALID), (dict(y=None), INVALID),
    (dict(q_heads=7), SHAPE), (dict(q_heads=0), SHAPE), (dict(kv_heads=0), SHAPE), (dict(dim=32), SHAPE), (dict(page=20), SHAPE), (dict(B=0), SHAPE), (dict(B=4097), SHAPE),
    (dict(pages=0), INVALID), (dict(table_pages=0), INVALID), (dict(table_stride=3), INVALID), (dict(ldq=1023), INVALID), (dict(ldy=1023), INVALID),
    (dict(window=-1), INVALID), (dict(mask_stride=31), INVALID), (dict(scale=float("inf")), INVALID), (dict(scale=float("nan")), INVALID), (dict(cap=-1.0), INVALID),
    (dict(cap=float("nan")), INVALID), (dict(q=ODD), INVALID), (dict(cache=F + 8), INVALID), (dict(table=F + 2), INVALID), (dict(length=F + 1), INVALID),
    (dict(y=ODD), INVALID), (dict(mask=F + 2), INVALID), (dict(table_pages=1 << 27, table_stride=1 << 27), SHAPE),
    (dict(B=4096, table_pages=1 << 22, table_stride=1 << 22), SHAPE)])
def test_attn_kv4_refuses(L, change, status):
    assert L.spdp_attn_kv4(*dict(ATTN, **change).values()) == status


def test_attn_kv4_refuses_more_units_than_32_bits_count(L):
    """2^24 pairs of a request and a key head of up to 124 units of 64 keys; with 6 more to each, as the kernel counts, above 2^31."""
    many = dict(ATTN, B=4096, q_heads=4096, kv_heads=4096, dim=64, ldq=1 << 18, ldy=1 << 18, mask_stride=1 << 13, table_pages=495, table_stride=495)
    assert 4096 * 4096 * (124 + 6) >= 2 ** 31
    assert L.spdp_attn_kv4(*many.values()) == SHAPE


@pytest.mark.parametrize("scale", [1.1e16, -1.1e16, 1e38])
def test_attn_kv4_refuses_scales_beyond_its_scores(L, scale):
    assert L.spdp_attn_kv4(*dict(ATTN, scale=scale).values()) == INVALID


def test_page_bytes(L):
    for heads, dim, page in ((1, 64, 16), (8, 128, 64), (3, 256, 256), (12, 128, 32)):
        assert spdp.spdp_kv4_page_bytes(heads, dim, page) == heads * page * 2 * (dim // 2 + dim // 32 * 2)
    for heads, dim, page in ((0, 128, 16), (1, 100, 16), (1, 128, 17)):
        with pytest.raises(spdp.SpdpError):
            spdp.spdp_kv4_page_bytes(heads, dim, page)
    assert L.spdp_kv4_page_bytes(1, 128, 16, None) == INVALID


@pytest.mark.parametrize("name,n", [("lora", 10), ("qk_norm_rope", 13), ("kv4_store", 9), ("attn_kv4", 14)])
def test_wrong_arguments_raise(L, name, n):
    call = getattr(L, "call_" + name)
    with pytest.raises(TypeError):
        call(*[0] * (n - 1))
    with pytest.raises(TypeError):
        call("x", *[0] * (n - 1))
    with pytest.raises((TypeError, OverflowError)):
        call(1 << 70, *[0] * (n - 1))
    with pytest.raises(TypeError, match="torch tensor"):
        call(*[0] * n)


HOST = -1            # "the current device" of calls on tensors in the host's memory, which the library never sees: a callback stands in for it


def arrived(L, name, *args):
    """What the entry point gets from a call on host tensors."""
    from paper_2607_21985_b200 import _pycall
    seen = []
    plain = lambda v: [v[i] for i in range(3)] if isinstance(v, ctypes.POINTER(ctypes.c_int)) and v else None if isinstance(v, ctypes.POINTER(ctypes.c_int)) else v
    cb = ctypes.CFUNCTYPE(ctypes.c_int, *getattr(L, "spdp_" + name).argtypes)(lambda *a: seen.append([plain(v) for v in a]) or -3)      # read while the call lasts
    assert getattr(_pycall, name)(ctypes.cast(cb, ctypes.c_void_p).value, HOST, *args) == -3
    return seen[0]


class StreamLike:
    cuda_stream = 99


def test_tensors_arrive_lora(L):
    import torch
    x, y, base = torch.zeros(5, 9).half()[:, 1:8], torch.zeros(5, 12)[:, :11], torch.zeros(5, 11)
    A, B = torch.zeros(3, 4, 10).half()[:, :2, :7], torch.zeros(3, 11, 6).half()[:, :, 2:4]
    adapter, scales, ranks = torch.zeros(5, dtype=torch.int32), torch.zeros(3), torch.zeros(3, dtype=torch.int32)
    p = lambda *t: [v.data_ptr() for v in t]
    assert arrived(L, "lora", x, adapter, A, B, y, base, scales, ranks, StreamLike()) == \
        p(x) + [5, 7, 9] + p(adapter, A) + [10, 40] + p(B) + [6, 66, 3, 2] + p(ranks, scales, base) + [11] + p(y) + [11, 12, 1, 99]
    one = torch.zeros(7).half()
    got = arrived(L, "lora", one, adapter[:1], A, B, y[0].half(), None, None, None, 5)
    assert got[:4] == [one.data_ptr(), 1, 7, 7] and got[13:15] == [None, None] and got[15] == got[17] and got[16] == 11 and got[18:] == [11, 11, 0, 5]
    assert arrived(L, "lora", torch.nn.Parameter(x.contiguous()), adapter, A, B, y, y, None, None, 0)[1:4] == [5, 7, 7]


def test_tensors_arrive_heads(L):
    import torch
    qkv = torch.zeros(6, 5 * 64).half()
    q, k = qkv[:, :192].unflatten(1, (3, 64)), qkv[:, 192:].unflatten(1, (2, 64))
    qo, ko = torch.zeros(6, 3, 64).half(), torch.zeros(6, 2, 64).half()
    pos, freq, w = torch.zeros(3, 8, dtype=torch.int32)[:, :6], torch.zeros(24), torch.zeros(64).half()
    p = lambda *t: [v.data_ptr() for v in t]
    assert arrived(L, "qk_norm_rope", q, k, qo, ko, pos, freq, [7, 8, 9], w, None, 0.5, 1, 3) == \
        p(q) + [320] + p(k) + [320, 0, 6, 3, 2, 64] + p(w) + [None, 0.5] + p(pos) + [8, 3, [7, 8, 9]] + p(freq) + [24, 1] + p(qo) + [192] + p(ko) + [128, 3]
    got = arrived(L, "qk_norm_rope", q.float(), None, qo, None, pos[1], freq, None, None, None, 0.0, 0, 3)
    assert got[2:9] == [None, 0, 1, 6, 3, 0, 64] and got[13:16] == [6, 1, [24, 0, 0]] and got[20:23] == [192, None, 0]
    assert arrived(L, "qk_norm_rope", q, None, qo, None, None, None, None, None, None, 0.0, 0, 3)[12:18] == [None, 0, 0, None, None, 0]
    for sections in ((7, 8), None, 5, (1, 2, "x")):
        with pytest.raises(TypeError):
            arrived(L, "qk_norm_rope", q, None, qo, None, pos, freq, sections, None, None, 0.0, 0, 3)


def test_tensors_arrive_cache(L):
    import torch
    p = lambda *t: [v.data_ptr() for v in t]
    k, v = torch.zeros(4, 3, 64).half(), torch.zeros(4, 200)[:, :192].unflatten(1, (3, 64))
    cache, slot, kv = torch.zeros(9, 3 * 16 * 72, dtype=torch.uint8), torch.zeros(4, dtype=torch.int64), torch.zeros(4, 6, 64).half()[:, :3]
    assert arrived(L, "kv4_store", k, v, slot, cache, 16, kv, None, 8) == \
        p(k) + [192] + p(v) + [200, 1, 4, 3, 64] + p(slot, cache) + [9, 16] + p(kv) + [384, None, 0, 8]
    q, y = torch.zeros(4, 6, 64).half(), torch.zeros(4, 400).half()[:, :384]
    table, length, mask = torch.zeros(4, 7, dtype=torch.int32)[:, :5], torch.zeros(4, dtype=torch.int32), torch.zeros(4, 13, dtype=torch.uint32)
    assert arrived(L, "attn_kv4", q, cache, 16, 3, table, length, y, 0.25, 2.0, 17, 0.5, mask, 8) == \
        p(q) + [384, 4, 6, 3, 64] + p(cache) + [9, 16] + p(table) + [7, 5] + p(length) + [0.25, 2.0, 17, 0.5] + p(y) + [400] + p(mask) + [13, 8]
    assert arrived(L, "attn_kv4", q, cache, 16, 3, table, length, y, 0.25, 0, 0, 0, None, 8)[18:] == [400, None, 0, 8]


def test_tensors_keep_their_references(L):
    import sys

    import torch
    h, i = torch.zeros(2, 4).half(), torch.zeros(2, dtype=torch.int32)
    A, B, y = torch.zeros(1, 3, 4).half(), torch.zeros(1, 5, 3).half(), torch.zeros(2, 5).half()
    things = (h, i, A, B, y, type(h), None)
    before = [sys.getrefcount(t) for t in things[:5]]
    for _ in range(50):
        arrived(L, "lora", h, i, A, B, y, None, None, None, 0)
        with pytest.raises(ValueError):
            arrived(L, "lora", h, i, A, B, h, None, None, None, 0)
    assert [sys.getrefcount(t) for t in things[:5]] == before


def test_binding_refuses_tensors():
    import torch
    h = torch.zeros(2, 4, dtype=torch.float16)
    ok = dict(X=h, adapter=torch.zeros(2, dtype=torch.int32), A=torch.zeros(1, 3, 4).half(), B=torch.zeros(1, 5, 3).half(), Y=torch.zeros(2, 5).half())
    for change in (dict(A=torch.zeros(1, 3, 5).half()), dict(B=torch.zeros(2, 5, 3).half()), dict(A=torch.zeros(1, 3, 4)), dict(X=h.float()), dict(adapter=None),
                   dict(Y=torch.zeros(2, 5).double()), dict(base=torch.zeros(2, 5)), {}):             # the last: not CUDA tensors
        with pytest.raises(ValueError):
            spdp.spdp_lora(**dict(ok, **change))
    x = torch.zeros(2, 3, 64).half()
    with pytest.raises(ValueError):
        spdp.spdp_qk_norm_rope(x, None, x, None, None, None)
    with pytest.raises(ValueError):
        spdp.spdp_qk_norm_rope(x.double(), None, x, None, None, None)
    with pytest.raises(ValueError):
        spdp.spdp_kv4_store(x, x, torch.zeros(2, dtype=torch.int64), torch.zeros(1, 16 * 3 * 72, dtype=torch.uint8), 16)
    with pytest.raises(ValueError):
        spdp.spdp_attn_kv4(x, torch.zeros(1, 16 * 3 * 72, dtype=torch.uint8), 16, 3, torch.zeros(2, 1, dtype=torch.int32), torch.zeros(2, dtype=torch.int32),
                           x.view(2, -1), 1.0)


def test_tensors_are_refused_one_by_one(L):
    import torch

    from paper_2607_21985_b200 import _pycall
    h = lambda *n: torch.zeros(*n).half()
    i = lambda *n: torch.zeros(*n, dtype=torch.int32)
    sets = {
        "lora": ([h(4, 8), i(4), h(2, 3, 8), h(2, 5, 3), h(4, 5), h(4, 5), torch.zeros(2), i(2), 0],
                 {0: (h(4, 9), h(4, 8).float(), h(4, 16)[:, ::2], h(1, 1, 4, 8), h(1)[0]), 1: (None, i(3), i(4).long(), i(8)[::2]), 2: (h(2, 3, 9), h(3, 8), h(2, 3, 16)[:, :, ::2]),
                  3: (h(1, 5, 3), h(2, 5, 4), h(2, 5, 6)[:, :, ::2]), 4: (h(4, 6), h(3, 5), h(4, 5).double(), h(5)), 5: (h(4, 5).float(), h(3, 5), h(5, 4).t()), 6: (torch.zeros(3), h(2)),
                  7: (i(1), torch.zeros(2))}),
        "qk_norm_rope": ([h(4, 3, 64), h(4, 2, 64), h(4, 3, 64), h(4, 2, 64), i(4), torch.zeros(8), None, h(64), h(64), 0.0, 0, 0],
                         {0: (h(4, 192), h(4, 3, 64).double(), h(4, 6, 64)[:, ::2], h(4, 3, 128)[:, :, ::2]), 1: (h(3, 2, 64), h(4, 2, 32), h(4, 2, 64).float()),
                          2: (h(4, 3, 64).float(), h(4, 2, 64)), 3: (h(4, 2, 64).float(), h(4, 3, 64)), 4: (i(5), i(4).long(), i(8)[::2], i(1, 1, 4)),
                          5: (torch.zeros(16)[::2], h(8)), 7: (h(63), torch.zeros(64)), 8: (h(128)[::2],)}),
        "kv4_store": ([h(4, 3, 64), h(4, 3, 64), torch.zeros(4, dtype=torch.int64), torch.zeros(2, 3 * 16 * 72, dtype=torch.uint8), 16, h(4, 3, 64), h(4, 3, 64), 0],
                      {0: (h(4, 3, 64).float(), h(4, 64)), 1: (h(4, 3, 64).double(), h(4, 2, 64)), 2: (None, i(4), torch.zeros(3, dtype=torch.int64)),
                       3: (torch.zeros(2, 3 * 16 * 72 + 1, dtype=torch.uint8), torch.zeros(3 * 16 * 72, dtype=torch.uint8), torch.zeros(2, 3 * 16 * 72, dtype=torch.int8)),
                       4: (32,), 5: (h(4, 3, 32), h(4, 3, 64).float()), 6: (h(3, 3, 64), h(4, 3, 64).float())}),
        "attn_kv4": ([h(4, 6, 64), torch.zeros(2, 3 * 16 * 72, dtype=torch.uint8), 16, 3, i(4, 5), i(4), h(4, 384), 0.1, 0.0, 0, 0.0, i(4, 12), 0],
                     {0: (h(4, 384), h(4, 6, 64).float()), 1: (torch.zeros(2, 3 * 16 * 72 * 2, dtype=torch.uint8)[:, ::2],), 3: (2,), 4: (i(3, 5), i(20), i(4, 10)[:, ::2], i(4, 5).long()),
                      5: (None, i(5), i(4).float()), 6: (h(4, 383), h(4, 384).float(), h(3, 384)), 11: (i(4, 11), i(3, 12), i(4, 12).long(), i(48), i(4, 24)[:, ::2])})}
    for name, (args, changes) in sets.items():
        arrived(L, name, *args)
        with pytest.raises(ValueError, match="current device"):
            getattr(_pycall, name)(1, 0, *args)
        for at, values in changes.items():
            for v in values:
                with pytest.raises(ValueError):
                    arrived(L, name, *args[:at], v, *args[at + 1:])
            if torch.is_tensor(args[at]):
                with pytest.raises(TypeError, match="torch tensor"):
                    arrived(L, name, *args[:at], [1.0], *args[at + 1:])


def test_oracle_codes_by_hand():
    x = np.zeros((1, 64), np.float16)
    x[0, :4] = [7.0, -7.0, 2.5, -1.49]
    x[0, 32:35] = [2.0 ** -24, 0.0, 0.0]              # its scale rounds to 0
    codes, scales = O.kv4_codes(x)
    assert scales[0].tolist() == [1.0, 0.0] and codes[0, :5].tolist() == [15, 1, 10, 7, 8] and (codes[0, 32:] == 8).all()
    assert O.kv4_values(codes, scales)[0, :4].tolist() == [7.0, -7.0, 2.0, -1.0]


def test_oracle_cache_layout_by_hand():
    """Dimension 32 g + 8 c + j is bits 4 j .. of word c G + g, bytes lowest first."""
    cache = O.Kv4Cache(np.zeros((2, 1 * 16 * 144), np.uint8), 1, 128, 16)
    k = np.zeros((1, 128), np.float16)
    k[0, 32 * 2 + 8 * 1 + 5] = 7.0
    cache.store(16 + 3, k, -k)
    row = cache.raw[1, 3 * 64:4 * 64].view(np.uint32)
    want = np.full(16, 0x88888888, np.uint32)
    want[1 * 4 + 2] = 0x88F88888
    assert np.array_equal(row, want) and cache.raw[1, 16 * 64 + 3 * 64:16 * 64 + 4 * 64].view(np.uint32)[6] == 0x88188888
    assert cache.raw[1, 2 * 1024 + 3 * 8:2 * 1024 + 3 * 8 + 8].view(np.float16).tolist() == [0.0, 0.0, 1.0, 0.0]
    assert np.array_equal(cache.load(19, 0, 1), -k[0].astype(np.float64)) and cache.raw[0].sum() == 0


def test_oracle_attention_and_rotation_by_hand():
    cache = O.Kv4Cache(np.zeros((1, 16 * 72), np.uint8), 1, 64, 16)
    for s in range(3):
        row = np.zeros((1, 64), np.float16)
        row[0, s] = 7.0
        cache.store(s, row, row)
    q = np.zeros((1, 64))
    q[0, 1] = np.log(3.0) / 7.0
    y, _, _, n = O.attention(q, cache, [0], 3, 1.0)
    assert n == 3 and np.allclose(y[0, :4], np.array([1.0, 3.0, 1.0, 0.0]) * 7 / 5)
    assert np.allclose(O.attention(q, cache, [0], 3, 1.0, window=1)[0][0, :3], [0, 0, 7])
    x, _ = O.norm_rope(np.array([[[3.0, 4.0, 0.0, 1.0]]]), None, 0.0, [[1], [2]], np.array([np.pi / 2, np.pi / 2]), (1, 1), False)
    assert np.allclose(x[0, 0], [0.0, -4.0, 3.0, -1.0])
    y, _, _ = O.lora([[1.0, 2.0]], [0], [[[1.0, 1.0], [5.0, 0.0]]], [[[2.0, 1.0]]], [[0.5]], [2.0], [1])
    assert y.tolist() == [[12.5]]
