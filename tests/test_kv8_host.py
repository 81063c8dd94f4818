"""The 8-bit cache and the handling of pages, without a GPU: refusals, the page size, the argument conversion, and the oracle itself against
hand-made values."""
import ctypes

import numpy as np
import pytest

from oracle import kv8 as O
from paper_2607_21985_b200 import build, spdp

F, ODD = 1 << 20, (1 << 20) + 1          # addresses that are never touched: every call here is refused first
INVALID, SHAPE = spdp.SPDP_ERR_INVALID_ARG, spdp.SPDP_ERR_UNSUPPORTED_SHAPE


@pytest.fixture(scope="module")
def L():
    build.build()
    return spdp.lib()


STORE = dict(k=F, ldk=256, v=F, ldv=256, vdt=0, N=3, heads=2, dim=128, B=2, first=F, table=F, table_stride=4, table_pages=4, length=F, cache=F, pages=5, page=16, ko=F, ldko=256,
             vo=F, ldvo=256, stream=None)


@pytest.mark.parametrize("change,status", [
    (dict(k=None), INVALID), (dict(v=None), INVALID), (dict(table=None), INVALID), (dict(length=None), INVALID), (dict(cache=None), INVALID), (dict(heads=0), SHAPE),
    (dict(heads=4097), SHAPE), (dict(dim=96), SHAPE), (dict(page=8), SHAPE), (dict(page=24), SHAPE), (dict(page=512), SHAPE), (dict(N=0), INVALID), (dict(N=(1 << 24) + 1), INVALID),
    (dict(B=0), INVALID), (dict(B=4097), SHAPE), (dict(first=None), INVALID), (dict(pages=0), INVALID), (dict(pages=1 << 31), INVALID), (dict(table_pages=0), INVALID), (dict(table_stride=3), INVALID),
    (dict(table_pages=1 << 27, table_stride=1 << 27), SHAPE), (dict(ldk=255), INVALID), (dict(ldv=255), INVALID), (dict(vdt=3), INVALID), (dict(ldko=255), INVALID), (dict(ldvo=255), INVALID),
    (dict(k=ODD), INVALID), (dict(vdt=1, v=F + 2), INVALID), (dict(first=F + 2), INVALID), (dict(table=F + 2), INVALID), (dict(length=F + 1), INVALID), (dict(cache=F + 8), INVALID),
    (dict(ko=ODD), INVALID), (dict(vo=ODD), INVALID)])
def test_kv8_store_refuses(L, change, status):
    assert L.spdp_kv8_store(*dict(STORE, **change).values()) == status


ATTN = dict(q=F, ldq=1024, N=5, q_heads=8, kv_heads=2, dim=128, B=2, first=F, cache=F, pages=9, page=16, table=F, table_stride=4, table_pages=4, length=F, scale=0.1, cap=0.0,
            window=0, sinks=0, thr=0.0, y=2 * F, ldy=1024, mask=F, mask_stride=32, stream=None)


@pytest.mark.parametrize("change,status", [
    (dict(q=None), INVALID), (dict(cache=None), INVALID), (dict(table=None), INVALID), (dict(length=None), INVALID), (dict(y=None), INVALID), (dict(first=None), INVALID),
    (dict(q_heads=7), SHAPE), (dict(q_heads=0), SHAPE), (dict(kv_heads=0), SHAPE), (dict(dim=32), SHAPE), (dict(page=20), SHAPE), (dict(B=0), INVALID), (dict(B=4097), SHAPE),
    (dict(N=0), INVALID), (dict(N=(1 << 24) + 1), INVALID), (dict(pages=0), INVALID), (dict(table_pages=0), INVALID), (dict(table_stride=3), INVALID), (dict(ldq=1023), INVALID),
    (dict(ldy=1023), INVALID), (dict(window=-1), INVALID), (dict(sinks=-1), INVALID), (dict(mask_stride=31), INVALID), (dict(scale=float("inf")), INVALID),
    (dict(scale=float("nan")), INVALID), (dict(cap=-1.0), INVALID), (dict(cap=float("nan")), INVALID), (dict(q=ODD), INVALID), (dict(first=F + 2), INVALID), (dict(cache=F + 8), INVALID),
    (dict(table=F + 2), INVALID), (dict(length=F + 1), INVALID), (dict(y=ODD), INVALID), (dict(mask=F + 2), INVALID), (dict(table_pages=1 << 27, table_stride=1 << 27), SHAPE),
    (dict(B=4096, table_pages=1 << 24, table_stride=1 << 24), SHAPE), (dict(N=1 << 24, q_heads=128, ldq=16384, ldy=16384, mask_stride=512), SHAPE)])
def test_attn_kv8_refuses(L, change, status):
    assert L.spdp_attn_kv8(*dict(ATTN, **change).values()) == status


STATE = dict(ref=F, pages=9, table=F, rows=3, table_stride=4, table_pages=4)
LISTS = dict(row=F, start=F, stop=F, n=2)
CACHE = dict(cache=F, layers=2, layer_stride=9 * 64, page_bytes=64)
BAD_STATE = [(dict(ref=None), INVALID), (dict(table=None), INVALID), (dict(pages=0), INVALID), (dict(rows=0), INVALID), (dict(table_pages=0), INVALID), (dict(table_stride=3), INVALID),
             (dict(ref=F + 2), INVALID), (dict(table=F + 2), INVALID), (dict(pages=(1 << 28) + 1, layer_stride=1 << 40), SHAPE), (dict(rows=(1 << 24) + 1), SHAPE),
             (dict(rows=1 << 20, table_pages=1 << 12, table_stride=1 << 12), SHAPE)]
BAD_LISTS = [(dict(row=None), INVALID), (dict(start=None), INVALID), (dict(stop=None), INVALID), (dict(row=F + 2), INVALID), (dict(start=F + 1), INVALID), (dict(stop=F + 3), INVALID),
             (dict(n=-1), INVALID), (dict(n=4097), INVALID)]
BAD_CACHE = [(dict(cache=None), INVALID), (dict(cache=F + 8), INVALID), (dict(layers=0), INVALID), (dict(layers=65537), SHAPE), (dict(layer_stride=9 * 64 - 16), INVALID),
             (dict(layer_stride=9 * 64 + 8), INVALID), (dict(page_bytes=0), INVALID), (dict(page_bytes=72, layer_stride=9 * 80), INVALID)]


@pytest.mark.parametrize("change,status", BAD_STATE + BAD_LISTS + [(dict(short=F + 2), INVALID)])
def test_kv_pages_take_refuses(L, change, status):
    change = {k: v for k, v in change.items() if k != "layer_stride"}
    assert L.spdp_kv_pages_take(*(dict(STATE, **LISTS, short=F, stream=None) | change).values()) == status


@pytest.mark.parametrize("change,status", BAD_STATE + BAD_LISTS)
def test_kv_pages_free_refuses(L, change, status):
    change = {k: v for k, v in change.items() if k != "layer_stride"}
    assert L.spdp_kv_pages_free(*(dict(STATE, **LISTS, stream=None) | change).values()) == status


@pytest.mark.parametrize("change,status", BAD_STATE + BAD_LISTS + BAD_CACHE + [(dict(page=0), SHAPE), (dict(page=24), SHAPE), (dict(page=1 << 17), SHAPE), (dict(short=F + 2), INVALID)])
def test_kv_pages_fork_refuses(L, change, status):
    assert L.spdp_kv_pages_fork(*(dict(CACHE, **STATE, page=16, **LISTS, short=F, stream=None) | change).values()) == status


@pytest.mark.parametrize("change,status", BAD_CACHE + [(dict(pages=0), INVALID), (dict(src=None), INVALID), (dict(dst=None), INVALID), (dict(src=F + 2), INVALID), (dict(dst=F + 1), INVALID),
                                                       (dict(n=-1), INVALID), (dict(n=4097), INVALID)])
def test_kv_pages_copy_refuses(L, change, status):
    assert L.spdp_kv_pages_copy(*(dict(CACHE, pages=9, src=F, dst=F, n=2, stream=None) | change).values()) == status


@pytest.mark.parametrize("change,status", BAD_STATE + BAD_CACHE + [(dict(live=F + 2), INVALID)])
def test_kv_pages_compact_refuses(L, change, status):
    assert L.spdp_kv_pages_compact(*(dict(CACHE, **STATE, live=F, stream=None) | change).values()) == status


def test_page_bytes(L):
    assert spdp.spdp_kv8_page_bytes(8, 128, 16) == 8 * 16 * 257
    for bad in [(0, 128, 16), (8, 100, 16), (8, 128, 8), (8, 128, 48), (4097, 64, 16)]:
        with pytest.raises(spdp.SpdpError):
            spdp.spdp_kv8_page_bytes(*bad)
    assert L.spdp_kv8_page_bytes(8, 128, 16, None) == INVALID


def test_tensors_are_checked(L):
    """What is no CUDA tensor of the right form raises before the library is called."""
    import torch
    h, i = torch.zeros(2, 4, 64, dtype=torch.float16), torch.zeros(2, dtype=torch.int32)
    cache, table = torch.zeros(3, 4 * 16 * 129, dtype=torch.uint8), torch.zeros(2, 2, dtype=torch.int32)
    y = torch.zeros(2, 256, dtype=torch.float16)
    for call in (lambda: spdp.spdp_kv8_store(h, h, cache, 16, table, i), lambda: spdp.spdp_attn_kv8(h, cache, 16, 4, table, i, y, 0.1), lambda: spdp.spdp_kv_pages_take(i, table, i, i, i),
                 lambda: spdp.spdp_kv_pages_free(i, table, i, i, i), lambda: spdp.spdp_kv_pages_fork(cache, i, table, 16, i, i, i), lambda: spdp.spdp_kv_pages_copy(cache, i, i),
                 lambda: spdp.spdp_kv_pages_compact(cache, i, table), lambda: spdp.spdp_kv8_store(h.float(), h, cache, 16, table, i),
                 lambda: spdp.spdp_attn_kv8(h[0], cache, 16, 4, table, i, y, 0.1), lambda: spdp.spdp_kv_pages_take(None, table, i, i, i), lambda: spdp.spdp_kv_pages_copy(cache, None, i)):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(TypeError):
        spdp.spdp_kv_pages_copy("cache", i, i)


@pytest.mark.parametrize("name,n", [("kv8_store", 12), ("attn_kv8", 17), ("kv_pages_take", 9), ("kv_pages_free", 8), ("kv_pages_fork", 11), ("kv_pages_copy", 6), ("kv_pages_compact", 7)])
def test_wrong_numbers_of_arguments_raise(L, name, n):
    from paper_2607_21985_b200 import _pycall
    for count in (n - 1, n + 1):
        with pytest.raises(TypeError):
            getattr(_pycall, name)(*[0] * count)


# ---- the oracle

def test_oracle_codes():
    # 1.0625 lies between 1 (code 56) and 1.125 (57): the even code; 464 would round past the largest number
    assert O.e4m3([0.0, 1.0, 1.0625, 1.1875, 448.0, 449.0, 2.0 ** -9, 2.0 ** -10, 2.0 ** -10 * 1.01, -1.0, 0.017]).tolist() == [0, 56, 56, 58, 126, 126, 1, 0, 1, 184, 9]
    assert O.value([0, 56, 126, 1, 8, 184, 254]).tolist() == [0.0, 1.0, 448.0, 2.0 ** -9, 2.0 ** -6, -1.0, -448.0]
    torch = pytest.importorskip("torch")
    x = np.random.default_rng(0).standard_normal(20000).astype(np.float32) * 2.0 ** np.random.default_rng(1).integers(-12, 8, 20000)
    x = np.clip(x, -448, 448).astype(np.float32)
    assert np.array_equal(torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy(), O.e4m3(x))


def test_oracle_scales():
    assert [O.scale_for(np.array([x])) for x in (0.0, 448.0, 448.5, 1.75, 1.7500001, 61440.0, 2.0 ** -24)] == [2.0 ** -15, 1.0, 2.0, 2.0 ** -8, 2.0 ** -7, 256.0, 2.0 ** -15]


def test_oracle_store_and_growth():
    cache = O.Kv8Cache(np.full((2, 16 * 129), 0xFF, np.uint8), 1, 64, 16)
    k = np.zeros((3, 1, 64), np.float16)
    k[0, 0, :3], k[2, 0, 3] = [1.0, -0.3, 2.0 ** -12], 900.0
    first = cache.store([1], 2, k[:2], k[:2])
    assert first[0][0, 0, 0] == 1.0 and abs(first[0][0, 0, 1] + 0.3) <= 0.3 * 2 ** -4 and first[0][0, 0, 2] == 2.0 ** -12
    assert cache.load([1], 0, 0, 1)[2] == 2.0 ** -12
    cell = cache.cell(1, 0, 0)
    assert cell[32 * 64 + 8:].sum() == 0 and cell[2 * 64 * 16 - 1] == 0
    second = cache.store([1], 3, k[2:], k[2:])
    assert abs(second[1][0, 0, 3] - 900.0) <= 900.0 * 2 ** -4
    assert cache.load([1], 0, 0, 1)[0] == 1.0 and cache.load([1], 0, 0, 1)[2] == 0.0       # the scale is 4 now: 2^-14 of it is less than half a step
    assert (cache.raw[0] == 0xFF).all()


def test_oracle_attention_sees():
    cache = O.Kv8Cache(np.zeros((3, 16 * 129), np.uint8), 1, 64, 16)
    n = 40
    v = np.zeros((n, 1, 64), np.float16)
    v[np.arange(n), 0, np.arange(n)] = 1.0
    cache.store([0, 1, 2], n, np.zeros((n, 1, 64), np.float16), v)
    y, _, _, keys = O.attention(np.zeros((2, 1, 64)), cache, [0, 1, 2], n, 1.0, window=3, sinks=2)
    assert keys.tolist() == [5, 5]
    assert np.flatnonzero(y[1, 0]).tolist() == [0, 1, 37, 38, 39] and np.flatnonzero(y[0, 0]).tolist() == [0, 1, 36, 37, 38] and np.allclose(y[y > 0], 0.2)
    y, _, _, keys = O.attention(np.zeros((1, 1, 64)), cache, [0, -1, 2], 33, 1.0)
    assert keys.tolist() == [17] and np.flatnonzero(y[0, 0]).tolist() == [*range(16), 32]


def test_oracle_pages():
    p = O.Pages([[0, 3, -1], [-1, -1, -1], [5, -1, -1]], [1, 0, 2, 1, 0, 1], np.arange(12, dtype=np.uint8).reshape(1, 6, 2))
    assert p.fork([0, 2], [1, 1], [20, 0]) == 0
    assert p.table[1].tolist() == [0, 1, -1] and p.ref.tolist() == [2, 1, 2, 1, 0, 1] and p.cache[0, 1].tolist() == [6, 7]
    p.free([0], [0], [3])
    assert p.ref.tolist() == [1, 1, 2, 0, 0, 1]
    assert p.compact() == 4 and p.table.tolist() == [[-1] * 3, [0, 1, -1], [3, -1, -1]] and p.ref.tolist() == [1, 1, 2, 1, 0, 0] and p.cache[0, 3].tolist() == [10, 11]
    assert p.take([1, 0], [2, 0], [3, 2]) == 1 and p.table.tolist() == [[5, -1, -1], [0, 1, 4], [3, -1, -1]]
