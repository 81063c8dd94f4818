"""Storing into the 8-bit cache where a warp goes through 16 tokens of several requests (many tokens times heads), where values are no
numbers, and where tokens are taken back: byte for byte against the oracle, as in test_gpu_kv8.py."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

import test_gpu_kv8 as K
from oracle import kv8 as O
from test_gpu_kv8 import dev, garbage, host, ints, rows_like, starts

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def S():
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA device")
    from paper_2607_21985_b200 import spdp
    spdp.lib()
    return spdp


def by_sixteen(N, heads):
    """Whether the second step of a case goes by 16 tokens to a warp, on this GPU: as the launch decides it."""
    return -(-N // 16) * 2 * heads > 4 * torch.cuda.get_device_properties(0).multi_processor_count


SHORT = [(1 + 7 * i % 25, 11 * i % 40) for i in range(50)]         # new tokens, tokens before them
MANY = [(i % 3, 5 * i % 33) for i in range(500)]


@pytest.mark.parametrize("heads,D,page,requests,f32,misaligned", [
    # few requests of uneven lengths behind what ends inside a cell; up to 31 of them a lane holds a request
    (8, 128, 16, [(211, 5), (1, 30), (97, 15), (0, 7), (160, 17), (3, 14), (333, 1)], True, False), (16, 64, 64, [(1, 15), (299, 3), (2, 31), (40, 16)], False, False),
    (10, 128, 32, [(17, n) for n in range(31)], False, True),
    # 16 tokens are those of several requests
    (12, 64, 32, SHORT, False, True), (16, 128, 16, SHORT, True, False), (20, 64, 16, MANY, False, False), (13, 64, 256, [(16, 0)] * 33, True, True),
    # heads of 256, rows apart and not
    (3, 256, 64, [(900, 11), (700, 3), (50, 29)], True, True), (7, 256, 16, [(15 + i % 3, i) for i in range(45)], False, False)])
def test_kv8_store_by_sixteen_tokens(S, heads, D, page, requests, f32, misaligned):
    assert by_sixteen(sum(n for n, _ in requests), heads)
    K.test_kv8_store(S, heads, D, page, requests, f32, misaligned)


@pytest.mark.parametrize("requests", [5, 40])
def test_kv8_store_by_sixteen_tokens_passes_over(S, requests):
    """Tokens of no request at both ends, more new tokens than a request has, lengths beyond the table and below 0, pages that do not exist."""
    rng = np.random.default_rng(requests)
    heads, D, page, each = 16, 128, 16, 4
    counts = [40, 18, 25, 10, 200] + [int(n) for n in rng.integers(0, 24, requests - 5)]
    length = [40, 5, 10 ** 9, -4, 33] + [int(n) for n in rng.integers(-3, 70, requests - 5)]
    first = 2 + starts(counts)
    N = int(first[-1]) + 9
    assert by_sixteen(N, heads)
    table = rng.permutation(each * requests).reshape(requests, each).astype(np.int32)
    pages = each * requests - 7                               # the last numbers are no pages
    table[0, 1], table[2, 0], table[4, 2] = -1, 2 ** 31 - 1, -2 ** 31
    raw = garbage(rng, pages, heads, D, page)
    want, cache = O.Kv8Cache(raw.copy(), heads, D, page), dev(raw)
    past = [max(0, min(n, each * page) - c) for n, c in zip(length, counts)]
    k, v = rows_like(rng, sum(past), heads, D), rows_like(rng, sum(past), heads, D)
    for b in range(requests):
        part = slice(sum(past[:b]), sum(past[:b + 1]))
        want.store(table[b], past[b], k[part], v[part])
    S.spdp_kv8_store(dev(k), dev(v), cache, page, dev(table), ints(*past), first=dev(starts(past)))
    torch.cuda.synchronize()
    assert np.array_equal(cache.cpu().numpy(), want.raw)
    k, v = rows_like(rng, N, heads, D, (0.01, 20.0)), rows_like(rng, N, heads, D, (0.01, 20.0))
    values = [np.full((N, heads, D), np.nan), np.full((N, heads, D), np.nan)]
    for b in range(requests):
        part = slice(first[b], first[b + 1])
        for out, x in zip(values, want.store(table[b], length[b], k[part], v[part])):
            out[part] = x
    kv, vv = (torch.full((N, heads, D), float("nan"), dtype=torch.float16, device="cuda") for _ in range(2))
    S.spdp_kv8_store(dev(k), dev(v), cache, page, dev(table), ints(*length), first=dev(first.astype(np.int32)), k_values=kv, v_values=vv)
    torch.cuda.synchronize()
    assert np.array_equal(cache.cpu().numpy(), want.raw)
    assert np.array_equal(host(kv), values[0], equal_nan=True) and np.array_equal(host(vv), values[1], equal_nan=True)
    assert np.isnan(values[0][:2]).all() and np.isnan(values[0][-9:]).all() and np.isnan(values[0][first[4]:first[4] + 167]).all()


@pytest.mark.parametrize("heads", [2, 20])                    # a warp to a token's cell, or to 16 tokens
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("f32,misaligned", [(False, False), (True, False), (False, True), (True, True)])
def test_kv8_store_no_numbers(S, heads, D, f32, misaligned):
    """NaN, of both signs and with other bits, is one of -61440 and 61440: of a token that joins a cell whose scale is large enough, that makes a cell grow, that
    begins one, and among others.  The other tokens of its cell are as with that number."""
    rng = np.random.default_rng(D + heads)
    page, past, counts = 16, [5, 5, 0, 3], [1, 1, 1, 300]
    length = [n + p for n, p in zip(counts, past)]
    table = np.arange(4 * 20, dtype=np.int32).reshape(4, 20)[:, ::-1].copy()
    raw = garbage(rng, 80, heads, D, page)
    want, cache = O.Kv8Cache(raw.copy(), heads, D, page), dev(raw)
    k, v = rows_like(rng, sum(past), heads, D), rows_like(rng, sum(past), heads, D)
    k[3, :, 1], v[3, :, 2] = 61440, -61440                    # of the first request
    for b in range(4):
        part = slice(sum(past[:b]), sum(past[:b + 1]))
        want.store(table[b], past[b], k[part], v[part])
    S.spdp_kv8_store(dev(k), dev(v), cache, page, dev(table), ints(*past), first=dev(starts(past)))
    first, N = starts(counts), sum(counts)
    assert by_sixteen(N, heads) == (heads == 20)
    k, v = rows_like(rng, N, heads, D), rows_like(rng, N, heads, D).astype(np.float32 if f32 else np.float16)
    none = np.zeros(k.shape, bool)
    for t in (0, 1, 2, 3, 20, 45, 302):
        none[t, :, [t % 7, D // 2 + 1, D - 1]] = True
    none[100] = True                                          # a token without a number
    which = np.cumsum(none.ravel()).reshape(none.shape) % 4
    k.view(np.uint16)[none] = np.array([0x7E00, 0xFE00, 0x7C01, 0xFFFF], np.uint16)[which[none]]
    if f32:
        v.view(np.uint32)[none] = np.array([0x7FC00000, 0xFFC00000, 0x7F800001, 0xFFFFFFFF], np.uint32)[which[none]]
    else:
        v.view(np.uint16)[none] = np.array([0xFE00, 0x7E00, 0xFC01, 0x7FFF], np.uint16)[which[none]]

    def placed(a):
        if not misaligned:
            return dev(a)
        t = torch.zeros(N, heads * D + 3, dtype=torch.from_numpy(a).dtype, device="cuda")[:, 1:heads * D + 1].unflatten(1, (heads, D))
        return t.copy_(dev(a))
    kv, vv = (torch.empty(N, heads, D, dtype=torch.float16, device="cuda") for _ in range(2))
    S.spdp_kv8_store(placed(k), placed(v), cache, page, dev(table), ints(*length), first=dev(first), k_values=kv, v_values=vv)
    torch.cuda.synchronize()
    got = [host(kv), host(vv)]
    for x, y in zip((k, v), got):
        assert (np.abs(y[none]) == O.MOST).all()
        x[none] = y[none]
    for b in range(4):
        part = slice(first[b], first[b + 1])
        for y, x in zip(got, want.store(table[b], length[b], k[part], v[part].astype(np.float16))):
            assert np.array_equal(y[part], x), b
    assert np.array_equal(cache.cpu().numpy(), want.raw)


@pytest.mark.parametrize("heads", [2, 40])
def test_kv8_store_of_tokens_that_are_taken_back(S, heads):
    """Drafted tokens that are rejected: the length goes back and others are stored in their place.  A cell keeps the scale it has grown to while tokens before the new ones
    stay in it, and starts anew at its first token."""
    rng = np.random.default_rng(heads)
    D, page, B = 64, 32, 3
    raw = garbage(rng, 9, heads, D, page)
    want, cache = O.Kv8Cache(raw.copy(), heads, D, page), dev(raw)
    table = rng.permutation(9).reshape(B, 3).astype(np.int32)
    have = [0] * B
    for step, (back, new, size) in enumerate([(0, 50, 1.0), (3, 8, 300.0), (7, 1, 0.01), (1, 1, 0.01), (9, 30, 0.1), (0, 4, 3000.0), (60, 60, 0.2), (16, 7, 1.0)]):
        have = [max(0, n - back - b) + new for b, n in enumerate(have)]
        k, v = rows_like(rng, B * new, heads, D, (size,)), rows_like(rng, B * new, heads, D, (size, size / 8))
        for b in range(B):
            want.store(table[b], have[b], k[b * new:(b + 1) * new], v[b * new:(b + 1) * new])
        S.spdp_kv8_store(dev(k), dev(v), cache, page, dev(table), ints(*have), first=dev(starts([new] * B)))
        torch.cuda.synchronize()
        got = O.Kv8Cache(cache.cpu().numpy(), heads, D, page)
        for b in range(B):                                   # what lies behind the last token may be anything
            for t in range(have[b]):
                for h in range(heads):
                    mine, theirs = (c.cell(int(table[b, t // page]), t % page, h) for c in (got, want))
                    assert np.array_equal(mine[32 * D:], theirs[32 * D:]), (step, b, t)
                    for places in want.places:
                        assert np.array_equal(mine[places[t % 16]], theirs[places[t % 16]]), (step, b, t)
