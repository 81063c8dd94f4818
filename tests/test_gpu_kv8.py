"""The 8-bit key/value cache, the attention over it and the handling of a cache's pages on the GPU against the 64-bit oracle, at the
sizes, masks, strides and values where they can go wrong.

Tolerances.  u = 2^-11 is half a step of fp16, v = 2^-24 half a step of fp32.  One product of the tensor cores adds 16 terms with
at most 2 v of the sum of their sizes lost at each of 17 additions."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import kv8 as O

pytestmark = pytest.mark.gpu
U, V = 2.0 ** -11, 2.0 ** -24
TINY = 2.0 ** -25                       # half the smallest fp16 step


@pytest.fixture(scope="module")
def S():
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA device")
    from paper_2607_21985_b200 import spdp
    spdp.lib()
    yield spdp
    # what the captured calls' graphs had stays with the driver until it is asked for: other tests look at free memory
    import ctypes
    torch.cuda.synchronize()
    assert ctypes.CDLL("libcudart.so.12").cudaDeviceGraphMemTrim(torch.cuda.current_device()) == 0


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def ints(*a):
    return torch.tensor(a, dtype=torch.int32, device="cuda")


def host(t):
    return t.cpu().numpy().astype(np.float64)


def starts(counts):
    return np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)


# ---- storing ----------------------------------------------------------------------------------------------------------------

def garbage(rng, pages, heads, D, page):
    """A cache in which nothing is a number: codes of NaN among the others, scales of any bits."""
    raw = rng.integers(0, 256, (pages, heads * page * (2 * D + 1)), dtype=np.uint8)
    raw[rng.random(raw.shape) < 0.3] = 0xFF
    return raw


def tables(rng, pages, lengths, page, spare=0):
    each = max(1, max(-(-n // page) for n in lengths)) + spare
    assert pages >= each * len(lengths)
    return rng.permutation(pages)[:each * len(lengths)].reshape(len(lengths), each).astype(np.int32)


def rows_like(rng, n, heads, D, sizes=(1.0,)):
    x = rng.standard_normal((n, heads, D)) * rng.choice(sizes, (n, heads, 1))
    return np.clip(x, -65504, 65504).astype(np.float16)


@pytest.mark.parametrize("heads,D,page,requests,f32,misaligned", [
    (1, 64, 16, [(1, 0)], False, False), (3, 128, 16, [(1, 5), (16, 0), (17, 0), (2, 15)], True, False), (2, 256, 32, [(40, 0)], False, True),
    (5, 64, 256, [(300, 7), (1, 255), (1, 256), (0, 3), (31, 1)], True, True), (8, 128, 64, [(77, 3), (1, 16)], False, True), (1, 256, 128, [(3, 14), (33, 129)], True, False),
    (4, 128, 16, [(1, n) for n in range(40)], False, False), (2, 64, 16, [(5, n) for n in range(33)], True, False), (12, 64, 16, [(700, 9)], False, False),
    (1, 128, 32, [(2000, 3), (900, 1)], True, False)])
def test_kv8_store(S, heads, D, page, requests, f32, misaligned):
    """Byte for byte, step by step: what a request has, then its new tokens (larger ones among them, whose cells grow)."""
    rng = np.random.default_rng(heads + D + len(requests))
    lengths = [n + past for n, past in requests]
    pages = sum(-(-n // page) for n in lengths) + len(lengths) * max(-(-n // page) for n in lengths) + 2
    table = tables(rng, pages, lengths, page)
    want = O.Kv8Cache(garbage(rng, pages, heads, D, page), heads, D, page)
    cache = dev(want.raw.copy())

    def placed(a):
        if not misaligned:
            return dev(a)
        t = torch.zeros(a.shape[0], heads * D + 3, dtype=torch.from_numpy(a).dtype, device="cuda")[:, 1:heads * D + 1].unflatten(1, (heads, D))
        return t.copy_(dev(a))
    for step, counts in enumerate([[past for _, past in requests], [n for n, _ in requests]]):
        N = sum(counts)
        if N == 0:
            continue
        sizes = (1.0, 0.01) if step == 0 else (0.001, 1.0, 40.0)
        k, v = rows_like(rng, N, heads, D, sizes), rows_like(rng, N, heads, D, sizes).astype(np.float32 if f32 else np.float16)
        if f32:
            v = v * np.float32(1.0003)                       # rounds to fp16
        if step == 1:
            k[0, 0, :6] = [65504, -65504, 61440, 61441, 0, -0.0]
            v[N // 2, -1, :4] = [np.inf, -np.inf, 2.0 ** -24, -(2.0 ** -24)]
        first, length = starts(counts), np.array([past + (n if step else 0) for n, past in requests], np.int32)
        values = [np.zeros((N, heads, D)), np.zeros((N, heads, D))]
        for b in range(len(requests)):
            part = slice(first[b], first[b + 1])
            for out, x in zip(values, want.store(table[b], length[b], k[part], v[part].astype(np.float16))):
                out[part] = x
        kv, vv = (torch.full((N + 1, heads * D + (3 if misaligned else 0)), 5.0, dtype=torch.float16, device="cuda") for _ in range(2))
        S.spdp_kv8_store(placed(k), placed(v), cache, page, dev(table), dev(length), first=dev(first), k_values=kv[:N, :heads * D].unflatten(1, (heads, D)),
                         v_values=vv[:N, :heads * D].unflatten(1, (heads, D)))
        torch.cuda.synchronize()
        assert np.array_equal(cache.cpu().numpy(), want.raw), step
        for got, x in ((kv, values[0]), (vv, values[1])):
            assert np.array_equal(host(got[:N, :heads * D]).reshape(x.shape), x)
            assert bool((got[N] == 5.0).all()) and bool((got[:, heads * D:] == 5.0).all())


def test_kv8_store_one_token_each_is_store_of_runs_of_one(S):
    rng = np.random.default_rng(1)
    heads, D, page, B = 3, 128, 32, 70
    lengths = [int(n) for n in rng.integers(1, 100, B)]
    pages = 4 * B + 1
    table, raw = tables(rng, pages, [128] * B, page), np.zeros((pages, heads * page * (2 * D + 1)), np.uint8)
    want = O.Kv8Cache(raw.copy(), heads, D, page)
    past = [rows_like(rng, n - 1, heads, D) for n in lengths]
    for b in range(B):
        want.store(table[b], lengths[b] - 1, past[b], past[b])
    before = want.raw.copy()
    k, v = rows_like(rng, B, heads, D, (1.0, 9.0)), rows_like(rng, B, heads, D, (1.0, 9.0))
    for b in range(B):
        want.store(table[b], lengths[b], k[b:b + 1], v[b:b + 1])
    for first in (None, dev(np.arange(B + 1, dtype=np.int32))):
        cache = dev(before)
        S.spdp_kv8_store(dev(k), dev(v), cache, page, dev(table), dev(np.array(lengths, np.int32)), first=first)
        assert np.array_equal(cache.cpu().numpy(), want.raw)


def test_kv8_store_token_by_token(S):
    """Tokens that join one by one, with sizes that go up and down over all of fp16: codes rounded again and again."""
    rng = np.random.default_rng(2)
    heads, D, page, n = 2, 64, 16, 50
    raw = garbage(rng, 5, heads, D, page)
    want, cache, table = O.Kv8Cache(raw.copy(), heads, D, page), dev(raw), np.array([[3, 0, 4, 1]], np.int32)
    for t in range(n):
        k, v = (np.clip(rng.standard_normal((1, heads, D)) * 2.0 ** rng.integers(-24, 17), -65504, 65504).astype(np.float16) for _ in range(2))
        want.store(table[0], t + 1, k, v)
        S.spdp_kv8_store(dev(k), dev(v), cache, page, dev(table), ints(t + 1))
        assert np.array_equal(cache.cpu().numpy(), want.raw), t


def test_kv8_store_passes_over(S):
    """Pages that do not exist, more new tokens than the request has, lengths beyond the table, tokens of no request."""
    rng = np.random.default_rng(3)
    heads, D, page = 2, 128, 16
    raw = garbage(rng, 9, heads, D, page)
    want = O.Kv8Cache(raw.copy(), heads, D, page)
    table = np.array([[0, -1, 2], [3, 9, 2 ** 31 - 1], [4, 5, 6], [7, 8, -2 ** 31], [1, 1, 1]], np.int32)
    first = np.array([2, 42, 60, 85, 95, 95], np.int32)                  # tokens 0, 1 and 95 .. 99 are of no request
    length = np.array([40, 5, 10 ** 9, -4, 3], np.int32)
    N = 100
    k, v = rows_like(rng, N, heads, D), rows_like(rng, N, heads, D)
    want.store(table[2], 23, k[:23], v[:23])
    cache = dev(want.raw.copy())
    values = [np.full((N, heads, D), np.nan), np.full((N, heads, D), np.nan)]
    for b in range(5):
        part = slice(first[b], first[b + 1])
        for out, x in zip(values, want.store(table[b], length[b], k[part], v[part])):
            out[part] = x
    kv, vv = (torch.full((N, heads, D), float("nan"), dtype=torch.float16, device="cuda") for _ in range(2))
    S.spdp_kv8_store(dev(k), dev(v), cache, page, dev(table), dev(length), first=dev(first), k_values=kv, v_values=vv)
    torch.cuda.synchronize()
    assert np.array_equal(cache.cpu().numpy(), want.raw)
    assert np.array_equal(host(kv), values[0], equal_nan=True) and np.array_equal(host(vv), values[1], equal_nan=True)
    assert np.isnan(values[0][:2]).all() and np.isnan(values[0][42:55]).all() and np.isnan(values[0][85:]).all()
    # starts below 0, beyond the last token and out of order touch nothing that is not theirs
    before = cache.clone()
    for odd in ([-9, 0, 0, 0, 0, 0], [100, 200, 300, 2 ** 31 - 1, 100, 100], [50, 40, 30, 20, 10, 0]):
        S.spdp_kv8_store(dev(k), dev(v), cache, page, dev(table), dev(np.zeros(5, np.int32)), first=ints(*odd))
    torch.cuda.synchronize()
    assert torch.equal(before, cache)


# ---- attention --------------------------------------------------------------------------------------------------------------

def filled(rng, heads, D, page, lengths, spare=2, sizes=(0.01, 1.0, 30.0)):
    """A cache of garbage with the keys of each request in shuffled pages; (table, oracle)."""
    each = max(1, max(-(-n // page) for n in lengths))
    pages = each * len(lengths) + spare
    cache = O.Kv8Cache(garbage(rng, pages, heads, D, page), heads, D, page)
    table = tables(rng, pages, lengths, page)
    for b, n in enumerate(lengths):
        cache.store(table[b], n, rows_like(rng, n, heads, D, (1.5,)), rows_like(rng, n, heads, D, sizes))
        for t in range(-(-n // 16) * 16 - n):                # behind the last key: no numbers
            for h in range(heads):
                for side in (0, 1):
                    cache.cell(int(table[b, (n + t) // page]), (n + t) % page, h)[cache.places[side][(n + t) % 16]] = 0xFF
    return table, cache


def attn_bound(want, spread, reach, keys, cap, most):
    """Scores: D / 16 products of 17 additions at 2 v of the sizes, 8 sums and roundings more; a cap adds 8 v of itself; the values' exponent, -15 .. 8, and the exponential 2^-20.
    Weights: twice the scores' error, one rounding u and, where small, half of fp16's smallest step, 2^-25, against a largest weight of 2^8 at least (2^12 of few tokens, whose values count by their
    cell's scale: at most twice its largest, or 448 * 2^-15): 2^-33 of the largest value; the result's rounding."""
    ds = (2 * 2 * V * (17 * 16 + 8) * reach + 8 * V * cap + 2.0 ** -20)[..., None]
    return U * np.abs(want) * 1.01 + (U + 2 * ds) * 1.01 * spread + (keys * 2.0 ** -33 * (most + 0.014))[:, None, None] + TINY


def attn_check(y, q, cache, table, first, length, scale, cap=0.0, window=0, sinks=0, most=200.0):
    for b in range(len(length)):
        part = slice(int(first[b]), int(first[b + 1]))
        want, spread, reach, keys = O.attention(host(q[part]), cache, table[b], int(length[b]), scale, cap, window, sinks)
        err = np.abs(host(y[part]).reshape(want.shape) - want)
        bound = attn_bound(want, spread, reach, keys, cap, most)
        assert np.all(err <= bound), (b, int(length[b]), float((err - bound).max()))


CASES = [
    # heads, group, D, page, (new tokens, keys before), cap, window, sinks
    (1, 1, 128, 16, [(1, 0)], 0.0, 0, 0), (2, 4, 128, 16, [(1, 0), (1, 14), (1, 15), (1, 16), (0, 9)], 0.0, 0, 0), (1, 8, 64, 32, [(1, 62), (1, 63), (1, 64), (1, 129)], 0.0, 0, 0),
    (3, 3, 128, 64, [(1, 199), (1, 2), (1, 63)], 20.0, 0, 0), (1, 9, 128, 16, [(1, 99), (1, 32)], 0.0, 0, 0), (2, 16, 64, 16, [(1, 69), (1, 0), (1, 299)], 5.0, 50, 0),
    (1, 20, 128, 128, [(1, 128), (1, 256)], 0.0, 1, 0), (2, 2, 256, 256, [(1, 39), (1, 299)], 0.0, 17, 0), (1, 12, 256, 16, [(1, 89)], 30.0, 0, 0),
    (1, 33, 64, 16, [(1, 49)], 0.0, 16, 3), (4, 1, 128, 32, [(1, n) for n in (699, 4, 0, 30, 31, 32, 63)], 0.0, 100, 4), (2, 4, 64, 16, [(1, 400)], 0.0, 30, 17),
    # a few tokens each, also beside single ones
    (2, 4, 128, 16, [(3, 0), (1, 40), (4, 13), (2, 200)], 0.0, 0, 0), (1, 8, 64, 32, [(8, 100), (5, 0)], 8.0, 0, 0), (3, 5, 128, 16, [(7, 90), (0, 3), (1, 0)], 0.0, 20, 5),
    (1, 1, 256, 32, [(12, 33), (1, 60)], 0.0, 9, 2), (2, 16, 128, 64, [(2, 150), (3, 61)], 0.0, 0, 0),
    # prompts and pieces of them
    (1, 1, 64, 16, [(150, 0)], 0.0, 0, 0), (2, 4, 128, 16, [(130, 0)], 0.0, 0, 0), (1, 8, 128, 64, [(64, 0), (65, 70), (1, 300), (33, 1)], 0.0, 0, 0), (3, 2, 64, 32, [(257, 40)], 15.0, 0, 0),
    (1, 3, 256, 16, [(100, 30)], 0.0, 0, 0), (1, 12, 128, 32, [(40, 260)], 0.0, 60, 7), (2, 1, 128, 16, [(300, 100), (129, 0)], 0.0, 33, 20), (1, 5, 256, 64, [(90, 0), (70, 200)], 9.0, 50, 1),
    (1, 16, 64, 128, [(70, 500)], 0.0, 128, 16), (4, 7, 64, 16, [(45, 3), (0, 0), (80, 17)], 0.0, 0, 0)]


@pytest.mark.parametrize("columns", [2, 1000])     # of the table behind the longest request's: with 1000 the keys may be too many for one cluster
@pytest.mark.parametrize("heads,group,D,page,requests,cap,window,sinks", CASES)
def test_attn_kv8(S, heads, group, D, page, requests, cap, window, sinks, columns):
    rng = np.random.default_rng(heads * 100 + group + D + len(requests))
    counts, length = [n for n, _ in requests], np.array([n + past for n, past in requests], np.int32)
    table, oracle = filled(rng, heads, D, page, length)
    first, N, H = starts(counts), sum(counts), heads * group
    q = dev(rng.standard_normal((N + 1, H * D + 4)).astype(np.float16))[:N, :H * D].unflatten(1, (H, D))
    y_all = torch.full((N + 1, H * D + 3), 9.0, dtype=torch.float16, device="cuda")
    words = H * D // 32
    mask = torch.full((N + 1, words + 1), 123, dtype=torch.int32, device="cuda")
    y, scale, thr = y_all[:N, :H * D], 1.3 / np.sqrt(D), 0.05
    tab, cache = dev(np.concatenate([table, np.full((len(table), columns), -7, np.int32)], 1)), dev(oracle.raw)
    S.spdp_attn_kv8(q, cache, page, heads, tab, dev(length), y, scale, first=dev(first), cap=cap, window=window, sinks=sinks, thr=thr, mask=mask[:N])
    torch.cuda.synchronize()
    attn_check(y, q, oracle, table, first, length, scale, cap, window, sinks)
    assert bool((y_all[N] == 9.0).all()) and bool((y_all[:, H * D:] == 9.0).all()) and bool((mask[N] == 123).all()) and bool((mask[:, words:] == 123).all())
    keep = ~(y.float().abs() <= thr)
    bits = mask[:N, :words].cpu().numpy().view(np.uint32)
    assert np.array_equal((bits[:, :, None] >> np.arange(32, dtype=np.uint32) & 1).reshape(N, -1).astype(bool), keep.cpu().numpy())
    kept = y.clone()
    S.spdp_attn_kv8(q, cache, page, heads, tab, dev(length), y, scale, first=dev(first), cap=cap, window=window, sinks=sinks)
    assert torch.equal(kept, y)
    if all(n == 1 for n in counts):                # the form without starts
        z = torch.empty_like(kept)
        S.spdp_attn_kv8(q, cache, page, heads, tab, dev(length), z, scale, cap=cap, window=window, sinks=sinks)
        attn_check(z, q, oracle, table, first, length, scale, cap, window, sinks)


@pytest.mark.parametrize("columns", [0, 600])
def test_attn_kv8_pages_that_do_not_exist_and_odd_lengths(S, columns):
    rng = np.random.default_rng(8)
    table, oracle = filled(rng, 2, 128, 16, [80, 80, 80, 80, 80])
    table[0, 1], table[0, 3], table[1, :] = -1, 2 ** 31 - 1, len(oracle.raw)
    table[3, 0] = -5                                         # the first tokens see nothing
    table = np.concatenate([table, np.full((5, columns), len(oracle.raw) + 3, np.int32)], 1)
    counts = [1, 3, 2, 40, 90]
    length = np.array([80, 80, 10 ** 9 if columns == 0 else 80, 40, 60], np.int32)       # the last has more new tokens than keys
    first = starts(counts)
    q, y = dev(rng.standard_normal((sum(counts) + 2, 4, 128)).astype(np.float16)), torch.full((sum(counts) + 2, 512), 4.0, dtype=torch.float16, device="cuda")
    S.spdp_attn_kv8(q, dev(oracle.raw), 16, 2, dev(table), dev(length), y, 0.1, first=dev(first))
    attn_check(y, q, oracle, table, first, length, 0.1)
    assert bool((y[1:4] == 0).all()) and bool((y[6:22] == 0).all()) and bool((y[46:76] == 0).all()) and bool((y[-2:] == 4.0).all())
    # lengths of nothing and starts that are none
    for f, n in (([0, 1, 4, 6, 46, 136], [0, -3, 0, 0, 0]), ([-7, -2, 0, 0, 0, 0], [9, 9, 9, 9, 9]), ([9, 8, 7, 6, 5, 4], [9, 9, 9, 9, 9]), ([500, 600, 700, 800, 900, 2 ** 31 - 1], [9, 9, 9, 9, 9])):
        y.fill_(4.0)
        S.spdp_attn_kv8(q, dev(oracle.raw), 16, 2, dev(table), ints(*n), y, 0.1, first=ints(*f))
        torch.cuda.synchronize()
        assert bool((y[:136] == (0.0 if f[1] == 1 else 4.0)).all()) and bool((y[136:] == 4.0).all())


@pytest.mark.parametrize("tokens", [1, 5, 60])
@pytest.mark.parametrize("columns", [0, 600])
def test_attn_kv8_scores_of_all_sizes(S, columns, tokens):
    """Scores that grow along the keys, fall, and lie far apart: the running maximum, and weights down to nothing."""
    rng = np.random.default_rng(9)
    D, page, n = 128, 16, 200
    table, oracle = filled(rng, 1, D, page, [n, n, n])
    for b, size in enumerate([lambda t: t // 4, lambda t: (n - t) // 4, lambda t: 104.0 * (t % 7 == 3)]):
        k = np.zeros((n, 1, D), np.float16)
        k[:, 0, 5] = [size(t) for t in range(n)]
        oracle.store(table[b], n, k, rng.standard_normal((n, 1, D)).astype(np.float16))
    q = np.zeros((3 * tokens, 2, D), np.float16)
    q[:, 0, 5], q[:, 1, 5] = 8.0, -3.0
    y = torch.empty(3 * tokens, 2 * D, dtype=torch.float16, device="cuda")
    first = starts([tokens] * 3)
    S.spdp_attn_kv8(dev(q), dev(oracle.raw), page, 1, dev(np.concatenate([table, np.zeros((3, columns), np.int32)], 1)), ints(n, n, n), y, 0.125, first=dev(first))
    attn_check(y, dev(q), oracle, table, first, [n] * 3, 0.125, most=30.0)


@pytest.mark.parametrize("tokens", [1, 70])
@pytest.mark.parametrize("sizes", [(2e-5,), (6e4,), (1e-3, 3e4), (3e4, 1e-3), (1e-6, 1.0)])
def test_attn_kv8_values_of_all_sizes(S, sizes, tokens):
    """Values near both ends of fp16's range; large ones in the second half of the keys, and in the first."""
    rng = np.random.default_rng(10)
    D, page, n = 64, 16, 400
    table, oracle = filled(rng, 1, D, page, [n])
    v = np.stack([size * rng.uniform(-1, 1, (1, D)) for size in (sizes[len(sizes) * t // n] for t in range(n))]).astype(np.float16)
    oracle.store(table[0], n, rng.standard_normal((n, 1, D)).astype(np.float16), v)
    q, y = dev(rng.standard_normal((tokens, 3, D)).astype(np.float16)), torch.empty(tokens, 3 * D, dtype=torch.float16, device="cuda")
    S.spdp_attn_kv8(q, dev(oracle.raw), page, 1, dev(table), ints(n), y, 0.2, first=ints(0, tokens))
    attn_check(y, q, oracle, table, [0, tokens], [n], 0.2, most=max(sizes))


@pytest.mark.parametrize("tokens", [1, 70])
def test_attn_kv8_caps_that_leave_nothing_of_the_scores(S, tokens):
    """A cap whose reciprocal is beyond 32 bits: all scores are 0 or as good as 0, whether the products are 0 or not."""
    rng = np.random.default_rng(11)
    table, oracle = filled(rng, 1, 64, 16, [100])
    q = np.stack([np.zeros((tokens, 64)), rng.standard_normal((tokens, 64))], 1).astype(np.float16)
    y = torch.empty(tokens, 128, dtype=torch.float16, device="cuda")
    S.spdp_attn_kv8(dev(q), dev(oracle.raw), 16, 1, dev(table), ints(100), y, 0.1, first=ints(0, tokens), cap=1e-40)
    attn_check(y, dev(q) * 0, oracle, table, [0, tokens], [100], 0.1)


@pytest.mark.parametrize("scale,cap", [(2.0, 1e-40), (1e16, 1e-24), (-1e16, 1e-30)])
@pytest.mark.parametrize("tokens", [1, 70])
def test_attn_kv8_small_caps_of_large_scales(S, tokens, scale, cap):
    """Products of 0 under a cap that the scale divided by is beyond 32 bits: weights of 1 like those of the others."""
    rng = np.random.default_rng(17)
    table, oracle = filled(rng, 1, 64, 16, [100])
    q = np.stack([np.zeros((tokens, 64)), rng.standard_normal((tokens, 64))], 1).astype(np.float16)
    q[:tokens // 2] = 0                  # all rows of a warp, and some
    y = torch.empty(tokens, 128, dtype=torch.float16, device="cuda")
    S.spdp_attn_kv8(dev(q), dev(oracle.raw), 16, 1, dev(table), ints(100), y, scale, first=ints(0, tokens), cap=cap)
    attn_check(y, dev(q) * 0, oracle, table, [0, tokens], [100], 0.1)


@pytest.mark.parametrize("tokens", [1, 90])
def test_attn_kv8_no_numbers(S, tokens):
    """NaN and Inf in one token's query reach that head of that token only."""
    rng = np.random.default_rng(12)
    table, oracle = filled(rng, 2, 128, 16, [100, 70])
    first = starts([tokens if tokens < 70 else 60, 1])
    N = int(first[-1])
    q = dev(rng.standard_normal((N, 8, 128)).astype(np.float16))
    y, z = (torch.empty(N, 8, 128, dtype=torch.float16, device="cuda") for _ in range(2))
    args = (dev(oracle.raw), 16, 2, dev(table), ints(100, 70))
    S.spdp_attn_kv8(q, *args, y.view(N, -1), 0.1, first=dev(first))
    q[0, 3, 7], q[N - 1, 6, 0] = float("nan"), float("inf")
    S.spdp_attn_kv8(q, *args, z.view(N, -1), 0.1, first=dev(first))
    assert bool(z[0, 3].isnan().all()) and bool(z[N - 1, 6].isnan().all())
    z[0, 3], z[N - 1, 6] = y[0, 3], y[N - 1, 6]
    assert torch.equal(y, z)


@pytest.mark.parametrize("scale", [-0.11, 0.0, 1e-20])
@pytest.mark.parametrize("tokens", [1, 6, 80])
def test_attn_kv8_scales_below_and_at_zero(S, tokens, scale):
    rng = np.random.default_rng(13)
    table, oracle = filled(rng, 2, 128, 16, [120, 90])
    first = starts([tokens, 1])
    wide = torch.full((2, table.shape[1] + 5), 10 ** 6, dtype=torch.int32, device="cuda")          # rows of the table apart
    wide[:, :table.shape[1]] = dev(table)
    q, y = dev(rng.standard_normal((tokens + 1, 6, 128)).astype(np.float16)), torch.empty(tokens + 1, 768, dtype=torch.float16, device="cuda")
    for window, sinks in ((0, 0), (30, 3)):
        S.spdp_attn_kv8(q, dev(oracle.raw), 16, 2, wide[:, :table.shape[1]], ints(120, 90), y, scale, first=dev(first), window=window, sinks=sinks)
        attn_check(y, q, oracle, table, first, [120, 90], scale, 0.0, window, sinks)


def test_attn_kv8_prompt_of_many_blocks(S):
    """More blocks of rows than a CTA lists by itself, beside requests of a few tokens and of none."""
    heads, group, D, page = 1, 16, 64, 64
    counts, past = [4001, 0, 2, 300], [0, 5, 70, 1000]
    length = [n + p for n, p in zip(counts, past)]
    each, N = -(-max(length) // page), sum(counts)
    gen = torch.Generator(device="cuda").manual_seed(14)
    table = torch.randperm(4 * each, generator=gen, device="cuda").view(4, each).int()
    cache = torch.full((4 * each, S.spdp_kv8_page_bytes(heads, D, page)), 0xFF, dtype=torch.uint8, device="cuda")
    k, v = (torch.randn(sum(length), heads, D, generator=gen, device="cuda").half() for _ in range(2))
    kv, vv = torch.empty_like(k), torch.empty_like(v)
    S.spdp_kv8_store(k, v, cache, page, table, ints(*length), first=dev(starts(length)), k_values=kv, v_values=vv)
    q, y = torch.randn(N, group, D, generator=gen, device="cuda").half(), torch.empty(N, group * D, dtype=torch.float16, device="cuda")
    S.spdp_attn_kv8(q, cache, page, heads, table, ints(*length), y, 0.125, first=dev(starts(counts)))
    for b in (0, 2, 3):
        n, T = counts[b], length[b]
        some = torch.arange(0, n, 7 if b == 0 else 1, device="cuda")
        keys = slice(starts(length)[b], starts(length)[b + 1])
        seen = torch.arange(T, device="cuda") <= (past[b] + some)[:, None]
        at = int(starts(counts)[b]) + some
        device_check(y[at], q[at], kv[keys].double().transpose(0, 1), vv[keys].double().transpose(0, 1), seen, 0.125, 7.0, 7.0)


def exact_on_device(q, k, v, seen, scale):
    """In 64 bits: q [n][H][D], k and v [kv heads][keys][D], seen [n][keys] -> (y, spread), [n][H][D]."""
    z = torch.einsum("nhgd,htd->hgnt", q.double().unflatten(1, (k.shape[0], -1)), k) * scale
    p = torch.softmax(z.masked_fill(~seen, -torch.inf), -1).nan_to_num(0.0)
    return tuple(torch.einsum("hgnt,htd->nhgd", p, x).flatten(1, 2) for x in (v, v.abs()))


def device_check(y, q, k, v, seen, scale, kmost, vmost):
    """As attn_bound, with the scores' reach from the largest key."""
    want, spread = exact_on_device(q, k, v, seen, scale)
    reach = scale * (q.double().abs().sum(-1) * kmost)[..., None]
    bound = U * want.abs() * 1.01 + (U + 2 * (reach * 1120 * V + 2.0 ** -20)) * 1.02 * spread + k.shape[1] * 2.0 ** -33 * (vmost + 0.014) + TINY
    err = (y.double().view_as(want) - want).abs()
    assert bool((err <= bound).all()), float((err - bound).max())


def test_attn_kv8_long_and_behind_four_gigabytes(S):
    """Long requests among short ones, single tokens and pieces of prompts, in pages whose addresses pass 32 bits; stored by the library itself."""
    heads, group, D, page = 2, 8, 128, 64
    per = S.spdp_kv8_page_bytes(heads, D, page)
    pages = (5 << 30) // per
    cache = torch.full((pages, per), 0xFF, dtype=torch.uint8, device="cuda")
    lengths, counts = [20000, 1, 700, 9000], [1, 1, 3, 200]
    each = -(-lengths[0] // page)
    gen = torch.Generator(device="cuda").manual_seed(4)
    table = (pages - 1 - torch.randperm(each * 4, generator=gen, device="cuda")).view(4, each).int()
    table[0, 5] = 0
    k, v = (torch.randn(sum(lengths), heads, D, generator=gen, device="cuda").half() for _ in range(2))
    kv, vv = torch.empty_like(k), torch.empty_like(v)
    S.spdp_kv8_store(k, v, cache, page, table, ints(*lengths), first=dev(starts(lengths)), k_values=kv, v_values=vv)
    N = sum(counts)
    q, y = torch.randn(N, heads * group, D, generator=gen, device="cuda").half(), torch.empty(N, heads * group * D, dtype=torch.float16, device="cuda")
    S.spdp_attn_kv8(q, cache, page, heads, table, ints(*lengths), y, 0.125, first=dev(starts(counts)))
    for b, (n, T) in enumerate(zip(counts, lengths)):
        mine, keys = slice(starts(counts)[b], starts(counts)[b + 1]), slice(starts(lengths)[b], starts(lengths)[b + 1])
        seen = torch.arange(T, device="cuda") <= torch.arange(T - n, T, device="cuda")[:, None]
        device_check(y[mine], q[mine], kv[keys].double().transpose(0, 1), vv[keys].double().transpose(0, 1), seen, 0.125, 7.0, 7.0)


@pytest.mark.parametrize("D,group,n,tokens", [(64, 1, 60001, 1), (128, 8, 60000, 1), (256, 9, 40007, 1), (128, 8, 50001, 5), (128, 4, 30003, 100), (64, 3, 20000, 700), (256, 2, 10000, 90)])
def test_attn_kv8_one_head_on_the_whole_gpu(S, D, group, n, tokens):
    """Every CTA has a part of a few triples: hundreds of partial sums."""
    page, gen = 128, torch.Generator(device="cuda").manual_seed(D + tokens)
    pages = -(-n // page)
    cache = torch.full((pages, S.spdp_kv8_page_bytes(1, D, page)), 0xFF, dtype=torch.uint8, device="cuda")
    table = torch.randperm(pages, generator=gen, device="cuda")[None].int()
    k, v = (torch.randn(n, 1, D, generator=gen, device="cuda").half() for _ in range(2))
    v[: n // 2] *= 4.0
    kv, vv = torch.empty_like(k), torch.empty_like(v)
    S.spdp_kv8_store(k, v, cache, page, table, ints(n), first=ints(0, n), k_values=kv, v_values=vv)
    q, y = torch.randn(tokens, group, D, generator=gen, device="cuda").half(), torch.empty(tokens, group * D, dtype=torch.float16, device="cuda")
    S.spdp_attn_kv8(q, cache, page, 1, table, ints(n), y, 0.3, first=ints(0, tokens))
    seen = torch.arange(n, device="cuda") <= torch.arange(n - tokens, n, device="cuda")[:, None]
    device_check(y, q, kv.double().transpose(0, 1), vv.double().transpose(0, 1), seen, 0.3, 7.0, 28.0)
    again = torch.empty_like(y)
    S.spdp_attn_kv8(q, cache, page, 1, table, ints(n), again, 0.3, first=ints(0, tokens))
    assert torch.equal(y, again)


@pytest.mark.parametrize("window,sinks", [(0, 0), (40, 4)])
def test_attn_kv8_many_requests(S, window, sinks):
    """More triples than CTAs, most of a few tokens, some of none, some long."""
    heads, group, D, page, B = 4, 2, 64, 16, 700
    rng = np.random.default_rng(9)
    counts = rng.integers(0, 3, B)
    counts[::97] = 70
    length = counts + rng.integers(0, 3, B) * (counts > 0)
    length[::51] += 200
    each, most = 20, int(length.max())
    assert most <= each * page
    gen = torch.Generator(device="cuda").manual_seed(9)
    table = torch.randperm(B * each, generator=gen, device="cuda").view(B, each).int()
    cache = torch.full((B * each, S.spdp_kv8_page_bytes(heads, D, page)), 0xFF, dtype=torch.uint8, device="cuda")
    k, v = (torch.randn(int(length.sum()), heads, D, generator=gen, device="cuda").half() for _ in range(2))
    kv, vv = torch.empty_like(k), torch.empty_like(v)
    S.spdp_kv8_store(k, v, cache, page, table, dev(length.astype(np.int32)), first=dev(starts(length)), k_values=kv, v_values=vv)
    N = int(counts.sum())
    q = torch.randn(N, heads * group, D, generator=gen, device="cuda").half()
    y = torch.full((N, heads * group * D), 3.0, dtype=torch.float16, device="cuda")
    S.spdp_attn_kv8(q, cache, page, heads, table, dev(length.astype(np.int32)), y, 0.125, first=dev(starts(counts)), window=window, sinks=sinks)
    for b in range(0, B, 3):
        if counts[b] == 0:
            continue
        T, n = int(length[b]), int(counts[b])
        mine, keys = slice(starts(counts)[b], starts(counts)[b + 1]), slice(starts(length)[b], starts(length)[b + 1])
        i, j = torch.arange(T - n, T, device="cuda")[:, None], torch.arange(T, device="cuda")
        seen = (j <= i) & ((i - j < window) | (j < sinks) if window else True)
        device_check(y[mine], q[mine], kv[keys].double().transpose(0, 1), vv[keys].double().transpose(0, 1), seen, 0.125, 7.0, 7.0)


def test_attn_kv8_captured_and_on_streams(S):
    """Two graphs and eager calls, one after another and at once, of single tokens and of prompts: each call's scratch memory is its own."""
    rng = np.random.default_rng(6)
    cases = []
    for counts, length in (([1, 1, 1], [300, 17, 90]), ([1, 2, 80], [1000, 17, 90]), ([150, 90, 1], [700, 90, 200])):
        table, oracle = filled(rng, 2, 128, 16, length)
        first, N = starts(counts), sum(counts)
        q, y = dev(rng.standard_normal((N, 8, 128)).astype(np.float16)), torch.empty(N, 1024, dtype=torch.float16, device="cuda")
        cases.append(dict(q=q, y=y, raw=dev(oracle.raw), table=table, tab=dev(np.concatenate([table, np.full((3, 600), -1, np.int32)], 1)), first=first, length=length, oracle=oracle,
                          dfirst=dev(first), dlength=ints(*length)))

    def call(c):
        S.spdp_attn_kv8(c["q"], c["raw"], 16, 2, c["tab"], c["dlength"], c["y"], 0.1, first=c["dfirst"])
    graphs, streams = [], [torch.cuda.Stream() for _ in cases]
    for c in cases:
        call(c)
        attn_check(c["y"], c["q"], c["oracle"], c["table"], c["first"], c["length"], 0.1)
        c["want"] = c["y"].clone()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            call(c)
        graphs.append(g)
    torch.cuda.synchronize()
    for i in range(20):
        for c, s, g in zip(cases, streams, graphs):
            with torch.cuda.stream(s):
                c["y"].fill_(7.0)
                if i % 2:
                    g.replay()
                else:
                    call(c)
        torch.cuda.synchronize()
        for c in cases:
            assert torch.equal(c["y"], c["want"])
    del graphs


# ---- pages ------------------------------------------------------------------------------------------------------------------

def page_state(rng, rows, table_pages, pages, layers=2, page_bytes=48, used=0.5):
    """Requests of random sizes on random pages; a few pages that are kept by nobody's row; padding between the rows of the table and between layers."""
    table, ref = np.full((rows, table_pages), -1), np.zeros(pages, int)
    free = list(rng.permutation(pages))
    for r in range(rows):
        for e in range(int(rng.integers(0, table_pages + 1))):
            if len(free) <= (1 - used) * pages:
                break
            table[r, e] = free.pop()
            ref[table[r, e]] = 1
    for _ in range(min(3, len(free))):
        ref[free.pop()] = 2
    want = O.Pages(table, ref, rng.integers(0, 256, (layers, pages, page_bytes), dtype=np.uint8))
    wide = torch.full((rows, table_pages + 3), 77, dtype=torch.int32, device="cuda")
    tab = wide[:, :table_pages].copy_(dev(table.astype(np.int32)))
    store = torch.full((layers, pages + 1, page_bytes), 9, dtype=torch.uint8, device="cuda")
    cache = store[:, :pages].copy_(dev(want.cache))
    return want, wide, tab, dev(ref.astype(np.int32)), store, cache


def same_state(want, wide, tab, ref, store, cache):
    torch.cuda.synchronize()
    assert np.array_equal(tab.cpu().numpy(), want.table) and np.array_equal(ref.cpu().numpy(), want.ref) and np.array_equal(cache.cpu().numpy(), want.cache)
    assert bool((wide[:, tab.shape[1]:] == 77).all()) and bool((store[:, cache.shape[1]:] == 9).all())


@pytest.mark.parametrize("rows,table_pages,pages", [(1, 1, 1), (5, 7, 40), (40, 3, 77), (300, 20, 5000), (3, 2000, 4000), (64, 300, 40000)])
def test_kv_pages_run_of_calls(S, rows, table_pages, pages):
    """Requests come, grow, fork, end, and the cache is brought together, again and again, also where pages run out."""
    rng = np.random.default_rng(rows + pages)
    state = page_state(rng, rows, table_pages, pages)
    want, wide, tab, ref, store, cache = state
    short = torch.full((1,), -9, dtype=torch.int32, device="cuda")
    for step in range(6):
        done = rng.permutation(rows)[:max(1, rows // 3)]
        args = [done, np.zeros(len(done), int) - 3, np.full(len(done), table_pages + 9)]
        want.free(*args)
        S.spdp_kv_pages_free(ref, tab, *[ints(*a.tolist()) for a in args])
        same_state(*state)
        empty = [int(r) for r in done]
        children, others = empty[:len(empty) // 2], [r for r in range(rows) if r not in empty]
        if others and children:
            parents = [int(r) for r in rng.choice(others, len(children))]
            lengths = [int(rng.integers(0, 16 * (want.table[p] >= 0).sum() + 1)) for p in parents]
            got = want.fork(parents, children, lengths)
            S.spdp_kv_pages_fork(cache, ref, tab, 16, ints(*parents), ints(*children), ints(*lengths), short)
            same_state(*state)
            assert int(short) == got
        grow = empty[len(children):] + [rows, -1]
        start, stop = [int(n) for n in rng.integers(-1, table_pages + 1, len(grow))], [int(n) for n in rng.integers(0, table_pages + 2, len(grow))]
        got = want.take(grow, start, stop)
        S.spdp_kv_pages_take(ref, tab, ints(*grow), ints(*start), ints(*stop), short)
        same_state(*state)
        assert int(short) == got
        if step % 2:
            live = want.compact()
            S.spdp_kv_pages_compact(cache, ref, tab, short)
            same_state(*state)
            assert int(short) == live


@pytest.mark.parametrize("page_bytes,layers,flat", [(16, 1, True), (16 * 129 * 2, 3, False), (16 * 8 * 257, 2, False), (40000, 1, True)])
def test_kv_pages_copy(S, page_bytes, layers, flat):
    rng = np.random.default_rng(page_bytes)
    want, wide, tab, ref, store, cache = page_state(rng, 2, 2, 50, layers, page_bytes)
    order = rng.permutation(50)
    src, dst = [*order[:20].tolist(), -1, 50, 2 ** 31 - 1, 3, int(order[45])], [*order[20:40].tolist(), int(order[40]), int(order[41]), int(order[42]), -2 ** 31, int(order[45])]
    want.copy(src, dst)
    S.spdp_kv_pages_copy(cache[0] if flat else cache, ints(*src), ints(*dst))
    same_state(want, wide, tab, ref, store, cache)
    S.spdp_kv_pages_copy(cache, ints(), ints())
    same_state(want, wide, tab, ref, store, cache)


def test_kv_pages_odd_tables_and_full_caches(S):
    """Entries that name no page, counts below 0, rows that do not exist, no free page at all, and every page free."""
    rng = np.random.default_rng(4)
    state = page_state(rng, 4, 5, 30)
    want, wide, tab, ref, store, cache = state
    want.table[1] = [30, -2 ** 31, 2 ** 31 - 1, -1, -1]
    want.ref[want.ref == 0] = rng.integers(-3, 1, int((want.ref == 0).sum()))
    tab.copy_(dev(want.table.astype(np.int32)))
    ref.copy_(dev(want.ref.astype(np.int32)))
    short = ints(-1)
    got = want.fork([1, 1, -1, 9], [2, 3, 2, 0], [70, 20, 5, 5])
    S.spdp_kv_pages_fork(cache, ref, tab, 16, ints(1, 1, -1, 9), ints(2, 3, 2, 0), ints(70, 20, 5, 5), short)
    same_state(*state)
    assert int(short) == got == 0
    want.free([1, 1], [0, 0], [5, 5])                         # an entry that is named twice
    S.spdp_kv_pages_free(ref, tab, ints(1, 1), ints(0, 0), ints(5, 5))
    same_state(*state)
    want.ref[:] = 1
    ref.fill_(1)
    got = want.take([0, 2], [0, 1], [5, 3])
    S.spdp_kv_pages_take(ref, tab, ints(0, 2), ints(0, 1), ints(5, 3), short)
    same_state(*state)
    assert int(short) == got == 7
    for n in (1, 0):
        want.ref[:] = n
        ref.fill_(n)
        live = want.compact()
        S.spdp_kv_pages_compact(cache, ref, tab, short)
        same_state(*state)
        assert int(short) == live == 30 * n
    short.fill_(5)
    S.spdp_kv_pages_take(ref, tab, ints(), ints(), ints(), short)
    assert int(short) == 0


def test_kv_pages_longest_row(S):
    """The last entries of a row of as many as a table may have."""
    most, count = 2 ** 31 - 1, 3000
    if torch.cuda.mem_get_info()[0] < 5 * most:
        pytest.skip("needs 11 GB of device memory")
    tab = torch.empty(1, most, dtype=torch.int32, device="cuda")
    ref, short = torch.zeros(4000, dtype=torch.int32, device="cuda"), ints(-1)
    tab[0, -count - 5:] = 17
    row, start, stop = ints(0), ints(most - count), ints(most)
    S.spdp_kv_pages_take(ref, tab, row, start, stop, short)
    torch.cuda.synchronize()
    assert int(short) == 0 and torch.equal(tab[0, -count:], torch.arange(count, dtype=torch.int32, device="cuda")) and int(ref.sum()) == count
    S.spdp_kv_pages_free(ref, tab, row, start, stop)
    torch.cuda.synchronize()
    assert bool((tab[0, -count:] == -1).all()) and bool((tab[0, -count - 5:-count] == 17).all()) and int(ref.abs().sum()) == 0
    del tab
    torch.cuda.empty_cache()


def test_kv_pages_captured(S):
    """A step's whole handling of pages in a graph, replayed on another state."""
    rng = np.random.default_rng(5)
    state = page_state(rng, 6, 6, 60)
    want, wide, tab, ref, store, cache = state
    row, start, stop, child, length, short, live, two, parent = ints(0, 1), ints(0, 0), ints(6, 6), ints(0, 1), ints(20, 16), ints(0), ints(0), ints(2, 2), ints(2, 3)

    def step():
        S.spdp_kv_pages_free(ref, tab, row, start, stop)
        S.spdp_kv_pages_fork(cache, ref, tab, 16, parent, child, length, short)
        S.spdp_kv_pages_take(ref, tab, row, two, stop, short)
        S.spdp_kv_pages_compact(cache, ref, tab, live)
    parents, lengths = [2, 3], [20, 16]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(4):
        graph.replay()
        want.free([0, 1], [0, 0], [6, 6])
        want.fork(parents, [0, 1], lengths)
        want.take([0, 1], [2, 2], [6, 6])
        assert want.compact() == int(live)
        same_state(*state)
        parents, lengths = parents[::-1], lengths[::-1]
        parent.copy_(parent.flip(0)), length.copy_(length.flip(0))
    del graph


# ---- together ---------------------------------------------------------------------------------------------------------------

def test_serving_with_forks_and_windows(S):
    """A prompt in two pieces, forked into three samples, single and double steps with a window and first tokens whose middle pages are freed, the cache brought
    together on the way: every token's attention against 64 bits over what the library says that its codes stand for."""
    heads, group, D, page, pages, layers, each = 2, 4, 64, 16, 64, 2, 12
    H, window, sinks, scale = heads * group, 40, 5, 0.15
    gen = torch.Generator(device="cuda").manual_seed(3)
    cache = torch.full((layers, pages, S.spdp_kv8_page_bytes(heads, D, page)), 0xFF, dtype=torch.uint8, device="cuda")
    ref, table, short = torch.zeros(pages, dtype=torch.int32, device="cuda"), torch.full((3, each), -1, dtype=torch.int32, device="cuda"), ints(0)
    ref[3::5] = 1                                            # others' pages
    kept = [[[torch.zeros(0, heads, D, dtype=torch.float64, device="cuda")] * 2 for _ in range(3)] for _ in range(layers)]
    length = [0, 0, 0]

    def step(rows, counts):
        first = starts(counts)
        S.spdp_kv_pages_take(ref, table, ints(*rows), ints(*[-(-length[r] // page) for r in rows]), ints(*[-(-(length[r] + n) // page) for r, n in zip(rows, counts)]), short)
        assert int(short) == 0
        for r, n in zip(rows, counts):
            length[r] += n
        tab, lengths = table[torch.tensor(rows, device="cuda")].contiguous(), ints(*[length[r] for r in rows])
        for layer in range(layers):
            N = int(first[-1])
            k, v, q = (torch.randn(N, h, D, generator=gen, device="cuda").half() for h in (heads, heads, H))
            kv, vv, y = torch.empty_like(k), torch.empty_like(v), torch.empty(N, H * D, dtype=torch.float16, device="cuda")
            S.spdp_kv8_store(k, v, cache[layer], page, tab, lengths, first=dev(first), k_values=kv, v_values=vv)
            S.spdp_attn_kv8(q, cache[layer], page, heads, tab, lengths, y, scale, first=dev(first), window=window, sinks=sinks)
            for i, r in enumerate(rows):
                part = slice(first[i], first[i + 1])
                kept[layer][r] = [torch.cat([a, b[part].double()]) for a, b in zip(kept[layer][r], (kv, vv))]
                ks, vs = (x.transpose(0, 1) for x in kept[layer][r])
                T, n = length[r], counts[i]
                a, b = torch.arange(T - n, T, device="cuda")[:, None], torch.arange(T, device="cuda")
                want, spread = exact_on_device(q[part], ks, vs, (b <= a) & ((a - b < window) | (b < sinks)), scale)
                # as device_check; a cell that grew rounded its other tokens' codes again: by 2^-10 of scales that double up to 2^-6, in keys (scores off by 2^-15 of q's sum, times scale, at
                # most) and values
                reach = scale * (q[part].double().abs().sum(-1) * 7.0)[..., None]
                moved = 2.0 ** -15
                bound = U * want.abs() * 1.01 + (U + 2 * (reach * 1120 * V + scale * q[part].double().abs().sum(-1)[..., None] * moved + 2.0 ** -20)) * 1.02 * spread + T * 2.0 ** -33 * 7.1 + moved + TINY
                err = (y[part].double().view_as(want) - want).abs()
                assert bool((err <= bound).all()), (layer, r, float((err - bound).max()))

    step([0], [50])
    step([0], [37])
    S.spdp_kv_pages_fork(cache, ref, table, page, ints(0, 0), ints(1, 2), ints(87, 87), short)
    assert int(short) == 0 and length[0] == 87
    for r in (1, 2):
        length[r] = 87
        for layer in range(layers):
            kept[layer][r] = list(kept[layer][0])
    for i in range(14):
        step([2, 0, 1], [1, 2, 1] if i % 3 else [1, 1, 1])
        gone = [max(1, (length[r] - window) // page) for r in range(3)]
        S.spdp_kv_pages_free(ref, table, ints(0, 1, 2), ints(1, 1, 1), ints(*gone))
        if i == 6:
            live = ints(0)
            S.spdp_kv_pages_compact(cache, ref, table, live)
            assert int(live) == int((ref > 0).sum()) and bool((ref[:int(live)] > 0).all())
    named = table[table >= 0].long()
    assert bool((torch.bincount(named, minlength=pages)[named] == ref[named]).all()) and int((ref > 0).sum()) < pages // 2 + 13
