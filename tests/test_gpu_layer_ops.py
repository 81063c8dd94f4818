"""The operators around the packed projections on the GPU against the 64-bit oracle, at the sizes, masks, strides and values where
they can go wrong, and a decode step that runs them together with the packed products.

Tolerances.  u = 2^-11 is half a step of fp16, v = 2^-24 half a step of fp32.  One product of the tensor cores adds 16 terms with
at most 2 v of the sum of their sizes lost at each of 17 additions."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import layer_ops as O
from oracle import spdp_oracle as SO
from paper_2607_21985_b200 import workloads as WL

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


def host(t):
    return t.cpu().numpy().astype(np.float64)


def replayed(call, inputs, outputs):
    """Outputs of a captured call, replayed after its inputs were overwritten and put back (eager calls before and between)."""
    kept = [t.clone() for t in inputs]
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for t, k in zip(inputs, kept):
        t.copy_(k)
    graph.replay()
    torch.cuda.synchronize()
    first = [t.clone() for t in outputs]
    for t, k in zip(inputs, kept):
        t.copy_(k)
    call()
    for t, k in zip(inputs, kept):
        t.copy_(k)
    graph.replay()
    torch.cuda.synchronize()
    for a, b in zip(first, outputs):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
    del graph
    return first


# ---- adapters ---------------------------------------------------------------------------------------------------------------

def lora_bound(y, t_part, b_part, K, rank, f32):
    """The vector between the products: 17 additions a step, K / 1024 steps of a warp, 16 additions of warps and CTAs, all at 2 v of the sizes;
    one rounding of it (u, or u^2 in two numbers); the second product (17 additions a step of 32 ranks, twice as many in two numbers); the result."""
    steps = 17 * (K // 1024 + 1) + 16
    second = 2 * 17 * 2 * (rank // 32 + 1)
    out = V if f32 else U
    return (steps * 2 * V) * t_part + ((4 * U * U if f32 else U) + second * 2 * V + 4 * V) * b_part + out * np.abs(y) * 1.01 + (0 if f32 else TINY)


def lora_case(seed, N, K, M, rank, count, f32=False, odd_rows=False, ranks=True, none=0.25):
    rng = np.random.default_rng(seed)
    adapter = rng.integers(0, count, N).astype(np.int32)
    adapter[rng.random(N) < none] = rng.choice([-1, count, -2 ** 31, 2 ** 31 - 1])
    wide = (lambda n: n + 3) if odd_rows else (lambda n: (n + 7) // 8 * 8)
    X = np.zeros((N, wide(K)), np.float16)
    X[:, :K] = rng.standard_normal((N, K))
    A = (rng.standard_normal((count, rank, wide(K))) / np.sqrt(K)).astype(np.float16)
    B = (rng.standard_normal((count, M, wide(rank))) * 0.2).astype(np.float16)
    c = dict(X=dev(X)[:, :K], adapter=dev(adapter), A=dev(A)[..., :K], B=dev(B)[..., :rank], scales=dev((rng.random(count) * 2 - 0.5).astype(np.float32)),
             base=torch.zeros(N, wide(M), dtype=torch.float32 if f32 else torch.float16, device="cuda"))
    c["base"] = c["base"].copy_(dev(rng.standard_normal((N, wide(M))).astype(np.float32)))[:, :M]
    r = rng.integers(0, rank + 1, count).astype(np.int32) if ranks else None
    c["ranks"] = dev(r) if ranks else None
    return c


def lora_check(c, Y, rank):
    ranks = None if c["ranks"] is None else c["ranks"].cpu().numpy()
    scales = None if c["scales"] is None else c["scales"].cpu().numpy()
    y, t_part, b_part = O.lora(host(c["X"]), c["adapter"].cpu().numpy(), host(c["A"]), host(c["B"]), host(c["base"]), scales, ranks)
    f32 = Y.dtype == torch.float32
    err = np.abs(host(Y) - y)
    assert np.all(err <= lora_bound(y, t_part, b_part, c["X"].shape[1], rank, f32)), float((err - lora_bound(y, t_part, b_part, c["X"].shape[1], rank, f32)).max())
    a = c["adapter"]
    none = (a < 0) | (a >= c["A"].shape[0])
    assert torch.equal(Y[none].contiguous().view(torch.uint8), c["base"][none].contiguous().view(torch.uint8))


SIZES = [(1, 1, 1, 1, 1), (1, 64, 64, 8, 1), (1, 4096, 256, 16, 3), (2, 31, 4200, 17, 2), (8, 257, 130, 5, 4), (9, 1000, 65, 32, 9), (33, 100, 65, 20, 3), (32, 512, 4097, 16, 32),
         (70, 1000, 300, 64, 5), (5, 300, 77, 100, 2), (3, 40, 9, 256, 2), (300, 128, 1, 1, 2), (40, 8200, 70, 33, 4), (2100, 64, 96, 16, 7), (64, 2048, 640, 128, 64),
         (8, 256, 4608, 64, 8), (16, 1024, 640, 32, 3), (13, 64, 8200, 256, 2), (16, 2048, 64, 16, 30), (4, 320, 20000, 24, 2), (17, 512, 128, 8, 5), (512, 96, 64, 72, 300), (513, 96, 64, 40, 300)]


@pytest.mark.parametrize("f32", [False, True])
@pytest.mark.parametrize("odd_rows", [False, True])
@pytest.mark.parametrize("N,K,M,rank,count", SIZES)
def test_lora(S, N, K, M, rank, count, odd_rows, f32):
    c = lora_case(N + K + M, N, K, M, rank, count, f32, odd_rows)
    guard = torch.full((N + 2, M + 5), 77.0, dtype=c["base"].dtype, device="cuda")
    Y = guard[1:N + 1, 2:M + 2]
    S.spdp_lora(Y=Y, **c)
    torch.cuda.synchronize()
    lora_check(c, Y, rank)
    guard[1:N + 1, 2:M + 2] = 77.0
    assert bool((guard == 77.0).all())
    # in place, twice the same bits
    for _ in range(2):
        Z = c["base"].clone()
        S.spdp_lora(**dict(c, Y=Z, base=None))
        lora_check(c, Z, rank)
        if _:
            assert torch.equal(Z, first)
        first = Z


@pytest.mark.parametrize("f32", [False, True])
@pytest.mark.parametrize("N,count,run", [(256, 300, 1), (257, 2, 1), (600, 31, 1), (1030, 9, 7), (700, 3, 100), (512, 1, 1), (90, 90, 1)])
def test_lora_tokens_of_many_adapters(S, N, count, run, f32):
    """Windows of tokens with as many adapters as tokens, with few that alternate, with runs across their borders."""
    K, M, rank = 72, 136, 24
    c = lora_case(N + count, N, K, M, rank, count, f32)
    c["adapter"] = c["adapter"][::run].repeat_interleave(run)[:N].contiguous()
    Y = torch.full_like(c["base"], 99.0)
    S.spdp_lora(Y=Y, **c)
    lora_check(c, Y, rank)
    Z = c["base"].clone()
    S.spdp_lora(**dict(c, Y=Z, base=None))
    assert torch.equal(Z, Y)


@pytest.mark.parametrize("none", [0.0, 1.0])
def test_lora_all_or_none(S, none):
    c = lora_case(5, 45, 96, 200, 12, 3, none=none, ranks=False)
    c["scales"] = None
    Y = torch.empty_like(c["base"])
    S.spdp_lora(Y=Y, **c)
    lora_check(c, Y, 12)
    # a single token as vectors
    y = c["base"][7].clone()
    S.spdp_lora(c["X"][7], c["adapter"][7:8], c["A"], c["B"], y)
    assert (y.double() - Y[7].double()).abs().max() <= 2 * U * Y[7].double().abs().max()


def test_lora_leaves_out_what_is_not_the_tokens(S):
    """NaN and Inf in weights behind an adapter's rank, in other adapters and in other tokens reach nobody."""
    c = lora_case(11, 40, 200, 150, 24, 4, none=0.0)
    c["ranks"] = dev(np.array([24, 7, 0, 9], np.int32))
    for a, r in enumerate([24, 7, 0, 9]):
        c["A"][a, r:] = float("nan")
        c["B"][a, :, r:] = float("inf")
    clean = dict(c, A=c["A"].nan_to_num(0.0), B=c["B"].nan_to_num(0.0, 0.0, 0.0))
    Y = torch.empty_like(c["base"])
    S.spdp_lora(Y=Y, **c)
    lora_check(clean, Y, 24)
    bad = 13
    c["X"][bad, 3] = float("nan")
    Z = torch.empty_like(c["base"])
    S.spdp_lora(Y=Z, **c)
    others = torch.arange(40, device="cuda") != bad
    assert torch.equal(Z[others], Y[others])
    assert int(c["adapter"][bad]) == 2 or bool(Z[bad].isnan().all())
    c["X"][bad, 3] = 0.0
    c["A"][0, 0, 0] = float("inf")
    S.spdp_lora(Y=Z, **c)
    others &= c["adapter"] != 0
    assert torch.equal(Z[others], Y[others])


@pytest.mark.parametrize("size", [2.0 ** -20, 2.0 ** 12])
def test_lora_range_between_the_products(S, size):
    """Vectors between the products far below and above fp16's range."""
    c = lora_case(12, 20, 256, 128, 8, 2, f32=True, none=0.0, ranks=False)
    c["A"].mul_(size)
    c["X"].mul_(8.0)
    if size < 1:
        c["A"].copy_((c["A"] * 2.0 ** 6).round() / 2.0 ** 6 + 2.0 ** -24)                 # subnormals
    c["scales"].fill_(0.25 if size > 1 else 4.0)
    Y = torch.empty_like(c["base"])
    S.spdp_lora(Y=Y, **c)
    lora_check(c, Y, 8)


def test_lora_captured_and_on_streams(S):
    c = lora_case(13, 50, 512, 700, 16, 5)
    Y = c["base"].clone()
    first, = replayed(lambda: S.spdp_lora(**dict(c, Y=Y, base=None)), [Y], [Y])
    lora_check(c, first, 16)
    others = [lora_case(20 + i, 40, 512, 700, 16, 5) for i in range(2)]
    streams, outs = [torch.cuda.Stream() for _ in others], [torch.empty_like(o["base"]) for o in others]
    torch.cuda.synchronize()
    for _ in range(10):
        for o, s, y in zip(others, streams, outs):
            with torch.cuda.stream(s):
                S.spdp_lora(Y=y, **o)
    torch.cuda.synchronize()
    for o, y in zip(others, outs):
        lora_check(o, y, 16)


# ---- head norms and rotation ------------------------------------------------------------------------------------------------

def heads_check(x, y, weight, eps, pos, freq, sections, adjacent):
    """Sum of squares: D / 2 additions and the root, 8 v in all on x / rms (256 squares at most in 16 chains); two products by the sine and cosine, whose angle is off by
    4 v turns (8 pi v radians) and whose values by 4 v; the rounding."""
    want, size = O.norm_rope(host(x), None if weight is None else host(weight), eps, pos, freq, sections, adjacent)
    err = np.abs(host(y) - want)
    assert np.all(err <= U * np.abs(want) * 1.01 + 64 * V * size + TINY), float((err / (size + 1e-9)).max())


@pytest.mark.parametrize("pad", [5, 8])            # rows that start anywhere, and on 16-byte boundaries
@pytest.mark.parametrize("N,q_heads,kv_heads,D,pairs,axes,adjacent,f32,norm", [
    (1, 1, 0, 2, 1, 1, False, False, True), (1, 32, 32, 128, 64, 1, False, False, True), (5, 3, 1, 64, 20, 2, True, False, True), (7, 12, 3, 64, 32, 3, False, True, True),
    (3, 8, 2, 256, 128, 4, False, False, True), (2, 5, 5, 250, 99, 2, False, True, True), (33, 2, 1, 80, 40, 1, True, True, False), (4, 9, 1, 96, 16, 1, False, False, True),
    (130, 64, 8, 128, 48, 3, False, True, True), (6, 4, 4, 128, 0, 0, False, False, True), (1, 1, 1, 6, 3, 1, True, True, True), (700, 16, 2, 128, 64, 1, False, False, False),
    (2, 100, 7, 34, 17, 2, False, False, True)])
def test_qk_norm_rope(S, N, q_heads, kv_heads, D, pairs, axes, adjacent, f32, norm, pad):
    rng = np.random.default_rng(N + D + pairs)
    qkv = dev((rng.standard_normal((N, (q_heads + 2 * kv_heads) * D + 8)) * 3).astype(np.float32 if f32 else np.float16))
    q, k = qkv[:, :q_heads * D].view(N, q_heads, D), qkv[:, q_heads * D:(q_heads + kv_heads) * D].view(N, kv_heads, D) if kv_heads else None
    pos = rng.integers(-50, 2 ** 20, (max(axes, 1), N)).astype(np.int32)
    freq = (500000.0 ** (-np.arange(pairs) / max(pairs, 1))).astype(np.float32) if pairs else None
    cuts = np.sort(rng.integers(0, pairs + 1, max(axes, 1) - 1))
    sections = tuple(int(v) for v in np.diff([0, *cuts, pairs]))
    qw, kw = (dev((1 + 0.2 * rng.standard_normal(D)).astype(np.float16)) for _ in range(2)) if norm else (None, None)
    q_all = torch.full((N, q_heads * D + pad), 7.0, dtype=torch.float16, device="cuda")
    q_out = q_all[:, :q_heads * D].view(N, q_heads, D)
    k_out = torch.empty(N, kv_heads, D, dtype=torch.float16, device="cuda") if kv_heads else None
    S.spdp_qk_norm_rope(q, k, q_out, k_out, dev(pos if axes != 1 else pos[0]) if pairs else None, dev(freq) if pairs else None, sections, qw, kw, 1e-5, adjacent)
    torch.cuda.synchronize()
    heads_check(q, q_out, qw, 1e-5, pos, freq, sections, adjacent)
    assert bool((q_all[:, q_heads * D:] == 7.0).all())
    if kv_heads:
        heads_check(k, k_out, kw, 1e-5, pos, freq, sections, adjacent)
    if not f32:                          # in place
        q2 = q.clone()
        S.spdp_qk_norm_rope(q2, None, q2, None, dev(pos) if pairs else None, dev(freq) if pairs else None, sections, qw, None, 1e-5, adjacent)
        heads_check(q, q2, qw, 1e-5, pos, freq, sections, adjacent)


def test_qk_norm_rope_far_positions_zeros_and_misaligned(S):
    """Positions to the end of 32 bits, heads of zeros, and rows that start anywhere give what aligned ones give."""
    N, H, D = 9, 3, 128
    rng = np.random.default_rng(3)
    x = rng.standard_normal((N, H, D)).astype(np.float16)
    x[2] = 0
    pos = np.array([0, 1, -1, 2 ** 31 - 1, -2 ** 31, 131072, 10 ** 6, 999999999, 7], np.int32)
    freq = (10000.0 ** (-np.arange(64) / 64)).astype(np.float32)
    w = dev((1 + 0.2 * rng.standard_normal(D)).astype(np.float16))
    q, out = dev(x), torch.empty(N, H, D, dtype=torch.float16, device="cuda")
    S.spdp_qk_norm_rope(q, None, out, None, dev(pos), dev(freq), q_weight=w)
    heads_check(q, out, w, 1e-6, pos[None], freq, (64,), False)
    assert bool((out[2] == 0).all())
    odd = torch.empty(N * (H * D + 1) + 1, dtype=torch.float16, device="cuda")[1:].view(N, H * D + 1)[:, :H * D].view(N, H, D)
    odd.copy_(q)
    out2 = torch.empty_like(out)
    S.spdp_qk_norm_rope(odd, None, out2, None, dev(pos), dev(freq), q_weight=w)
    heads_check(q, out2, w, 1e-6, pos[None], freq, (64,), False)


def test_qk_norm_rope_captured(S):
    q, out = torch.randn(20, 4, 64, device="cuda").half(), torch.empty(20, 4, 64, dtype=torch.float16, device="cuda")
    pos, freq = torch.arange(20, dtype=torch.int32, device="cuda"), torch.rand(32, device="cuda")
    first, = replayed(lambda: S.spdp_qk_norm_rope(q, None, out, None, pos, freq), [q], [out])
    heads_check(q, first, None, 0.0, pos.cpu().numpy()[None], freq.cpu().numpy(), (32,), False)


# ---- the 4-bit cache --------------------------------------------------------------------------------------------------------

def same_bytes(got, want):
    return np.array_equal(got.cpu().numpy(), want)


@pytest.mark.parametrize("N,heads,D,page,f32,misaligned", [(1, 1, 64, 16, False, False), (5, 3, 128, 16, True, False), (40, 2, 256, 32, False, False), (77, 8, 128, 64, True, True),
                                                           (33, 1, 64, 128, False, True), (300, 5, 64, 256, True, False)])
def test_kv4_store(S, N, heads, D, page, f32, misaligned):
    rng = np.random.default_rng(N)
    pages = -(-N // page) + 3
    raw = rng.integers(0, 256, (pages, heads * page * (D + D // 8)), dtype=np.uint8)         # everything else stays as it was
    k = rng.standard_normal((N, heads, D)).astype(np.float16)
    v = (rng.standard_normal((N, heads, D)) * 10.0 ** rng.integers(-9, 4, (N, heads, 1))).astype(np.float32 if f32 else np.float16)
    k[0, 0, :32] = 0
    k[N // 2, 0, :4] = [65504, -65504, 2.5 * 9360, -3.5 * 9360]
    slot = rng.permutation(pages * page)[:N].astype(np.int64)
    if N > 4:
        slot[1], slot[2], slot[3] = -1, pages * page, 2 ** 40
    want = O.Kv4Cache(raw.copy(), heads, D, page)
    for n in range(N):
        want.store(slot[n], k[n], v[n].astype(np.float16))

    def placed(a):
        if not misaligned:
            return dev(a)
        t = torch.zeros(N, heads * D + 3, dtype=torch.from_numpy(a).dtype, device="cuda")[:, 1:heads * D + 1].unflatten(1, (heads, D))
        return t.copy_(dev(a))
    cache = dev(raw)
    kv, vv = (torch.empty(N, heads, D, dtype=torch.float16, device="cuda") for _ in range(2))
    S.spdp_kv4_store(placed(k), placed(v), dev(slot), cache, page, k_values=kv, v_values=vv)
    torch.cuda.synchronize()
    assert same_bytes(cache, want.raw)
    for got, x in ((kv, k), (vv, v.astype(np.float16))):
        with np.errstate(over="ignore"):             # 7 times the scale of 65504 is past fp16
            values = O.kv4_values(*O.kv4_codes(x)).astype(np.float16)
        assert np.array_equal(got.cpu().numpy(), values)
    again = dev(raw)
    S.spdp_kv4_store(placed(k), placed(v), dev(slot), again, page)
    assert torch.equal(again, cache)


def filled(rng, heads, D, page, lengths, spare=2):
    """A cache of garbage (NaN scales among it) with the keys of each request in shuffled pages; (cache, table, oracle)."""
    each = max(1, max(-(-n // page) for n in lengths))
    pages = each * len(lengths) + spare
    raw = rng.integers(0, 256, (pages, heads * page * (D + D // 8)), dtype=np.uint8)
    raw[rng.random(raw.shape) < 0.3] = 0xFF
    table = rng.permutation(pages)[:each * len(lengths)].reshape(len(lengths), each).astype(np.int32)
    cache = O.Kv4Cache(raw, heads, D, page)
    for b, n in enumerate(lengths):
        for t in range(n):
            cache.store(int(table[b, t // page]) * page + t % page, (rng.standard_normal((heads, D)) * 1.5).astype(np.float16),
                        (rng.standard_normal((heads, D)) * rng.choice([0.01, 1.0, 30.0])).astype(np.float16))
    return dev(raw), table, cache


def attn_check(y, q, cache, table, length, scale, cap=0.0, window=0, most=150.0):
    """Scores: 8 products of 17 additions at 2 v of the sizes and 4 more sums; a cap adds 8 v of itself.  Weights: twice the scores' error, 2^-21 for the exponential, one
    rounding u and, where small, half of fp16's smallest step against a weight of at least 1; values: one rounding u; the result.  `most`: no value is larger (150: 30 standard
    deviations' worth of the largest rows)."""
    for b in range(len(length)):
        want, spread, reach, keys = O.attention(host(q[b]), cache, table[b], int(length[b]), scale, cap, window)
        ds = (2 * 2 * V * (17 * 16 + 8) * reach + 8 * V * cap + 2.0 ** -21)[:, None]
        bound = U * np.abs(want) * 1.01 + (2 * U + 2 * ds) * 1.01 * spread + keys * TINY * most + TINY
        err = np.abs(host(y[b]).reshape(want.shape) - want)
        assert np.all(err <= bound), (b, int(length[b]), float((err - bound).max()))


@pytest.mark.parametrize("columns", [2, 1000])     # of the table behind the longest request's: with 1000 the keys may be too many for one cluster
@pytest.mark.parametrize("heads,group,D,page,lengths,cap,window", [
    (1, 1, 128, 16, [1], 0.0, 0), (2, 4, 128, 16, [0, 1, 15, 16, 17], 0.0, 0), (1, 8, 64, 32, [63, 64, 65, 0, 130], 0.0, 0), (3, 3, 128, 64, [200, 3, 64, 128], 20.0, 0),
    (1, 9, 128, 16, [100, 33], 0.0, 0), (2, 16, 64, 16, [70, 1, 300], 5.0, 50), (1, 20, 128, 128, [129, 257], 0.0, 1), (2, 2, 256, 256, [40, 300], 0.0, 17),
    (1, 12, 256, 16, [90, 16], 30.0, 0), (1, 33, 64, 16, [50], 0.0, 16), (4, 1, 128, 32, [700, 5, 0, 31, 32, 33, 64, 1], 0.0, 100)])
def test_attn_kv4(S, heads, group, D, page, lengths, cap, window, columns):
    rng = np.random.default_rng(heads * 100 + group + D)
    cache, table, oracle = filled(rng, heads, D, page, lengths)
    B, H = len(lengths), heads * group
    q = dev(rng.standard_normal((B, H * D + 4)).astype(np.float16))[:, :H * D].unflatten(1, (H, D))
    length = np.array(lengths, np.int32)
    if B > 4:
        length[0] = -5 if length[0] == 0 else length[0]
    y_all = torch.full((B + 1, H * D + 3), 9.0, dtype=torch.float16, device="cuda")
    words = H * D // 32
    mask = torch.full((B + 1, words + 1), 123, dtype=torch.int32, device="cuda")
    y, scale, thr = y_all[:B, :H * D], 1.3 / np.sqrt(D), 0.05
    tab = dev(np.concatenate([table, np.full((B, columns), -7, np.int32)], 1))
    S.spdp_attn_kv4(q, cache, page, heads, tab, dev(length), y, scale, cap=cap, window=window, thr=thr, mask=mask[:B])
    torch.cuda.synchronize()
    attn_check(y, q, oracle, table, length, scale, cap, window)
    assert bool((y_all[B] == 9.0).all()) and bool((y_all[:, H * D:] == 9.0).all()) and bool((mask[B] == 123).all()) and bool((mask[:, words:] == 123).all())
    keep = ~(y.float().abs() <= thr)
    bits = mask[:B, :words].cpu().numpy().view(np.uint32)
    assert np.array_equal((bits[:, :, None] >> np.arange(32, dtype=np.uint32) & 1).reshape(B, -1).astype(bool), keep.cpu().numpy())
    for b, n in enumerate(length):
        if n <= 0:
            assert bool((y[b] == 0).all())
    first = y.clone()
    S.spdp_attn_kv4(q, cache, page, heads, tab, dev(length), y, scale, cap=cap, window=window)
    assert torch.equal(first, y)


@pytest.mark.parametrize("columns", [5, 600])
def test_attn_kv4_pages_that_do_not_exist_and_lengths_beyond_the_table(S, columns):
    rng = np.random.default_rng(8)
    cache, table, oracle = filled(rng, 2, 128, 16, [80, 80, 40])
    table[0, 1], table[0, 3], table[1, :] = -1, 2 ** 31 - 1, len(oracle.raw)
    table = np.concatenate([table, np.full((3, columns - 5), len(oracle.raw) + 3, np.int32)], 1)
    length = np.array([80, 80, 10 ** 9], np.int32)
    for t in range(40, 80):
        oracle.store(int(table[2, t // 16]) * 16 + t % 16, np.ones((2, 128), np.float16), np.ones((2, 128), np.float16))
    cache = dev(oracle.raw)
    q, y = dev(rng.standard_normal((3, 4, 128)).astype(np.float16)), torch.empty(3, 512, dtype=torch.float16, device="cuda")
    S.spdp_attn_kv4(q, cache, 16, 2, dev(table), dev(length), y, 0.1)
    attn_check(y, q, oracle, table, length, 0.1)
    assert bool((y[1] == 0).all())


@pytest.mark.parametrize("columns", [0, 600])
def test_attn_kv4_scores_of_all_sizes(S, columns):
    """Scores that grow along the keys, fall, and lie far apart: the running maximum, and weights down to nothing."""
    rng = np.random.default_rng(9)
    heads, D, page, n = 1, 128, 16, 200
    cache, table, oracle = filled(rng, heads, D, page, [n, n, n])
    for b, size in enumerate([lambda t: t / 4, lambda t: (n - t) / 4, lambda t: 100.0 * (t % 7 == 3)]):
        for t in range(n):
            k = np.zeros((1, D), np.float16)
            k[0, 5] = size(t)
            oracle.store(int(table[b, t // page]) * page + t % page, k, rng.standard_normal((1, D)).astype(np.float16))
    q = np.zeros((3, 2, D), np.float16)
    q[:, 0, 5], q[:, 1, 5] = 8.0, -3.0
    y = torch.empty(3, 2 * D, dtype=torch.float16, device="cuda")
    S.spdp_attn_kv4(dev(q), dev(oracle.raw), page, heads, dev(np.concatenate([table, np.zeros((3, columns), np.int32)], 1)), dev(np.full(3, n, np.int32)), y, 0.125)
    attn_check(y, dev(q), oracle, table, [n] * 3, 0.125)


@pytest.mark.parametrize("sizes", [(2e-4,), (6e4,), (1e-3, 3e4), (3e4, 1e-3)])
def test_attn_kv4_values_of_all_sizes(S, sizes):
    """Values near both ends of fp16's range; large ones in the second half of the keys, and in the first."""
    rng = np.random.default_rng(10)
    heads, D, page, n = 1, 64, 16, 400
    cache, table, oracle = filled(rng, heads, D, page, [n])
    for t in range(n):
        size = sizes[len(sizes) * t // n]
        oracle.store(int(table[0, t // page]) * page + t % page, rng.standard_normal((1, D)).astype(np.float16), (size * rng.uniform(-1, 1, (1, D))).astype(np.float16))
    q, y = dev(rng.standard_normal((1, 3, D)).astype(np.float16)), torch.empty(1, 3 * D, dtype=torch.float16, device="cuda")
    S.spdp_attn_kv4(q, dev(oracle.raw), page, heads, dev(table), dev(np.array([n], np.int32)), y, 0.2)
    attn_check(y, q, oracle, table, [n], 0.2, most=max(sizes))


@pytest.mark.parametrize("columns", [0, 600])
def test_attn_kv4_caps_that_leave_nothing_of_the_scores(S, columns):
    """A cap whose reciprocal is beyond 32 bits: all scores are 0 or as good as 0, whether the products are 0 or not."""
    rng = np.random.default_rng(11)
    cache, table, oracle = filled(rng, 1, 64, 16, [40])
    q, y = dev(np.stack([np.zeros(64), rng.standard_normal(64)])[None].astype(np.float16)), torch.empty(1, 128, dtype=torch.float16, device="cuda")
    S.spdp_attn_kv4(q, cache, 16, 1, dev(np.concatenate([table, np.zeros((1, columns), np.int32)], 1)), dev(np.array([40], np.int32)), y, 0.1, cap=1e-40)
    attn_check(y, q * 0, oracle, table, [40], 0.1)


def plain_attention(q, k, v, scale):
    """In 64 bits on the device: q [H][D], k and v [kv heads][keys][D]."""
    z = torch.einsum("hgd,htd->hgt", q.double().unflatten(0, (k.shape[0], -1)), k) * scale
    return torch.einsum("hgt,htd->hgd", torch.softmax(z, -1), v).flatten(0, 1)


def test_attn_kv4_long_and_behind_four_gigabytes(S):
    """A long request among short ones, in pages whose addresses pass 32 bits; stored by the library itself."""
    heads, group, D, page = 2, 8, 128, 64
    per = S.spdp_kv4_page_bytes(heads, D, page)
    pages = (5 << 30) // per
    cache = torch.full((pages, per), 0xFF, dtype=torch.uint8, device="cuda")
    lengths = [20000, 1, 700]
    each = -(-lengths[0] // page)
    gen = torch.Generator(device="cuda").manual_seed(4)
    table = (pages - 1 - torch.randperm(each * 3, generator=gen, device="cuda")).view(3, each).int()
    table[0, 5] = 0
    ks, vs = [], []
    for b, n in enumerate(lengths):
        t = torch.arange(n, device="cuda")
        k, v = (torch.randn(n, heads, D, generator=gen, device="cuda").half() for _ in range(2))
        kv, vv = torch.empty_like(k), torch.empty_like(v)
        S.spdp_kv4_store(k, v, table[b, t // page].long() * page + t % page, cache, page, k_values=kv, v_values=vv)
        ks.append(kv.double().transpose(0, 1)), vs.append(vv.double().transpose(0, 1))
    q = torch.randn(3, heads * group, D, generator=gen, device="cuda").half()
    y = torch.empty(3, heads * group * D, dtype=torch.float16, device="cuda")
    S.spdp_attn_kv4(q, cache, page, heads, table, torch.tensor(lengths, dtype=torch.int32, device="cuda"), y, 0.125)
    for b in range(3):
        want = plain_attention(q[b], ks[b], vs[b], 0.125)
        spread = plain_attention(q[b], ks[b], vs[b].abs(), 0.125)
        # as in attn_check; the values that went back were rounded to fp16 once (keys: u of the scores' reach, at most 0.125 * 128 * 20)
        reach = 0.125 * (q[b].double().abs().sum(-1) * 6.0)[:, None]
        bound = U * want.abs() * 1.01 + (3 * U + 2 * reach * (U + 560 * V) + 2.0 ** -20) * 1.02 * spread + lengths[b] * TINY * 6.0 + TINY
        err = (y[b].double().view_as(want) - want).abs()
        assert bool((err <= bound).all()), (b, float((err - bound).max()))


@pytest.mark.parametrize("D,group,n", [(64, 1, 60001), (128, 8, 60000), (256, 9, 40007)])
def test_attn_kv4_one_head_on_the_whole_gpu(S, D, group, n):
    """Every CTA has a part of the one triple: hundreds of partial sums."""
    page, gen = 128, torch.Generator(device="cuda").manual_seed(D)
    pages = -(-n // page)
    cache = torch.full((pages, S.spdp_kv4_page_bytes(1, D, page)), 0xFF, dtype=torch.uint8, device="cuda")
    table = torch.randperm(pages, generator=gen, device="cuda")[None].int()
    t = torch.arange(n, device="cuda")
    k, v = (torch.randn(n, 1, D, generator=gen, device="cuda").half() for _ in range(2))
    v[: n // 2] *= 4.0
    kv, vv = torch.empty_like(k), torch.empty_like(v)
    S.spdp_kv4_store(k, v, table[0, t // page].long() * page + t % page, cache, page, k_values=kv, v_values=vv)
    q, y = torch.randn(1, group, D, generator=gen, device="cuda").half(), torch.empty(1, group * D, dtype=torch.float16, device="cuda")
    S.spdp_attn_kv4(q, cache, page, 1, table, torch.tensor([n], dtype=torch.int32, device="cuda"), y, 0.3)
    ks, vs = kv.double().transpose(0, 1), vv.double().transpose(0, 1)
    want, spread = plain_attention(q[0], ks, vs, 0.3), plain_attention(q[0], ks, vs.abs(), 0.3)
    # as in the test above: keys are below 6, values below 24
    reach = 0.3 * (q[0].double().abs().sum(-1) * 6.0)[:, None]
    bound = U * want.abs() * 1.01 + (3 * U + 2 * reach * (U + 560 * V) + 2.0 ** -20) * 1.02 * spread + n * TINY * 24.0 + TINY
    err = (y[0].double().view_as(want) - want).abs()
    assert bool((err <= bound).all()), float((err - bound).max())
    again = torch.empty_like(y)
    S.spdp_attn_kv4(q, cache, page, 1, table, torch.tensor([n], dtype=torch.int32, device="cuda"), again, 0.3)
    assert torch.equal(y, again)


def test_attn_kv4_many_requests(S):
    """More triples than CTAs, most of one key, some of none, a few long."""
    heads, group, D, page, B = 4, 2, 64, 16, 700
    gen = torch.Generator(device="cuda").manual_seed(9)
    length = torch.randint(0, 4, (B,), generator=gen, device="cuda", dtype=torch.int32)
    length[::97] = torch.tensor([300, 1, 16, 17, 512, 0, 33, 64], dtype=torch.int32, device="cuda")[:len(length[::97])]
    each = 32
    table = torch.randperm(B * each, generator=gen, device="cuda").view(B, each).int()
    cache = torch.full((B * each, S.spdp_kv4_page_bytes(heads, D, page)), 0xFF, dtype=torch.uint8, device="cuda")
    kv, vv = (torch.zeros(B, 512, heads, D, dtype=torch.float16, device="cuda") for _ in range(2))
    t = torch.arange(512, device="cuda")
    slot = torch.where(t < length[:, None], table[:, t // page].long() * page + t % page, -1).view(-1)
    k, v = (torch.randn(B * 512, heads, D, generator=gen, device="cuda").half() for _ in range(2))
    S.spdp_kv4_store(k, v, slot, cache, page, k_values=kv.view(-1, heads, D), v_values=vv.view(-1, heads, D))
    q = torch.randn(B, heads * group, D, generator=gen, device="cuda").half()
    y, mask = torch.full((B, heads * group * D), 3.0, dtype=torch.float16, device="cuda"), torch.full((B, heads * group * D // 32), 5, dtype=torch.int32, device="cuda")
    S.spdp_attn_kv4(q, cache, page, heads, table, length, y, 0.125, mask=mask)
    score = torch.einsum("bhgd,bthd->bhgt", q.double().view(B, heads, group, D), kv.double()) * 0.125
    score.masked_fill_((t >= length[:, None])[:, None, None], -torch.inf)
    p = torch.softmax(score, -1).nan_to_num(0.0)
    want, spread = (torch.einsum("bhgt,bthd->bhgd", p, x).reshape(B, -1) for x in (vv.double(), vv.double().abs()))
    reach = 0.125 * q.double().abs().sum(-1).repeat_interleave(D, 1) * 6.0
    bound = U * want.abs() * 1.01 + (3 * U + 2 * reach * (U + 560 * V) + 2.0 ** -20) * 1.02 * spread + 512 * TINY * 6.0 + TINY       # as in the next test
    assert bool(((y.double() - want).abs() <= bound).all())
    assert bool((y[length == 0] == 0).all()) and bool((mask[length == 0] == 0).all())


@pytest.mark.parametrize("columns", [0, 600])
def test_attn_kv4_captured_and_on_streams(S, columns):
    """Two graphs and eager calls, one after another and at once: each call's scratch memory is its own."""
    rng = np.random.default_rng(6)
    cases = []
    for i in range(2):
        cache, table, oracle = filled(rng, 2, 128, 16, [300, 17, 90])
        q, y = dev(rng.standard_normal((3, 8, 128)).astype(np.float16)), torch.empty(3, 1024, dtype=torch.float16, device="cuda")
        length = dev(np.array([300, 17, 90], np.int32))
        cases.append((q, cache, dev(np.concatenate([table, np.full((3, columns), -1, np.int32)], 1)), length, y, oracle, table))

    def call(c):
        S.spdp_attn_kv4(c[0], c[1], 16, 2, c[2], c[3], c[4], 0.1)
    for c in cases:
        first, = replayed(lambda: call(c), [c[0]], [c[4]])
        attn_check(first, c[0], c[5], c[6], [300, 17, 90], 0.1)
    graphs, streams = [], [torch.cuda.Stream() for _ in cases]
    for c in cases:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            call(c)
        graphs.append(g)
    want = [c[4].clone() for c in cases]
    torch.cuda.synchronize()
    for _ in range(20):
        for c, s, g in zip(cases, streams, graphs):
            c[4].fill_(5.0)
        torch.cuda.synchronize()
        for c, s, g in zip(cases, streams, graphs):
            with torch.cuda.stream(s):
                g.replay()
                call(c)
        torch.cuda.synchronize()
        for c, w in zip(cases, want):
            assert torch.equal(c[4], w)
    # other lengths in a captured call's own memory
    cases[0][3].copy_(dev(np.array([5, 299, 0], np.int32)))
    graphs[0].replay()
    torch.cuda.synchronize()
    c = cases[0]
    attn_check(c[4][:1], c[0][:1], c[5], c[6][:1], [5], 0.1)
    assert bool((c[4][2] == 0).all())
    del graphs


def test_tensors_of_another_device_are_refused(S, monkeypatch):
    """The calls run on the current device: tensors of another one are refused before anything is launched."""
    c = lora_case(1, 4, 64, 64, 8, 2)
    x = torch.zeros(4, 2, 64, dtype=torch.float16, device="cuda")
    cache = torch.zeros(2, S.spdp_kv4_page_bytes(2, 64, 16), dtype=torch.uint8, device="cuda")
    i32 = torch.zeros(4, dtype=torch.int32, device="cuda")
    S.spdp_lora(Y=c["base"].clone(), **c)
    monkeypatch.setattr(S, "_device", lambda: torch.cuda.device_count())
    for call in (lambda: S.spdp_lora(Y=c["base"].clone(), **c), lambda: S.spdp_qk_norm_rope(x, None, x, None, None, None),
                 lambda: S.spdp_kv4_store(x, x, i32.long(), cache, 16), lambda: S.spdp_attn_kv4(x, cache, 16, 2, i32[:, None], i32, x.view(4, -1), 1.0)):
        with pytest.raises(ValueError, match="current device"):
            call()


# ---- together ---------------------------------------------------------------------------------------------------------------

def test_decode_steps_of_an_attention_block(S):
    """Three users' tokens through packed q/k/v, adapters, norms and rotation, the cache, attention and the packed o-projection over the columns that the
    mask keeps; several steps, then the same steps from a graph."""
    rng = np.random.default_rng(21)
    B, K, heads, group, D, page, steps = 3, 256, 2, 4, 64, 16, 20
    H = heads * group
    qkv_rows = (H + 2 * heads) * D
    pruned = lambda m, k: WL.prune_global_magnitude(rng.standard_normal((m, k), dtype=np.float32) * np.float32(0.05), 0.5).astype(np.float16)
    Wqkv, Wo = pruned(qkv_rows, K), pruned(K, H * D)
    hq, ho = S.spdp_pack_tiled_cbc(dev(Wqkv)), S.spdp_pack_tiled_cbc(dev(Wo))
    try:
        f16 = lambda *s: torch.empty(*s, dtype=torch.float16, device="cuda")
        x, adapter = f16(B, K), dev(np.array([1, -1, 0], np.int32))
        A, Bw = dev((rng.standard_normal((2, 8, K)) / 16).astype(np.float16)), dev((rng.standard_normal((2, qkv_rows, 8)) * 0.1).astype(np.float16))
        qkv = torch.empty(B, qkv_rows, dtype=torch.float32, device="cuda")
        q, k = f16(B, H, D), f16(B, heads, D)
        pos, freq = torch.zeros(B, dtype=torch.int32, device="cuda"), dev((10000.0 ** (-np.arange(D // 2) / (D // 2))).astype(np.float32))
        w = dev((1 + 0.1 * rng.standard_normal(D)).astype(np.float16))
        table = torch.randperm(2 * B, device="cuda").view(B, 2).int()
        cache = torch.full((2 * B, S.spdp_kv4_page_bytes(heads, D, page)), 0xFF, dtype=torch.uint8, device="cuda")
        slot, length = torch.zeros(B, dtype=torch.int64, device="cuda"), torch.zeros(B, dtype=torch.int32, device="cuda")
        kv, vv, y, out = f16(B, heads, D), f16(B, heads, D), f16(B, H * D), f16(B, K)
        mask = torch.empty(B, H * D // 32, dtype=torch.int32, device="cuda")
        thr = 0.02

        def step():
            S.spdp_spmspv_batch(hq, x, S.SPDP_DP_ABS_GT, 0.3, qkv)
            S.spdp_lora(x, adapter, A, Bw, qkv)
            v = qkv[:, (H + heads) * D:].view(B, heads, D)
            S.spdp_qk_norm_rope(qkv[:, :H * D].view(B, H, D), qkv[:, H * D:(H + heads) * D].view(B, heads, D), q, k, pos, freq, q_weight=w, k_weight=w)
            S.spdp_kv4_store(k, v, slot, cache, page, k_values=kv, v_values=vv)
            S.spdp_attn_kv4(q, cache, page, heads, table, length, y, D ** -0.5, thr=thr, mask=mask)
            S.spdp_spmspv_batch(ho, y, S.SPDP_DP_MASK, 0.0, out, mask=mask)

        xs = dev(rng.standard_normal((steps, B, K)).astype(np.float16))

        def run(go):
            outs = []
            cache.fill_(0xFF)
            for t in range(steps):
                x.copy_(xs[t]), pos.fill_(t), length.fill_(t + 1)
                slot.copy_(table[:, t // page].long() * page + t % page)
                go()
                outs.append([a.clone() for a in (qkv, q, k, kv, vv, y, mask, out)])
            torch.cuda.synchronize()
            return outs
        first = run(step)
        keys, values = np.zeros((steps, B, heads, D)), np.zeros((steps, B, heads, D))
        for t, (gqkv, gq, gk, gkv, gvv, gy, gmask, gout) in enumerate(first):
            X = host(xs[t])
            act = np.abs(X) > np.float32(0.3)
            base = (X * act) @ host(dev(Wqkv)).T
            want, t_part, b_part = O.lora(X, adapter.cpu().numpy(), host(A), host(Bw), base)
            size = (np.abs(X) * act) @ np.abs(host(dev(Wqkv))).T
            assert np.all(np.abs(host(gqkv) - want) <= lora_bound(want, t_part, b_part, K, 8, True) + 1e-3 * size + 1e-5)
            p = np.full((1, B), t)
            heads_check(gqkv[:, :H * D].view(B, H, D), gq, w, 1e-6, p, freq.cpu().numpy(), (D // 2,), False)
            heads_check(gqkv[:, H * D:(H + heads) * D].view(B, heads, D), gk, w, 1e-6, p, freq.cpu().numpy(), (D // 2,), False)
            keys[t] = O.kv4_values(*O.kv4_codes(gk.cpu().numpy()))
            values[t] = O.kv4_values(*O.kv4_codes(gqkv[:, (H + heads) * D:].view(B, heads, D).half().cpu().numpy()))
            assert np.array_equal(gkv.cpu().numpy(), keys[t].astype(np.float16)) and np.array_equal(gvv.cpu().numpy(), values[t].astype(np.float16))
            for b in range(B):
                kk, vv_ = dev(keys[:t + 1, b].transpose(1, 0, 2)), dev(values[:t + 1, b].transpose(1, 0, 2))
                want_y = host(plain_attention(gq[b], kk, vv_, D ** -0.5))
                spread = host(plain_attention(gq[b], kk, vv_.abs(), D ** -0.5))
                reach = D ** -0.5 * np.abs(host(gq[b])).sum(-1, keepdims=True) * np.abs(keys[:t + 1, b]).max()
                bound = U * np.abs(want_y) * 1.01 + (2 * U + 4 * V * 300 * reach + 2.0 ** -20) * 1.01 * spread + steps * TINY * np.abs(values).max() + TINY
                assert np.all(np.abs(host(gy[b]).reshape(H, D) - want_y) <= bound)
            bits = gmask.cpu().numpy().view(np.uint32)
            keep = ~(np.abs(host(gy)) <= np.float32(thr))
            assert np.array_equal((bits[:, :, None] >> np.arange(32, dtype=np.uint32) & 1).reshape(B, -1).astype(bool), keep) and 0 < keep.mean() < 1
            o_size = (np.abs(host(gy)) * keep) @ np.abs(host(dev(Wo))).T
            assert np.all(np.abs(host(gout) - (host(gy) * keep) @ host(dev(Wo)).T) <= 1e-3 * o_size + 1e-5)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step()
        for a, b in zip(first, run(graph.replay)):
            for s, t in zip(a, b):
                assert torch.equal(s, t)
        del graph
    finally:
        S.spdp_free(hq)
        S.spdp_free(ho)


def test_adapters_beside_a_prompt(S):
    """spdp_spmm and the adapters of two prompts and a token without one, added in place."""
    rng = np.random.default_rng(30)
    N, K, M = 90, 520, 700
    W = WL.prune_global_magnitude(rng.standard_normal((M, K), dtype=np.float32) * np.float32(0.05), 0.5).astype(np.float16)
    X, A, B = rng.standard_normal((N, K)).astype(np.float16), (rng.standard_normal((2, 16, K)) / 23).astype(np.float16), (rng.standard_normal((2, M, 16)) * 0.1).astype(np.float16)
    adapter = np.array([0] * 50 + [1] * 39 + [-1], np.int32)
    h = S.spdp_pack_tiled_cbc(dev(W))
    try:
        Y = torch.empty(N, M, dtype=torch.float32, device="cuda")
        S.spdp_spmm(h, dev(X), Y)
        S.spdp_lora(dev(X), dev(adapter), dev(A), dev(B), Y)
        base = X.astype(np.float64) @ W.astype(np.float64).T
        want, t_part, b_part = O.lora(X, adapter, A, B, base)
        size = np.abs(X.astype(np.float64)) @ np.abs(W.astype(np.float64)).T
        assert np.all(np.abs(host(Y) - want) <= lora_bound(want, t_part, b_part, K, 16, True) + 1e-3 * size + 1e-5)
        assert S.spdp_last_device_status(h) == 0
    finally:
        S.spdp_free(h)
