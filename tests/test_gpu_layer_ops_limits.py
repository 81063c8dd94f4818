"""The operators around the packed projections where their range ends: caps far above the scores, infinite vectors between an adapter's
products, values beside infinite ones that do not turn, adapters that stand between one another.  Tolerances as in test_gpu_layer_ops.py:
u = 2^-11 is half a step of fp16, v = 2^-24 of fp32."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import layer_ops as O
from test_gpu_layer_ops import TINY, U, V, dev, filled, host

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def S():
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA device")
    from paper_2607_21985_b200 import spdp
    spdp.lib()
    return spdp


# ---- capped scores ----------------------------------------------------------------------------------------------------------

def capped_check(y, q, cache, table, length, scale, cap, most):
    """Scores before the cap: 8 products of 17 additions at 2 v of the sizes and 4 more sums, as without one (the cap only makes differences smaller).  The cap itself: tanh to
    within 8 v where it is formed from an exponential, which is 8 v cap on the score, and as the exponential is taken only from a quarter of the cap on, where tanh is above 0.244, no
    more than 33 v of the score; below that a polynomial, whose cut end (6 v) and few roundings are below 8 v of the score.  The rest as without a cap: weights 2^-21 for their exponential, u
    and half of fp16's smallest step; u for the result."""
    for b in range(len(length)):
        want, spread, reach, keys = O.attention(host(q[b]), cache, table[b], int(length[b]), scale, cap)
        ds = (2 * 2 * V * (17 * 16 + 8) * reach + np.minimum(8 * V * cap, 33 * V * reach) + 2.0 ** -21)[:, None]
        bound = U * np.abs(want) * 1.01 + (2 * U + 2 * ds) * 1.01 * spread + keys * TINY * most + TINY
        err = np.abs(host(y[b]).reshape(want.shape) - want)
        assert np.all(err <= bound), (b, float(err.max()), float((err - bound).max()))


@pytest.mark.parametrize("columns", [0, 1000])     # a cluster to a triple; a line that all CTAs share
@pytest.mark.parametrize("size,cap", [(2.0, 1e3), (2.0, 1e5), (2.0, 1e6), (2.0, 1e9), (2.0, 1e30), (2.0, 1e38), (40.0, 100.0), (40.0, 300.0), (3.0, 1.0), (6.0, 20.0), (300.0, 1e3), (20.0, 1e4)])
@pytest.mark.parametrize("group,D", [(2, 64), (9, 128), (1, 256)])
def test_attn_kv4_caps_of_all_sizes(S, group, D, size, cap, columns):
    """Scores of `size`, from far below the cap to beyond it."""
    rng = np.random.default_rng(group * 1000 + D)
    page, n = 16, [150, 33, 1]
    cache, table, oracle = filled(rng, 1, D, page, n)
    q = dev(rng.standard_normal((3, group, D)).astype(np.float16))
    y = torch.empty(3, group * D, dtype=torch.float16, device="cuda")
    wide = dev(np.concatenate([table, np.zeros((3, columns), np.int32)], 1))
    scale = size / (1.5 * np.sqrt(D))              # keys are of size 1.5
    S.spdp_attn_kv4(q, cache, page, 1, wide, dev(np.array(n, np.int32)), y, scale, cap=cap)
    capped_check(y, q, oracle, table, n, float(np.float32(scale)), float(np.float32(cap)), 150.0)


@pytest.mark.parametrize("cap", [0.0, 1.0, 50.0, 1e30])
@pytest.mark.parametrize("columns", [0, 1000])
def test_attn_kv4_nan_of_a_head_is_its_own(S, columns, cap):
    rng = np.random.default_rng(40)
    cache, table, oracle = filled(rng, 1, 64, 16, [100, 20])
    q = dev(rng.standard_normal((2, 4, 64)).astype(np.float16))
    y = torch.empty(2, 256, dtype=torch.float16, device="cuda")
    q[0, 2, 17] = float("nan")
    mask = torch.zeros(2, 8, dtype=torch.int32, device="cuda")
    S.spdp_attn_kv4(q, cache, 16, 1, dev(np.concatenate([table, np.zeros((2, columns), np.int32)], 1)), dev(np.array([100, 20], np.int32)), y, 0.125, cap=cap, thr=1e9, mask=mask)
    assert bool(y[0, 128:192].isnan().all())
    # |NaN| is not at most thr: its columns are kept, and no other
    assert mask.tolist() == [[0, 0, 0, 0, -1, -1, 0, 0], [0] * 8]
    clean = torch.cat([q[0, :2], q[0, 3:]])[None]
    capped = cap if cap else 1e38                   # the same bound without a cap
    capped_check(torch.cat([y[0, :128], y[0, 192:]])[None], clean, oracle, table[:1], [100], 0.125, capped, 150.0)
    capped_check(y[1:], q[1:], oracle, table[1:], [20], 0.125, capped, 150.0)


# ---- adapters ---------------------------------------------------------------------------------------------------------------

def same_kind(got, want):
    """NaN, Inf and -Inf where `want` (64 bits) has them, finite elsewhere."""
    got = got.double().cpu().numpy()
    return np.array_equal(np.isnan(got), np.isnan(want)) and np.array_equal(np.isposinf(got), np.isposinf(want)) and np.array_equal(np.isneginf(got), np.isneginf(want))


@pytest.mark.parametrize("f32", [False, True])
@pytest.mark.parametrize("N,K,M,rank,odd", [(1, 64, 72, 1, True), (4, 64, 72, 8, False), (16, 128, 200, 40, False), (40, 64, 72, 16, False), (40, 64, 72, 64, False), (40, 65, 71, 5, True),
                                            (600, 64, 72, 8, False), (600, 64, 72, 72, False), (7, 66, 70, 34, True)])
def test_lora_infinite_vectors_between_the_products(S, N, K, M, rank, odd, f32):
    """An infinite x makes a token's vector infinite: its results are Inf, -Inf or NaN as the formula has them, the other tokens' finite."""
    rng = np.random.default_rng(N + K + rank)
    one = lambda *s: (rng.choice([-1.0, 1.0], s) * rng.uniform(0.1, 1.0, s)).astype(np.float16)      # no zeros, so that Inf stays Inf
    X, A, B = one(N, K), one(2, rank, K) / np.float16(8), one(2, M, rank)
    B[0] = np.abs(B[0])
    B[0, M // 2:] *= -1.0                                   # adapter 0: every term of a result has the same sign
    A[0] = np.abs(A[0])
    B[1, 3] = 0.0
    bad = rng.permutation(N)[:max(1, N // 3)]
    X[bad, rng.integers(0, K, len(bad))] = rng.choice([np.inf, -np.inf], len(bad))
    adapter = np.arange(N, dtype=np.int32) % 2
    scales = np.array([0.5, -2.0], np.float32)
    base = rng.standard_normal((N, M)).astype(np.float32)
    Y = torch.empty(N, M, dtype=torch.float32 if f32 else torch.float16, device="cuda")
    S.spdp_lora(dev(X), dev(adapter), dev(A), dev(B), Y, base=dev(base).to(Y.dtype), scales=dev(scales))
    with np.errstate(invalid="ignore"):
        t = np.stack([(A[a].astype(np.float64) * X[n].astype(np.float64)).sum(-1) for n, a in enumerate(adapter)])
        want = np.stack([base[n] + float(scales[a]) * (B[a].astype(np.float64) * t[n]).sum(-1) for n, a in enumerate(adapter)])
    assert np.isinf(want).any() and same_kind(Y, want)


@pytest.mark.parametrize("N,rank", [(5, 16), (60, 16), (60, 64), (60, 20), (5, 7)])
@pytest.mark.parametrize("shared", ["none", "A", "B", "both"])
def test_lora_adapters_between_one_another(S, N, rank, shared):
    """Adapters whose rows stand between each other's (weights kept as [rank][count][K] and [M][count][rank]), and one A or B for all: the same bits as from copies."""
    rng = np.random.default_rng(N + rank)
    count, K, M = 3, 128, 200
    X, adapter = dev(rng.standard_normal((N, K)).astype(np.float16)), dev(rng.integers(-1, count + 1, N).astype(np.int32))
    A, B = dev(rng.standard_normal((rank, count, K)).astype(np.float16)).permute(1, 0, 2), dev(rng.standard_normal((M, count, rank)).astype(np.float16)).permute(1, 0, 2)
    if shared in ("A", "both"):
        A = A[1:2].expand(count, rank, K)
    if shared in ("B", "both"):
        B = B[1:2].expand(count, M, rank)
    base = dev(rng.standard_normal((N, M)).astype(np.float32)).half()
    Y, Z = torch.empty_like(base), torch.empty_like(base)
    S.spdp_lora(X, adapter, A, B, Y, base=base)
    S.spdp_lora(X, adapter, A.contiguous(), B.contiguous(), Z, base=base)
    assert torch.equal(Y, Z)


# ---- head norms and rotation ------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("pad", [0, 3])            # rows on 16-byte boundaries, and anywhere
@pytest.mark.parametrize("f32", [False, True])
@pytest.mark.parametrize("D,pairs,adjacent", [(128, 0, False), (128, 0, True), (128, 16, False), (128, 10, True), (256, 40, False), (64, 31, True), (96, 8, False), (128, 64, False)])
def test_qk_norm_rope_values_that_do_not_turn_stay(S, D, pairs, adjacent, f32, pad):
    """Inf, NaN, the largest numbers and -0 where nothing turns come out as they are and reach no other value; where a pair turns by an angle of 0 beside them, the formula."""
    N, H = 5, 3
    rng = np.random.default_rng(D + pairs)
    x = rng.standard_normal((N, H, D)).astype(np.float16)
    rest = np.arange(2 * pairs, D)
    for n in range(N):
        for h in range(H):
            some = rng.permutation(rest)[:5]
            x[n, h, some] = np.array([np.inf, -np.inf, np.nan, -0.0, 65504], np.float16)[:len(some)]
    x[0, 0, 2 * pairs:] = -0.0
    if pairs:
        x[1, 1, 0] = np.inf                          # turns with its partner, and with no other
    wide = torch.zeros(N, H * D + pad, dtype=torch.float32 if f32 else torch.float16, device="cuda")
    q = wide[:, :H * D].unflatten(1, (H, D))
    q.copy_(dev(x))
    out = torch.empty(N, H * D + pad, dtype=torch.float16, device="cuda")[:, :H * D].unflatten(1, (H, D))
    pos, freq = torch.arange(N, dtype=torch.int32, device="cuda"), torch.rand(pairs, device="cuda") if pairs else None
    S.spdp_qk_norm_rope(q, None, out, None, pos, freq, adjacent=adjacent)
    got, want = out.cpu().numpy(), x[..., 2 * pairs:]
    bits = got[..., 2 * pairs:].view(np.uint16)
    assert np.array_equal(np.isnan(got[..., 2 * pairs:]), np.isnan(want)) and np.array_equal(bits[~np.isnan(want)], want.view(np.uint16)[~np.isnan(want)])
    if pairs:
        touched = np.zeros((N, H, D), bool)
        touched[1, 1, [0, 1 if adjacent else pairs]] = True
        assert np.isfinite(got[..., :2 * pairs][~touched[..., :2 * pairs]]).all()
