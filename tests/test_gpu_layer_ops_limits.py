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
