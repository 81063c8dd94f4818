"""The operators around the projections, without a GPU: refusals at the ends of what the calls take."""
import pytest

from paper_2607_21985_b200 import build, spdp
from test_layer_ops_host import ATTN, INVALID, LORA, SHAPE, arrived

INT32_MAX = 2 ** 31 - 1


@pytest.fixture(scope="module")
def L():
    build.build()
    return spdp.lib()


@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
def test_attn_kv4_refuses_keys_too_near_the_end_of_32_bits(L, page):
    """The kernel forms the numbers of keys up to 32 stages of 128 behind the stage for which it asks for pages, and a stage behind a run's end: within 8192 of
    the last key, which have to fit 32 bits too."""
    pages = (INT32_MAX - 8192) // page + 1
    one = dict(ATTN, B=1, q_heads=1, kv_heads=1, dim=64, page=page)
    assert (pages * page // 64 + 8) <= INT32_MAX            # not refused for its units
    for more in (0, 1, 63, 600):
        assert L.spdp_attn_kv4(*dict(one, table_pages=pages + more, table_stride=pages + more).values()) == SHAPE


def test_attn_kv4_looks_no_further_ahead_than_what_is_refused():
    """The kernel's arithmetic followed in whole numbers: the largest key number that is formed for any run whose last key is the largest that is taken."""
    worst = 0
    for run in (*range(1, 600), *range(2000, 2200), 8191, 8192, 8193, 100000, 100001):      # keys of the run; it ends at k1 = 0
        k0 = -run
        for w in range(4):
            stages = ((run + 31) // 32 - w + 3) // 4
            page_of = lambda i: max(k0 + 32 * (w + 4 * (i + lane // 2)) + 16 * (lane & 1) for lane in range(32))
            worst = max(worst, page_of(0), page_of(16))
            for i in range(max(stages, 0)):
                worst = max(worst, k0 + 32 * w + 128 * (i + 1) + 32)                        # the stage behind, and its end
                if i % 16 == 15:
                    worst = max(worst, page_of(i + 17))
    assert 4000 < worst < 8192


@pytest.mark.parametrize("change", [
    dict(lda=191, stride_a=64), dict(lda=192, stride_a=63), dict(lda=192, stride_a=65), dict(lda=192, stride_a=1), dict(ldb=23, stride_b=8), dict(ldb=24, stride_b=7), dict(ldb=24, stride_b=9),
    dict(stride_a=-64), dict(stride_b=-1), dict(stride_a=1 << 50), dict(stride_b=1 << 50),
    dict(count=2 ** 31 - 1, stride_a=1 << 38, stride_b=1 << 38), dict(count=1, M=1 << 30, ldbase=1 << 30, ldy=1 << 30, ldb=1 << 35),        # 2^69 and 2^65 elements
    dict(M=1 << 30, ldbase=1 << 30, ldy=1 << 30, ldb=1 << 35), dict(M=1 << 30, ldbase=1 << 30, ldy=1 << 30, ldb=1 << 34, stride_b=1 << 34)])
def test_lora_refuses_adapters_that_overlap_or_cannot_exist(L, change):
    """Adapters one after another, or row between row, or all the same; whose last element is within 2^60 of the first."""
    assert L.spdp_lora(*dict(LORA, **change).values()) == INVALID


def test_attn_kv4_takes_no_mask_but_32_bit_integers(L):
    import torch
    args = [torch.zeros(4, 6, 64).half(), torch.zeros(2, 3 * 16 * 72, dtype=torch.uint8), 16, 3, torch.zeros(4, 5, dtype=torch.int32), torch.zeros(4, dtype=torch.int32),
            torch.zeros(4, 384).half(), 0.1, 0.0, 0, 0.0]
    for dtype in (torch.int32, torch.uint32):
        mask = torch.zeros(4, 13, dtype=dtype)
        assert arrived(L, "attn_kv4", *args, mask, 0)[19:21] == [mask.data_ptr(), 13]
    for dtype in (torch.float32, torch.int16, torch.uint8, torch.float64, torch.bool):
        with pytest.raises(ValueError, match="32-bit"):
            arrived(L, "attn_kv4", *args, torch.zeros(4, 13, dtype=dtype), 0)
