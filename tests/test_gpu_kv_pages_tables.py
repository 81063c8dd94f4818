"""Bringing a cache's pages together where the table has far more entries than the kernel has threads, in tables of all forms: pages that many
entries share, entries that name none, rows apart from one another."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows,table_pages,pages,padding", [
    (1, 1, 2, 0), (1, 4096, 300, 0), (4097, 1, 300, 3), (1, 1_500_001, 5000, 0), (1_500_001, 1, 5000, 1), (3001, 701, 40000, 5), (151_553, 3, 20000, 2), (7, 151_552, 900, 1)])
def test_kv_pages_compact_renames_every_entry(rows, table_pages, pages, padding):
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA device")
    from paper_2607_21985_b200 import spdp
    rng = np.random.default_rng(rows + table_pages)
    used = np.sort(rng.choice(pages, pages // 2, replace=False))
    table = np.where(rng.random((rows, table_pages)) < 0.7, used[rng.integers(0, len(used), (rows, table_pages))], rng.choice([-1, -2 ** 31, pages, 2 ** 31 - 1], (rows, table_pages)))
    table[rows - 1, table_pages - 1] = used[-1]              # the last entry names the last page in use
    inside = table[(table >= 0) & (table < pages)]
    ref = np.bincount(inside, minlength=pages)
    wide = torch.full((rows, table_pages + padding), 77, dtype=torch.int32, device="cuda")
    tab = wide[:, :table_pages].copy_(torch.from_numpy(table.astype(np.int32)))
    counts, live = torch.from_numpy(ref.astype(np.int32)).cuda(), torch.zeros(1, dtype=torch.int32, device="cuda")
    cache = torch.arange(pages, dtype=torch.int32, device="cuda")[:, None].repeat(1, 4).view(torch.uint8)     # a page holds its number
    spdp.spdp_kv_pages_compact(cache, counts, tab, live)
    torch.cuda.synchronize()
    now = ref > 0
    n = int(now.sum())
    old, new = n + np.flatnonzero(now[n:]), np.flatnonzero(~now[:n])
    place = np.arange(pages)
    place[old] = new
    ref[new], ref[old] = ref[old], 0
    want = np.where((table >= 0) & (table < pages), place[np.clip(table, 0, pages - 1)], table)
    assert int(live) == n and np.array_equal(tab.cpu().numpy(), want) and np.array_equal(counts.cpu().numpy(), ref) and bool((wide[:, table_pages:] == 77).all())
    numbers = cache.view(torch.int32).cpu().numpy()
    assert np.array_equal(numbers[new], np.repeat(old[:, None], 4, 1)) and np.array_equal(numbers[:n][now[:n]], np.repeat(np.flatnonzero(now[:n])[:, None], 4, 1))
