"""Attention of chunks over batches of 40 to 200 sequences with different numbers of rows: what the plan of such calls can come across, against the plain
64-bit implementation and with the tolerances of test_gpu_paged_rows."""
import numpy as np
import pytest
import torch

from paged_any import BF16, E4M3, F32, cache_of, ints
from paper_2604_13519_amd import ops
from test_gpu_paged_rows import TYPES, check, random_tree, seen_of, tolerance
from test_gpu_paged_rows import plain as plain_rows

pytestmark = pytest.mark.gpu


def ragged(n, most_rows, most_before, seed, empty=0.3):
    """Rows and earlier positions of n sequences: some without rows, the first and last among them."""
    rng = np.random.default_rng(seed)
    new = [int(x) for x in rng.integers(0, most_rows + 1, n)]
    new = [0 if rng.random() < empty or i in (0, n - 1) else r for i, r in enumerate(new)]
    new[n // 2] = most_rows
    return [int(x) for x in rng.integers(0, most_before + 1, n)], new


@pytest.mark.parametrize("dtype,qdtype", TYPES)
@pytest.mark.parametrize("n", [40, 63, 64, 65, 200])
def test_ragged_batches(dtype, qdtype, n):
    """Few rows each (tiles of 16), some more (128; fp32 32), many (256: more than 512 columns a sequence on average)."""
    before, new = ragged(n, 6, 300, n)
    check(before, new, 4, 2, 64, dtype, qdtype, seed=n, spare=2, tag="few")
    before, new = ragged(n, 60 if n == 200 else 150, 200, n + 1)
    check(before, new, 8, 2, 64 if n % 2 else 128, dtype, qdtype, seed=n + 1, tag="some")
    before, new = ragged(n, 30 if n == 200 else 100, 100, n + 2, empty=0.1)
    check(before, new, 34, 1, 64, dtype, qdtype, seed=n + 2, spare=1, tag="many")
    before, new = ragged(n, 300, 50, n + 3, empty=0.97)                             # one long chunk and little else
    check(before, new, 4, 1, 64, dtype, qdtype, seed=n + 3, tag="one")


@pytest.mark.parametrize("dtype,qdtype", TYPES)
@pytest.mark.parametrize("n", [64, 130])
def test_ragged_batches_with_splits_windows_and_trees(dtype, qdtype, n):
    """One KV head: contexts of some thousand positions are split over workgroups."""
    before, new = ragged(n, 3, 200, n)
    before[3], before[n // 2] = 3000, 2500
    check(before, new, 4, 1, 64, dtype, qdtype, seed=n, spare=3, tag="splits")
    check(before, new, 4, 1, 64, dtype, qdtype, window=700, seed=n, tag="splits of a window")
    before, new = ragged(n, 70, 200, n + 1)
    before[3], before[n // 2], new[3] = 3000, 2500, 5
    check(before, new, 4, 1, 128, dtype, qdtype, seed=n + 1, tag="splits, more rows")
    check(before, new, 4, 1, 64, dtype, qdtype, window=45, seed=n + 1, tag="window")
    new = [min(r, 65) for r in new]
    rng = np.random.default_rng(n)
    for rows in (new, [min(r, 4) for r in new]):
        check(before, rows, 4, 1, 64, dtype, qdtype, trees=[random_tree(rng, r) if r else [] for r in rows], seed=n + 2, spare=1, tag="tree")


def test_offsets_that_decrease_stay_in_bounds():
    """64 sequences and more, offsets in any order: no row outside [0, n_rows) is read or written, and the next call is right."""
    for dtype, hq, hkv in ((BF16, 4, 1), (E4M3, 4, 1), (F32, 4, 2), (BF16, 16, 1)):
        hd, rows, n = 64, 300, 70
        pages, table, K, V = cache_of([90], hkv, hd, dtype, 3)
        many = table.expand(n, -1).contiguous()
        g = torch.Generator().manual_seed(7)
        wide = torch.randn((rows + 8, hq * hd), generator=g).to(BF16).cuda()
        wide[rows:] = float("nan")
        q = wide[:rows]
        sets = torch.full((rows + 8,), -1, dtype=torch.int64, device="cuda")[:rows]
        tables = [[rows] * 3 + [5] * (n - 2), [90, rows] + [0] * (n - 1), list(range(n, -1, -1)), [rows - i for i in range(n + 1)], [0, rows] * (n // 2) + [7],
                  [0, 1 << 30] + [-(1 << 31)] * (n - 1), [(1 << 31) - 1] * n + [0]]
        tables += [torch.randint(0, rows + 1, (n + 1,), generator=g).tolist() for _ in range(6)]
        for at, off in enumerate(tables):
            for kw in ({}, dict(window=30), dict(ancestors=sets)):
                print("decreasing", dtype, hq, at, kw.keys(), flush=True)
                out, lse = torch.full((rows + 8, hq * hd), 7.0, dtype=BF16, device="cuda"), torch.full((rows + 8, hq), 7.0, device="cuda")
                ops.ts_kv_attend_rows(*pages.pages, many, ints([20] * n), ints(off), q, 90, scales=pages.scales, out=out[:rows], lse=lse[:rows], **kw)
                assert bool((out[rows:] == 7).all()) and bool((lse[rows:] == 7).all()), (dtype, at)
                assert not bool(lse[:rows].isnan().any()), (dtype, at)           # the rows behind q are NaN
        off = [min(i, 60) for i in range(n + 1)]
        out, lse = ops.ts_kv_attend_rows(*pages.pages, many, ints([20] * n), ints(off), q, 90, scales=pages.scales)
        want, want_lse, rough, d = plain_rows(q[:60].cpu().view(60, hq, hd), K[0][:21], V[0][:21], seen_of(20, 1).expand(60, -1), hd ** -0.5)
        assert bool(((out[:60].double().cpu().view(60, hq, hd) - want).abs() <= tolerance(want, rough, d, 21, dtype, BF16, rows * hq // hkv / n)).all())
