"""Attention of chunks over batches of 63 to 200 sequences with different numbers of rows: what the plan of such calls can come across, against the plain
64-bit implementation and with the tolerances of test_gpu_paged_rows."""
import pytest
import torch

from paged_any import BF16, E4M3, F32, cache_of, ints
from paper_2604_13519_amd import ops
from test_gpu_paged_rows import seen_of, tolerance
from test_gpu_paged_rows import plain as plain_rows

pytestmark = pytest.mark.gpu


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
