"""Attention of chunks of rows over paged caches of fp32, bf16 and 8-bit values, against a plain 64-bit implementation.

Tolerance of an output: a score of hd products (three times that for fp32 rows over bf16 or 8-bit pages) in fp32 is off by at most
d = (3 hd + 8) 2^-24 scale sum |q k|; a weight e^s / sum e^s changes by less than 2 d relatively; t is what the exponential and the
probability's form add: 2^-20 where it keeps 24 bits, half a step of bf16, 2^-8, more where it is rounded to bf16 (bf16 rows, more than 16
columns a sequence); N additions cost N 2^-24 on each of the two sums.  So out is off by at most (2 d + t + 2 (N + 64) 2^-24) sum w |v| and half
a step of its type; lse by d + 2^-20 + (N + 64) 2^-24 and half a step."""
import math

import numpy as np
import pytest
import torch

from paged_any import E4M3, BF16, F32, cache_of, ints, store
from paper_2604_13519_amd import ops

pytestmark = pytest.mark.gpu

TYPES = [(BF16, BF16), (BF16, F32), (E4M3, BF16), (E4M3, F32), (F32, F32), (F32, BF16)]


def seen_of(n, rows, window=0, sets=None):
    """[rows][n + rows] truth values: what each row of a chunk behind n positions sees."""
    key, row = torch.arange(n + rows)[None], torch.arange(rows)[:, None]
    if sets is None:
        seen = key <= n + row
        return seen & (key > n + row - window) if window else seen
    own = key - n
    bits = torch.tensor([[(s >> j) & 1 for j in range(64)] for s in sets], dtype=torch.bool)
    seen = torch.ones((rows, n + rows), dtype=torch.bool)
    for j in range(1, rows):
        seen[:, n + j] = bits[:, j - 1] if j <= 64 else False
    return seen & (own < rows)


def plain(q, K, V, seen, scale):
    """One sequence in 64 bits: q [rows][hq][hd], K and V [keys][hkv][hd], seen [rows][keys] -> (out, lse, sum w |v|, d)."""
    rows, hq, hd = q.shape
    hkv = K.shape[1]
    q = q.double().view(rows, hkv, hq // hkv, hd).permute(1, 0, 2, 3).reshape(hkv, -1, hd)
    k, v = K.double().permute(1, 2, 0).contiguous(), V.double().transpose(0, 1).contiguous()
    mask = seen[None, :, None].expand(hkv, rows, hq // hkv, -1).reshape(hkv, rows * (hq // hkv), -1)
    s = (scale * torch.matmul(q, k)).masked_fill(~mask, -math.inf)
    lse = torch.logsumexp(s, 2)
    w = torch.exp(s - torch.where(lse == -math.inf, 0.0, lse)[..., None])
    size = torch.matmul(q.abs(), k.abs()).masked_fill(~mask, 0.0).amax(2)
    d = (3 * hd + 8) * 2.0 ** -24 * abs(scale) * size
    back = lambda x: x.view(hkv, rows, hq // hkv, -1).permute(1, 0, 2, 3).reshape(rows, hq, -1)  # noqa: E731
    return back(torch.matmul(w, v)), back(lse)[..., 0], back(torch.matmul(w, v.abs())), back(d)[..., 0]


def tolerance(want, rough, d, n, dtype, qdtype, columns_each):
    t = 2.0 ** -20 + (2.0 ** -8 if dtype != F32 and qdtype == BF16 and columns_each > 16 else 0.0)
    return (2 * d[..., None] + t + 2 * (n + 64) * 2.0 ** -24) * rough + torch.finfo(qdtype).eps / 2 * want.abs() + 1e-30


def check(before, new, hq, hkv, hd, dtype, qdtype, window=0, trees=None, scale=None, seed=0, more_len=0, spare=0, tag=""):
    """Chunks of new[s] rows behind before[s] positions."""
    print("rows", tag, before[:6], new[:6], hq, hkv, hd, dtype, qdtype, window, more_len, flush=True)
    lengths = [a + b for a, b in zip(before, new)]
    pages, table, K, V = cache_of(lengths, hkv, hd, dtype, seed)
    g = torch.Generator().manual_seed(seed + 1)
    rows, n = sum(new) + spare, len(new)
    q = torch.randn((rows, hq * hd), generator=g).to(qdtype)
    offsets = [sum(new[:i]) for i in range(n + 1)]
    out = torch.full((rows, hq * hd), 7.0, dtype=qdtype, device="cuda")
    lse = torch.full((rows, hq), 7.0, device="cuda")
    sets = None
    if trees is not None:
        flat = [a for t in trees for a in t] + [0] * spare
        sets = torch.tensor([a if a < 1 << 63 else a - (1 << 64) for a in flat], dtype=torch.int64, device="cuda")
    got, got_lse = ops.ts_kv_attend_rows(*pages.pages, table, ints(before), ints(offsets), q.cuda(), max(lengths) + more_len, window=window, scale=scale, ancestors=sets,
                                         scales=pages.scales, out=out, lse=lse)
    assert got is out and got_lse is lse
    out, lse = out.double().cpu(), lse.double().cpu()
    assert bool((out[sum(new):] == 7).all()) and bool((lse[sum(new):] == 7).all())
    sc = hd ** -0.5 if scale is None else scale
    columns = rows * (hq // hkv) / n
    for i in range(n):
        if not new[i]:
            continue
        a, b = offsets[i], offsets[i + 1]
        seen = seen_of(before[i], new[i], window, None if trees is None else trees[i])
        want, want_lse, rough, d = plain(q[a:b].view(-1, hq, hd), K[i], V[i], seen, sc)
        N = min(lengths[i], window or lengths[i])
        tol = tolerance(want, rough, d, N, dtype, qdtype, columns)
        worst = float(((out[a:b].view(-1, hq, hd) - want).abs() / tol).max())
        assert worst <= 1.0, "%s sequence %d: %.3g of the tolerance" % (tag, i, worst)
        l_tol = d + 2.0 ** -20 + (N + 64) * 2.0 ** -24 + 2.0 ** -23 * want_lse.abs()
        off = float(((lse[a:b] - want_lse).abs() / l_tol).max())
        assert off <= 1.0, "%s lse of sequence %d: %.3g" % (tag, i, off)


@pytest.mark.parametrize("dtype,qdtype", TYPES)
@pytest.mark.parametrize("rows", [1, 2, 3, 7, 8, 16, 17, 31, 33, 64, 65, 130])
def test_rows_and_lengths(dtype, qdtype, rows):
    for n in (0, 1, 15, 16, 17, 31, 47, 63, 64, 100, 129, 400):
        check([n], [rows], 4, 2, 64, dtype, qdtype, seed=n + rows)
    check([333], [rows], 8, 2, 128, dtype, qdtype, seed=rows, more_len=5000)


@pytest.mark.parametrize("dtype,qdtype", TYPES)
@pytest.mark.parametrize("hq,hkv", [(1, 1), (3, 1), (5, 5), (7, 1), (12, 4), (16, 1), (17, 1), (34, 2), (64, 8), (70, 1)])
def test_heads(dtype, qdtype, hq, hkv):
    check([70, 300, 0, 5], [1, 1, 1, 1], hq, hkv, 64, dtype, qdtype, seed=hq)
    check([70, 300, 0, 5], [9, 1, 20, 40], hq, hkv, 64, dtype, qdtype, seed=hq + 50)
    check([200], [5], hq, hkv, 128, dtype, qdtype, seed=hq + 100)


@pytest.mark.parametrize("hd", [8, 16, 32, 64, 128])
def test_fp32_head_sizes(hd):
    for n, rows in ((0, 1), (0, 40), (40, 3), (700, 17)):
        check([n, 3, 0], [rows, 1, 2], 6, 2, hd, F32, F32, seed=hd + n)


@pytest.mark.parametrize("dtype,qdtype", TYPES)
def test_ragged_batches_with_spare_rows_and_empty_sequences(dtype, qdtype):
    rng = np.random.default_rng(5)
    for case in range(6):
        n = int(rng.integers(1, 30))
        before = [int(x) for x in rng.integers(0, 1 << int(rng.integers(1, 11)), n)]
        new = [int(x) for x in rng.integers(0, 1 << int(rng.integers(1, 7)), n)]
        new[-1] += 1
        check(before, new, 8, 2, 64 if case % 2 else 128, dtype, qdtype, seed=case, more_len=case * 333, spare=case % 3)


@pytest.mark.parametrize("dtype,qdtype", TYPES)
def test_whole_prompts(dtype, qdtype):
    check([0, 0, 0], [257, 64, 300], 4, 1, 64, dtype, qdtype, seed=1)
    check([0, 0], [515, 130], 6, 2, 128, dtype, qdtype, seed=2)
    check([0], [1100], 2, 2, 64, dtype, qdtype, seed=3)


@pytest.mark.parametrize("dtype,qdtype", TYPES)
def test_windows(dtype, qdtype):
    for window in (1, 2, 16, 31, 33, 64, 100, 128, 500, 4000):
        check([1, 33, 150, 900, 0, 2048], [3, 20, 1, 40, 100, 5], 4, 2, 64, dtype, qdtype, window=window, seed=window)
    check([3000, 5000], [1, 1], 8, 2, 128, dtype, qdtype, window=1500, seed=2)


def test_scales():
    for dtype, qdtype in TYPES:
        for scale in (1.0, 0.0, -0.3, 3.0):
            check([1, 200], [4, 30], 4, 2, 128, dtype, qdtype, scale=scale, seed=9)


def random_tree(rng, rows):
    sets = [0]
    for j in range(1, rows):
        sets.append(sets[int(rng.integers(max(0, j - 6), j))] | 1 << (j - 1))
    return sets


@pytest.mark.parametrize("dtype,qdtype", TYPES)
def test_draft_trees(dtype, qdtype):
    rng = np.random.default_rng(8)
    for case, (before, new) in enumerate((([0], [1]), ([0], [65]), ([77], [65]), ([500], [25]), ([1000, 3, 250], [65, 9, 33]), ([31, 32, 33, 64], [17, 16, 65, 64]))):
        check(before, new, 8, 2, 128 if case % 2 else 64, dtype, qdtype, trees=[random_tree(rng, r) for r in new], seed=case, tag="tree", spare=case % 2)
    check([200], [65], 4, 4, 64, dtype, qdtype, trees=[[(1 << 64) - 1] * 65], seed=3, tag="all of the chunk")
    check([200], [65], 4, 4, 64, dtype, qdtype, trees=[[0] * 65], seed=3, tag="the root alone")
    check([20], [70], 4, 4, 64, dtype, qdtype, trees=[[(1 << 64) - 1] * 70], seed=4, tag="rows beyond 64 are not seen")
    check([20], [5], 4, 4, 64, dtype, qdtype, trees=[[(1 << 64) - 1] * 5], seed=4, tag="bits beyond the chunk")


@pytest.mark.parametrize("dtype,qdtype", TYPES)
def test_long_contexts(dtype, qdtype):
    check([9000, 4100], [3, 20], 8, 1, 128, dtype, qdtype, seed=2)
    check([12000], [1], 4, 1, 64, dtype, qdtype, seed=3)
    check([5000] * 3, [16] * 3, 4, 2, 64, dtype, qdtype, seed=4, more_len=40000)


@pytest.mark.parametrize("dtype,qdtype", TYPES)
def test_one_row_a_sequence_without_offsets(dtype, qdtype):
    lengths = [5, 700, 1, 0, 64]
    pages, table, K, V = cache_of([n + 1 for n in lengths], 2, 64, dtype, 3)
    for hq in (2, 8, 40):
        q = torch.randn((5, hq * 64)).to(qdtype).cuda()
        a = ops.ts_kv_attend_rows(*pages.pages, table, ints(lengths), None, q, 701, scales=pages.scales)
        b = ops.ts_kv_attend_rows(*pages.pages, table, ints(lengths), ints(range(6)), q, 701, scales=pages.scales)
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
        if dtype != E4M3:
            c = ops.ts_kv_attend(*pages.pages, table, ints([n + 1 for n in lengths]), q, 701)
            assert float((a[0].double() - c[0].double()).abs().max()) <= 2.0 ** -6 and float((a[1] - c[1]).abs().max()) <= 1e-5


@pytest.mark.parametrize("dtype,qdtype", TYPES)
@pytest.mark.parametrize("rows", [2, 40])
def test_what_is_not_seen_has_no_influence_whatever_it_is(dtype, qdtype, rows):
    """Keys and values of a chunk's later rows, of other branches of a tree and of places without a position: infinities and NaN."""
    hq, hkv, hd, n = 8, 2, 64, 37
    pages, table, K, V = cache_of([n + rows], hkv, hd, dtype, 5)
    q = torch.randn((rows, hq * hd), generator=torch.Generator().manual_seed(2)).to(qdtype).cuda()
    call = lambda p, **kw: ops.ts_kv_attend_rows(*p.pages, table, ints([n]), ints([0, rows]), q, n + rows, scales=p.scales, **kw)  # noqa: E731
    tree = torch.tensor([0] + [1 << (j - 1) for j in range(1, rows)], dtype=torch.int64, device="cuda")      # every row sees the root and itself
    for kw in ({}, dict(window=20), dict(ancestors=tree)):
        clean = call(pages, **kw)
        for bad in (math.inf, -math.inf, math.nan):
            if dtype == E4M3 and bad != math.nan:
                continue
            for j in sorted({1, rows // 2, rows - 1}):
                other = pages.clone()
                store(other, table, n + j, bad)
                out, lse = call(other, **kw)
                free = [r for r in range(rows) if (r != j if "ancestors" in kw else r < j)]
                assert torch.equal(out[free], clean[0][free]) and torch.equal(lse[free], clean[1][free]), (kw, bad, j)
                hit = out[j].view(hq, hd)[:, 3]
                assert bool(hit.isnan().all()) if dtype == E4M3 else not bool(hit.isfinite().any())
        if "window" in kw:
            other = pages.clone()
            store(other, table, n - 20, math.nan)                                # the position in front of every row's window
            out, lse = call(other, **kw)
            assert torch.equal(out, clean[0]) and torch.equal(lse, clean[1])


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_seen_infinities(dtype):
    """An infinite value makes its dimension infinite in the rows that see it; a key of -infinity counts for nothing."""
    hq, hd, n, rows = 4, 64, 30, 20
    pages, table, K, V = cache_of([n + rows], 1, hd, dtype, 6)
    q = (torch.randn((rows, hq * hd), generator=torch.Generator().manual_seed(3)).abs() + 0.01).to(dtype).cuda()
    call = lambda p: ops.ts_kv_attend_rows(*p.pages, table, ints([n]), ints([0, rows]), q, n + rows)  # noqa: E731
    clean, clean_lse = call(pages)
    for at in (0, 17, n, n + 7, n + rows - 1):
        page, slot = int(table[0, at // 16]), at % 16
        other = pages.clone()
        other.pages[1][page, 0, 7, slot], other.pages[1][page, 0, 33, slot] = math.inf, -math.inf
        out, lse = call(other)
        out, was = out.view(rows, hq, hd), clean.view(rows, hq, hd)
        sees = [r for r in range(rows) if n + r >= at]
        rest = [d for d in range(hd) if d not in (7, 33)]
        assert bool((out[sees][..., 7] == math.inf).all()) and bool((out[sees][..., 33] == -math.inf).all()), at
        assert torch.equal(out[..., rest], was[..., rest]) and torch.equal(lse, clean_lse)
        assert torch.equal(out[[r for r in range(rows) if r not in sees]], was[[r for r in range(rows) if r not in sees]])
        other = pages.clone()
        other.pages[0][page, 0, slot] = -math.inf
        out, lse = call(other)
        seen = seen_of(n, rows)
        seen[:, at] = False
        k2 = K[0].clone()
        want, want_lse, rough, d = plain(q.cpu().view(rows, hq, hd), k2, V[0], seen, hd ** -0.5)
        tol = tolerance(want, rough, d, n + rows, dtype, dtype, 80)
        dead = (~seen.any(1)).nonzero()[:, 0].tolist()
        live = [r for r in range(rows) if r not in dead]
        assert bool(((out.double().cpu().view(rows, hq, hd) - want).abs() <= tol)[live].all()), at
        assert bool((out[dead] == 0).all()) and bool((lse[dead] == -math.inf).all())


def test_bad_pages_lengths_and_offsets_are_not_followed():
    for dtype in (BF16, E4M3, F32):
        hq, hkv, hd, n, rows = 4, 2, 64, 180, 20
        pages, table, K, V = cache_of([n + rows], hkv, hd, dtype, 3)
        q = torch.randn((rows, hq * hd)).to(BF16).cuda()
        call = lambda t, length=n, off=(0, rows), top=n + rows, out=None: ops.ts_kv_attend_rows(  # noqa: E731
            *pages.pages, t, ints([length] * (len(off) - 1)), ints(off), q, top, scales=pages.scales, out=out)
        for bad in (-1, 1 << 30, -(1 << 31), (1 << 31) - 1, pages.pages[0].shape[0]):
            for at in (0, 5, 11, 12):
                t = table.clone()
                t[0, at] = bad
                out, lse = call(t)
                seen = seen_of(n, rows)
                seen[:, at * 16:at * 16 + 16] = False
                want, want_lse, rough, d = plain(q.cpu().view(rows, hq, hd), K[0], V[0], seen, hd ** -0.5)
                assert bool(((out.double().cpu().view(rows, hq, hd) - want).abs() <= tolerance(want, rough, d, n + rows, dtype, BF16, 40)).all()), (bad, at)
        out, lse = call(torch.full_like(table, -7))
        assert bool((out == 0).all()) and bool((lse == -math.inf).all())
        for length in (-rows - 5, -(1 << 31)):                  # no position
            out, lse = call(table, length)
            assert bool((out == 0).all()) and bool((lse == -math.inf).all())
        seen = seen_of(0, rows)                                 # rows 8 .. have positions 0 ..
        out, lse = call(table, -8)
        want, want_lse, rough, d = plain(q.cpu().view(rows, hq, hd)[8:], K[0][:12], V[0][:12], seen_of(0, 12), hd ** -0.5)
        assert bool((out[:8] == 0).all()) and bool(((out.double().cpu().view(rows, hq, hd)[8:] - want).abs() <= tolerance(want, rough, d, 12, dtype, BF16, 40)).all())
        near = call(table, (1 << 31) - 1, top=64)               # positions beyond max_len are not seen
        seen = torch.ones((rows, 64), dtype=torch.bool)
        want, want_lse, rough, d = plain(q.cpu().view(rows, hq, hd), K[0][:64], V[0][:64], seen, hd ** -0.5)
        assert bool(((near[0].double().cpu().view(rows, hq, hd) - want).abs() <= tolerance(want, rough, d, 64, dtype, BF16, 40)).all())
        for off in ((0, 1 << 30), (-(1 << 31), rows), (5, 3), (rows, 0), (-3, 4), ((1 << 31) - 1, -(1 << 31)), (0, 30, 2, 20)):      # stay in bounds
            out = torch.full((rows, hq * hd), 7.0, dtype=BF16, device="cuda")
            call(torch.cat([table] * (len(off) - 1)), off=off, out=out)
        assert bool((call(table, off=(5, 3), out=torch.full((rows, hq * hd), 7.0, dtype=BF16, device="cuda"))[0] == 7).all())


@pytest.mark.parametrize("dtype,qdtype", TYPES)
def test_windows_that_end_behind_max_len(dtype, qdtype):
    """The window counts from a row's position; rows whose window lies at max_len and beyond see nothing, beside rows of the same tile that do."""
    hq, hkv, hd, n, top = 8, 2, 64, 2100, 2048
    for rows in (1, 3, 80):
        for window in (100, 128, 60):
            pages, table, K, V = cache_of([n + rows], hkv, hd, dtype, 3)
            q = torch.randn((rows, hq * hd), generator=torch.Generator().manual_seed(4)).to(qdtype)
            ws = ops.ts_kv_attend_rows_workspace(1, rows, hq, hkv, hd, top, window)
            if ws is not None:
                ws.fill_(255)                                  # NaN: a part that nobody wrote shows
            out, lse = ops.ts_kv_attend_rows(*pages.pages, table, ints([n]), ints([0, rows]), q.cuda(), top, window=window, scales=pages.scales, workspace=ws)
            seen = seen_of(n, rows, window)
            seen[:, top:] = False
            want, want_lse, rough, d = plain(q.view(rows, hq, hd), K[0], V[0], seen, hd ** -0.5)
            none = ~seen.any(1)
            assert bool((out.cpu()[none] == 0).all()) and bool((lse.cpu()[none] == -math.inf).all())
            assert bool(((out.double().cpu().view(rows, hq, hd) - want).abs() <= tolerance(want, rough, d, window, dtype, qdtype, rows * 4)).all()), (rows, window)


def test_strided_rows():
    pages, table, K, V = cache_of([60], 2, 64, BF16, 8)
    wide = torch.full((20, 4 * 64 + 9), math.nan, dtype=BF16, device="cuda")
    wide[:, 3:259] = torch.randn((20, 256), device="cuda")
    want, want_lse = ops.ts_kv_attend_rows(*pages.pages, table, ints([40]), ints([0, 20]), wide[:, 3:259].contiguous(), 60)
    out = torch.full((24, 300), 5.0, dtype=BF16, device="cuda")
    got, lse = ops.ts_kv_attend_rows(*pages.pages, table, ints([40]), ints([0, 20]), wide[:, 3:259], 60, out=out[1:21, 7:263])
    assert torch.equal(got, want) and torch.equal(lse, want_lse)
    out[1:21, 7:263] = 5.0
    assert bool((out == 5.0).all())


@pytest.mark.parametrize("dtype", [BF16, E4M3, F32])
def test_results_repeat_and_workspaces_may_be_larger(dtype):
    before, new = [3000, 100, 2000], [5, 30, 1]
    pages, table, K, V = cache_of([a + b for a, b in zip(before, new)], 2, 128, dtype, 8)
    q = torch.randn((36, 8 * 128)).to(BF16).cuda()
    first = ops.ts_kv_attend_rows(*pages.pages, table, ints(before), ints([0, 5, 35, 36]), q, 3005, scales=pages.scales)
    big = ops.ts_kv_attend_rows_workspace(3, 36, 8, 2, 128, 100000)
    big.fill_(255)
    for ws in (None, big):
        again = ops.ts_kv_attend_rows(*pages.pages, table, ints(before), ints([0, 5, 35, 36]), q, 3005, scales=pages.scales, workspace=ws)
        assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])


def test_pages_beyond_32_bits():
    hkv, hd = 8, 128
    n = (1 << 32) // (hkv * 16 * hd) + 40                       # 4.3 GB of 8-bit keys
    small, table, K, V = cache_of([470], hkv, hd, E4M3, 2, identity=True)
    p = small.pages[0].shape[0]
    raw = [torch.zeros((n,) + tuple(x.shape[1:]), dtype=torch.uint8, device="cuda") for x in small.pages + small.scales]
    for x, y in zip(raw, small.pages + small.scales):
        x[-p:] = y.view(torch.uint8)
    q = torch.randn((30, 32 * hd), device="cuda").to(BF16)
    far = ops.ts_kv_attend_rows(raw[0].view(E4M3), raw[1].view(E4M3), table + (n - p), ints([440]), ints([0, 30]), q, 470, scales=(raw[2], raw[3]))
    near = ops.ts_kv_attend_rows(*small.pages, table, ints([440]), ints([0, 30]), q, 470, scales=small.scales)
    assert torch.equal(far[0], near[0]) and torch.equal(far[1], near[1])
    rows = ops.ts_kv_read(raw[0].view(E4M3), raw[1].view(E4M3), table + (n - p), None, ints([0, 470]), 470, scales=(raw[2], raw[3]))
    want = ops.ts_kv_read(*small.pages, table, None, ints([0, 470]), 470, scales=small.scales)
    assert torch.equal(rows[0], want[0]) and torch.equal(rows[1], want[1])


def test_many_sequences():
    n, hd = 5000, 64
    pages, table, K, V = cache_of([3] * 7, 1, hd, BF16, 2)
    many = table[torch.arange(n, device="cuda") % 7].contiguous()
    q = torch.randn((n, 4 * hd), device="cuda").to(BF16)
    out, lse = ops.ts_kv_attend_rows(*pages.pages, many, ints([2] * n), None, q, 3)
    again, lse2 = ops.ts_kv_attend_rows(*pages.pages, many, ints([2] * n), ints(range(n + 1)), q, 3)
    assert torch.equal(out, again) and torch.equal(lse, lse2)
    for i in (0, 1, 6, 7, 2500, n - 1):
        want, _, rough, d = plain(q[i:i + 1].cpu().view(1, 4, hd), K[i % 7], V[i % 7], torch.ones((1, 3), dtype=torch.bool), hd ** -0.5)
        assert bool(((out[i].double().cpu().view(1, 4, hd) - want).abs() <= tolerance(want, rough, d, 3, BF16, BF16, 4)).all())


def test_another_stream_and_a_captured_step_with_other_contents():
    """Lengths, offsets, tables and sets are read when the kernels run; eager calls of the same buffers between replays."""
    hq, hkv, hd, rows = 8, 2, 128, 40
    pages, table, K, V = cache_of([900, 300], hkv, hd, E4M3, 4)
    q = torch.randn((rows, hq * hd), device="cuda").to(BF16)
    lengths, offsets = ints([800, 200]), ints([0, 30, 40])
    ws = ops.ts_kv_attend_rows_workspace(2, rows, hq, hkv, hd, 1000)
    out, lse = torch.zeros((rows, hq * hd), dtype=BF16, device="cuda"), torch.zeros((rows, hq), device="cuda")
    call = lambda w, o, e: ops.ts_kv_attend_rows(*pages.pages, table, lengths, offsets, q, 1000, scales=pages.scales, workspace=w, out=o, lse=e)  # noqa: E731
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call(ws, out, lse)
    side.synchronize()
    want = [x.clone() for x in call(None, None, None)]
    assert torch.equal(out, want[0]) and torch.equal(lse, want[1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(ws, out, lse)
    for step, (a, b) in enumerate((([800, 200], [0, 30, 40]), ([5, 290], [0, 40, 40]), ([860, 0], [0, 0, 40]), ([1, 2], [0, 3, 9]))):
        lengths.copy_(ints(a))
        offsets.copy_(ints(b))
        out.zero_()
        lse.zero_()
        graph.replay()
        torch.cuda.synchronize()
        want = call(None, None, None)
        assert torch.equal(out, want[0]) and torch.equal(lse, want[1]), step


def test_gradients_are_refused():
    pages, table, K, V = cache_of([20], 2, 64, BF16, 8)
    q = torch.randn((4, 256), device="cuda").to(BF16).requires_grad_()
    with pytest.raises(ValueError, match="q requires a gradient"):
        ops.ts_kv_attend_rows(*pages.pages, table, ints([16]), ints([0, 4]), q, 20)
    with torch.no_grad():
        ops.ts_kv_attend_rows(*pages.pages, table, ints([16]), ints([0, 4]), q, 20)
