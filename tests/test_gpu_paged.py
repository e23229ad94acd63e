"""Appending to a paged cache and attention of one token over it, against plain 64-bit implementations.

Tolerances.  A rotated value: the angle is reduced in 64 bits and rounded to fp32 (2^-26 of a turn: 9e-8 radians), sine and
cosine are good to two steps, three fp32 roundings follow: below 2^-21 (|x| + |y|); then half a step of the stored type.
Attention: a score of hd products (three times that for fp32 queries on a bf16 cache) in fp32 is off by at most
d = (3 hd + 8) 2^-24 scale sum |q k|; a weight e^s / sum e^s changes by less than 2 d relatively (+ 2^-21 for the exponentials),
by 2^-16 where probabilities enter as two bf16 terms (16 bits, half a step each of two), and N additions cost N 2^-24 on each
of the two sums: out is off by at most (2 d + t + 2 (N + 64) 2^-24) sum w |v| and half a step of its type; lse by d + 2^-20 +
(N + 64) 2^-24 and half a step."""
import math

import numpy as np
import pytest
import torch

import workloads as wl
from paper_2604_13519_amd import binding as B
from paper_2604_13519_amd import ops

pytestmark = pytest.mark.gpu


def make_cache(lengths, hkv, hd, dtype, seed, spare_pages=2, extra=0, fill=math.nan):
    """Pages in random order; places that hold no position are NaN."""
    g = torch.Generator().manual_seed(seed)
    need = [max(1, -(-(n + extra) // 16)) for n in lengths]
    total = sum(need) + spare_pages
    order = torch.randperm(total, generator=g)
    table = torch.full((len(lengths), max(need) + 1), -1, dtype=torch.int32)
    k = torch.full((total, hkv, 16, hd), fill, dtype=dtype)
    v = torch.full((total, hkv, hd, 16), fill, dtype=dtype)
    at, K, V = 0, [], []
    for i, n in enumerate(lengths):
        pages = order[at:at + need[i]]
        at += need[i]
        table[i, :need[i]] = pages.to(torch.int32)
        K.append(torch.randn((n, hkv, hd), generator=g).to(dtype))
        V.append(torch.randn((n, hkv, hd), generator=g).to(dtype))
        p, s = pages[torch.arange(n) // 16], torch.arange(n) % 16
        k[p, :, s] = K[i]
        v[p, :, :, s] = V[i]
    return k.cuda(), v.cuda(), table.cuda(), K, V


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def plain_attend(q, K, V, hkv, hd, window, scale):
    """One sequence in 64 bits: (out, lse, tolerance of out, of lse), heads first."""
    hq = q.numel() // hd
    n = K.shape[0]
    lo = max(0, n - window) if window else 0
    K, V = K[lo:].double(), V[lo:].double()
    q = q.double().view(hq, hd)
    out = torch.zeros((hq, hd), dtype=torch.float64)
    lse = torch.full((hq,), -math.inf, dtype=torch.float64)
    rough, l_tol = torch.zeros((hq, hd), dtype=torch.float64), torch.zeros(hq, dtype=torch.float64)
    if n == 0:
        return out, lse, rough, l_tol, torch.zeros(hq, dtype=torch.float64)
    d = torch.zeros(hq, dtype=torch.float64)
    for h in range(hq):
        k, v = K[:, h // (hq // hkv)], V[:, h // (hq // hkv)]
        s = scale * (k @ q[h])
        w = torch.softmax(s, 0)
        out[h], lse[h] = w @ v, torch.logsumexp(s, 0)
        rough[h] = w @ v.abs()
        d[h] = (3 * hd + 8) * 2.0 ** -24 * abs(scale) * float((k.abs() @ q[h].abs()).max())
    return out, lse, rough, d, d


def check_attend(lengths, hq, hkv, hd, dtype, qdtype, window=0, scale=None, seed=0, max_len=None, tag=""):
    print("attend", tag, lengths[:8], hq, hkv, hd, dtype, qdtype, window, max_len, flush=True)
    k, v, table, K, V = make_cache(lengths, hkv, hd, dtype, seed)
    g = torch.Generator().manual_seed(seed + 1)
    q = torch.randn((len(lengths), hq * hd), generator=g).to(qdtype)
    top = max(lengths) if max_len is None else max_len
    out, lse = ops.ts_kv_attend(k, v, table, ints(lengths), q.cuda(), top, window=window, scale=scale)
    out, lse = out.double().cpu().view(len(lengths), hq, hd), lse.double().cpu()
    s = hd ** -0.5 if scale is None else scale
    t = 2.0 ** -20 if qdtype == torch.float32 or dtype == torch.float32 else 2.0 ** -16
    for i, n in enumerate(lengths):
        want, want_lse, rough, d, _ = plain_attend(q[i], K[i], V[i], hkv, hd, window, s)
        if n == 0:
            assert bool((out[i] == 0).all()) and bool((lse[i] == -math.inf).all())
            continue
        N = min(n, window or n)
        tol = (2 * d[:, None] + t + 2 * (N + 64) * 2.0 ** -24) * rough + torch.finfo(qdtype).eps / 2 * want.abs() + 1e-30
        worst = ((out[i] - want).abs() / tol).max().item()
        assert worst <= 1.0, "%s sequence %d (%d keys): %.3g of the tolerance" % (tag, i, n, worst)
        l_tol = d + 2.0 ** -20 + (N + 64) * 2.0 ** -24 + 2.0 ** -23 * want_lse.abs()
        assert bool(((lse[i] - want_lse).abs() <= l_tol).all()), "%s lse of sequence %d" % (tag, i)


TYPES = [(torch.bfloat16, torch.bfloat16), (torch.bfloat16, torch.float32), (torch.float32, torch.float32), (torch.float32, torch.bfloat16)]


@pytest.mark.parametrize("dtype,qdtype", TYPES)
@pytest.mark.parametrize("n", [0, 1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 127, 128, 129, 255, 257, 511, 1000])
def test_attend_lengths(dtype, qdtype, n):
    check_attend([n], 8, 2, 64, dtype, qdtype, seed=n)
    check_attend([n], 4, 4, 128, dtype, qdtype, seed=n + 1, max_len=n + 5000)          # more splits than the length fills


@pytest.mark.parametrize("dtype,qdtype", TYPES)
@pytest.mark.parametrize("hq,hkv", [(1, 1), (3, 1), (5, 5), (8, 1), (12, 4), (16, 1), (17, 1), (34, 2), (64, 8), (40, 1)])
def test_attend_heads(dtype, qdtype, hq, hkv):
    check_attend([70, 300, 0, 5], hq, hkv, 64, dtype, qdtype, seed=hq)
    check_attend([333], hq, hkv, 128, dtype, qdtype, seed=hq + 100)


@pytest.mark.parametrize("hd", [8, 16, 32, 64, 128])
def test_attend_fp32_head_sizes(hd):
    for n in (1, 40, 700):
        check_attend([n, 3, 0], 6, 2, hd, torch.float32, torch.float32, seed=hd + n)


@pytest.mark.parametrize("dtype,qdtype", TYPES)
def test_attend_ragged(dtype, qdtype):
    rng = np.random.default_rng(5)
    for case in range(6):
        lengths = [int(x) for x in rng.integers(0, 1 << int(rng.integers(1, 12)), int(rng.integers(1, 40)))]
        check_attend(lengths, 8, 2, 64 if case % 2 else 128, dtype, qdtype, seed=case, max_len=max(lengths) + case * 333)


@pytest.mark.parametrize("dtype,qdtype", TYPES[:3])
def test_attend_window_and_scale(dtype, qdtype):
    for window in (1, 2, 16, 31, 32, 33, 100, 128, 500, 4000):
        check_attend([1, 33, 150, 900, 0, 2048], 8, 4, 64, dtype, qdtype, window=window, seed=window)
    for scale in (1.0, 0.0, -0.3, 3.0):
        check_attend([1, 200], 4, 2, 128, dtype, qdtype, scale=scale, seed=9)


def test_attend_long():
    check_attend([20011, 31999], 8, 1, 128, torch.bfloat16, torch.bfloat16, seed=2)
    check_attend([9000] * 3, 16, 8, 64, torch.bfloat16, torch.float32, seed=3)


def test_attend_bad_pages_and_unseen_places_have_no_influence():
    """Keys on pages outside the pool, beyond the table or beyond max_len are as if they were not there."""
    for dtype in (torch.bfloat16, torch.float32):
        k, v, table, K, V = make_cache([200], 2, 64, dtype, 3, spare_pages=0)
        q = torch.randn((1, 256)).to(dtype)
        for bad in (-1, 13, 1 << 30, -(1 << 31)):
            for at in (0, 5, 11, 12):
                t = table.clone()
                t[0, at] = bad
                out, lse = ops.ts_kv_attend(k, v, t, ints([200]), q.cuda(), 200)
                keep = [p for p in range(200) if p // 16 != at]
                want, want_lse, rough, d, _ = plain_attend(q[0], K[0][keep], V[0][keep], 2, 64, 0, 0.125)
                tol = (2 * d[:, None] + 2.0 ** -16 + 600 * 2.0 ** -24) * rough + torch.finfo(dtype).eps / 2 * want.abs()
                assert bool(((out.double().cpu().view(4, 64) - want).abs() <= tol).all()), (bad, at)
        out, lse = ops.ts_kv_attend(k, v, torch.full_like(table, -7), ints([200]), q.cuda(), 200)
        assert bool((out == 0).all()) and bool((lse == -math.inf).all())
        narrow, short = table[:, :4], ops.ts_kv_attend(k, v, table, ints([64]), q.cuda(), 64)
        for got in (ops.ts_kv_attend(k, v, narrow, ints([200]), q.cuda(), 200), ops.ts_kv_attend(k, v, table, ints([200]), q.cuda(), 64),
                    ops.ts_kv_attend(k, v, narrow, ints([1 << 30]), q.cuda(), 1 << 30)):
            assert float((got[0] - short[0]).abs().max()) <= 2.0 ** -6 and float((got[1] - short[1]).abs().max()) <= 1e-5
        out, lse = ops.ts_kv_attend(k, v, table, ints([-5]), q.cuda(), 200)
        assert bool((out == 0).all()) and bool((lse == -math.inf).all())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_attend_window_of_lengths_beyond_max_len(dtype):
    """The window is the last positions of the length; of those, what lies at max_len and beyond is not seen."""
    hq, hd = 4, 64
    k, v, table, K, V = make_cache([1000], 2, hd, dtype, 17)
    q = torch.randn((1, hq * hd), generator=torch.Generator().manual_seed(3)).to(dtype)
    for n, top, window in ((200, 64, 150), (200, 200, 150), (1000, 700, 301), (1000, 700, 350), (999, 998, 3), (1 << 30, 800, (1 << 30) - 90)):
        out, lse = ops.ts_kv_attend(k, v, table, ints([n]), q.cuda(), top, window=window)
        lo = n - window
        want, want_lse, rough, d, _ = plain_attend(q[0], K[0][lo:top], V[0][lo:top], 2, hd, 0, 0.125)
        tol = (2 * d[:, None] + 2.0 ** -20 + 2 * (top + 64) * 2.0 ** -24) * rough + torch.finfo(dtype).eps / 2 * want.abs()
        assert bool(((out.double().cpu().view(hq, hd) - want).abs() <= tol).all()), (n, top, window)
        assert bool(((lse.double().cpu()[0] - want_lse).abs() <= d + 2.0 ** -20 + (top + 64) * 2.0 ** -24 + 2.0 ** -23 * want_lse.abs()).all())
    for n, top, window in ((200, 64, 100), (200, 64, 136), ((1 << 31) - 1, 1000, 1000), ((1 << 31) - 1, 0, 5)):
        out, lse = ops.ts_kv_attend(k, v, table, ints([n]), q.cuda(), top, window=window)
        assert bool((out == 0).all()) and bool((lse == -math.inf).all()), (n, top, window)


def test_attend_special_values_that_are_seen():
    for dtype in (torch.bfloat16, torch.float32):
        k, v, table, K, V = make_cache([300], 1, 64, dtype, 4)
        q = torch.ones((1, 128), device="cuda").to(dtype)
        first = int(table[0, 0])
        clean, _ = ops.ts_kv_attend(k, v, table, ints([300]), q, 300)
        k2 = k.clone()
        k2[first, 0, 3] = -math.inf                            # a score of -infinity: the key counts for nothing
        out, lse = ops.ts_kv_attend(k2, v, table, ints([300]), q, 300)
        keep = [p for p in range(300) if p != 3]
        want, want_lse, rough, d, _ = plain_attend(q.cpu()[0], K[0][keep], V[0][keep], 1, 64, 0, 0.125)
        assert bool(((out.double().cpu().view(2, 64) - want).abs() <= (2 * d[:, None] + 2.0 ** -15) * rough + torch.finfo(dtype).eps * want.abs()).all())
        out, lse = ops.ts_kv_attend(k2[first:first + 1].contiguous(), v[first:first + 1].contiguous(), ints([[0]]), ints([3]), q, 300)
        assert bool(torch.isfinite(out).all())
        k2[:] = -math.inf                                      # every score: nothing is left
        out, lse = ops.ts_kv_attend(k2, v, table, ints([300]), q, 300)
        assert bool((out == 0).all()) and bool((lse == -math.inf).all())
        k2 = k.clone()
        k2[first, 0, 3, 0] = math.nan
        out, lse = ops.ts_kv_attend(k2, v, table, ints([300]), q, 300)
        assert bool(out.isnan().all()) and bool(lse.isnan().all())
        v2 = v.clone()
        v2[first, 0, 7, 3] = math.inf
        out, _ = ops.ts_kv_attend(k, v2, table, ints([300]), q, 300)
        out = out.view(2, 64)
        assert bool((out[:, 7] == math.inf).all()) and torch.equal(out[:, :7], clean.view(2, 64)[:, :7]) and torch.equal(out[:, 8:], clean.view(2, 64)[:, 8:])


@pytest.mark.parametrize("dtype,qdtype", TYPES)
@pytest.mark.parametrize("n", [3, 40, 300])
def test_attend_infinite_keys_and_values(dtype, qdtype, n):
    """A key of -infinity counts for nothing and an infinite value makes its dimension infinite, whatever the query's and the
    probability's last bits are; the other keys and dimensions are as without them."""
    hd, hq = 64, 24
    for q_of in (lambda g: torch.ones((1, hq * hd)), lambda g: torch.randn((1, hq * hd), generator=g).abs() + 0.01):
        q = q_of(torch.Generator().manual_seed(n)).to(qdtype).cuda()
        k, v, table, K, V = make_cache([n], 1, hd, dtype, 31 + n)
        clean, clean_lse = ops.ts_kv_attend(k, v, table, ints([n]), q, n)
        for at in sorted({0, 1, n // 2, n - 1}):
            page, slot = int(table[0, at // 16]), at % 16
            k2 = k.clone()
            k2[page, 0, slot, 5] = -math.inf
            out, lse = ops.ts_kv_attend(k2, v, table, ints([n]), q, n)
            keep = [p for p in range(n) if p != at]
            want, want_lse, rough, d, _ = plain_attend(q.cpu()[0], K[0][keep], V[0][keep], 1, hd, 0, 0.125)
            tol = (2 * d[:, None] + 2.0 ** -20 + 2 * (n + 64) * 2.0 ** -24) * rough + torch.finfo(qdtype).eps / 2 * want.abs()
            assert bool(((out.double().cpu().view(hq, hd) - want).abs() <= tol).all()), ("key", at)
            assert bool(((lse.double().cpu()[0] - want_lse).abs() <= d + 2.0 ** -20 + (n + 64) * 2.0 ** -24 + 2.0 ** -23 * want_lse.abs()).all())
            v2 = v.clone()
            v2[page, 0, 7, slot], v2[page, 0, 33, slot] = math.inf, -math.inf
            out, lse = ops.ts_kv_attend(k, v2, table, ints([n]), q, n)
            out, other = out.view(hq, hd), [i for i in range(hd) if i not in (7, 33)]
            assert bool((out[:, 7] == math.inf).all()) and bool((out[:, 33] == -math.inf).all()), ("value", at)
            assert torch.equal(out[:, other], clean.view(hq, hd)[:, other]) and torch.equal(lse, clean_lse)


def test_attend_scores_far_apart_in_any_order():
    """The running maximum rises at every block, falls at every block, and stays."""
    for dtype in (torch.bfloat16, torch.float32):
        for order in (1, -1, 0):
            n = 1000
            k, v, table, K, V = make_cache([n], 1, 64, dtype, 6)
            size = torch.arange(n).double() * 0.5 * abs(order)
            size = size.flip(0) if order < 0 else size
            K = [(torch.ones((n, 1, 64)).double() * size[:, None, None] / 8).to(dtype)]
            p, s = table.cpu()[0][torch.arange(n) // 16].long(), torch.arange(n) % 16
            k[p.cuda(), :, s.cuda()] = K[0].cuda()
            q = torch.ones((1, 128)).to(dtype)
            out, lse = ops.ts_kv_attend(k, v, table, ints([n]), q.cuda(), n)
            want, want_lse, rough, d, _ = plain_attend(q[0], K[0], V[0], 1, 64, 0, 0.125)
            tol = (2 * d[:, None] + 2.0 ** -16 + 2200 * 2.0 ** -24) * rough + torch.finfo(dtype).eps / 2 * want.abs()
            assert bool(((out.double().cpu().view(2, 64) - want).abs() <= tol).all())


@pytest.mark.parametrize("dtype,qdtype", TYPES)
def test_attend_probabilities_have_24_bits(dtype, qdtype):
    """Two keys with values v and -1: out = (v - p) / (1 + p), which shows p's last bits where v is near p.  Scores have one
    term, |score| < 1, so p is off by the roundings of scale log2(e), of the score and of the exponential (below 2^-22.4) and
    the two sums and the quotient by 5 half steps: 2^-21 in all, then half a step of the output."""
    hd, hq = 128, 1024
    scale = 2.0 ** -10
    q = torch.zeros((hq, hd))
    q[:, 0] = torch.arange(hq) % 128 + 128                     # bf16 holds 128 .. 255
    q[:, 0] *= 2.0 ** (torch.arange(hq) // 256)                # scores -1/8 .. -1 over all heads
    k = torch.zeros((1, 1, 16, hd), dtype=dtype)
    k[0, 0, 1, 0] = -0.5
    v = torch.full((1, 1, hd, 16), math.nan, dtype=dtype)
    v[0, 0, :, 0] = 0.5 + torch.arange(hd) / 256.0             # bf16 holds them: 0.5 .. 1 in steps of 2^-8
    v[0, 0, :, 1] = -1.0
    for shift in (1.0, 0.93, 0.871):
        s = scale * shift
        out, _ = ops.ts_kv_attend(k.cuda(), v.cuda(), ints([[0]]), ints([2]), q.to(qdtype).view(1, -1).cuda(), 2, scale=s)
        s32 = float(torch.tensor(s, dtype=torch.float32))      # what the call takes
        p = torch.exp(-0.5 * s32 * q[:, :1].double())
        want = (v[0, 0, :, 0].double()[None] - p) / (1 + p)
        err = (out.double().cpu().view(hq, hd) - want).abs()
        tol = 2.0 ** -21 + torch.finfo(qdtype).eps / 2 * want.abs()
        assert bool((err <= tol).all()), "%.3g of the tolerance" % float((err / tol).max())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_attend_largest_finite_queries(dtype):
    """fp32 queries up to the largest number: their scores are finite where the keys are small.  A score has one term."""
    hd = 64
    top = torch.finfo(torch.float32).max
    k, v, table, K, V = make_cache([40], 1, hd, dtype, 21)
    k = torch.where(k.isnan(), k, k * 2.0 ** -126).to(dtype)
    K = [K[0] * 2.0 ** -126]
    q = torch.zeros((4, hd))
    q[0, 3], q[1, 9], q[2, 0], q[3, 63] = top, -top, 3.397e38, -1.5 * 2.0 ** 127
    out, lse = ops.ts_kv_attend(k, v, table, ints([40]), q.view(1, -1).cuda(), 40, scale=0.25)
    want, want_lse, rough, d, _ = plain_attend(q.view(-1), K[0], V[0], 1, hd, 0, 0.25)
    tol = (2 * d[:, None] + 2.0 ** -20 + 2 * 104 * 2.0 ** -24) * rough + 2.0 ** -24 * want.abs()
    assert bool(((out.double().cpu().view(4, hd) - want).abs() <= tol).all())
    assert bool(((lse.double().cpu()[0] - want_lse).abs() <= d + 2.0 ** -20 + 104 * 2.0 ** -24 + 2.0 ** -23 * want_lse.abs()).all())


def test_attend_strided_rows_and_padding():
    lengths = [40, 700, 3]
    k, v, table, K, V = make_cache(lengths, 2, 64, torch.bfloat16, 8)
    wide = torch.full((3, 4 * 64 + 9), math.nan, dtype=torch.bfloat16, device="cuda")
    wide[:, 3:3 + 256] = torch.randn((3, 256), device="cuda")
    q = wide[:, 3:3 + 256]
    want, want_lse = ops.ts_kv_attend(k, v, table, ints(lengths), q.contiguous(), 700)
    out = torch.full((5, 300), 5.0, dtype=torch.bfloat16, device="cuda")
    got, lse = ops.ts_kv_attend(k, v, table, ints(lengths), q, 700, out=out[1:4, 7:263])
    assert torch.equal(got, want) and torch.equal(lse, want_lse)
    out[1:4, 7:263] = 5.0
    assert bool((out == 5.0).all())


def test_attend_pages_beyond_32_bits():
    """A pool whose last pages start beyond 2^32 bytes and 2^31 elements."""
    hkv, hd = 8, 128
    n = (1 << 31) // (hkv * 16 * hd) + 40                      # 4.3 GB of keys
    k = torch.zeros((n, hkv, 16, hd), dtype=torch.bfloat16, device="cuda")
    v = torch.zeros((n, hkv, hd, 16), dtype=torch.bfloat16, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(1)
    small_k = torch.randn((30, hkv, 16, hd), generator=g, device="cuda").bfloat16()
    small_v = torch.randn((30, hkv, hd, 16), generator=g, device="cuda").bfloat16()
    k[-30:], v[-30:] = small_k, small_v
    q = torch.randn((1, 32 * hd), generator=g, device="cuda").bfloat16()
    t = torch.arange(30, dtype=torch.int32, device="cuda")[None]
    far = ops.ts_kv_attend(k, v, t + (n - 30), ints([470]), q, 470)
    near = ops.ts_kv_attend(small_k, small_v, t, ints([470]), q, 470)
    assert torch.equal(far[0], near[0]) and torch.equal(far[1], near[1])
    rows = torch.randn((1, (32 + 16) * hd), generator=g, device="cuda").bfloat16()
    a, b, c = rows.split((32 * hd, 8 * hd, 8 * hd), 1)
    ops.ts_kv_append(k, v, t + (n - 30), ints([470]), ints([0, 1]), a, b, c, 1e4)
    ops.ts_kv_append(small_k, small_v, t, ints([470]), ints([0, 1]), a, b, c, 1e4)
    assert torch.equal(k[-30:], small_k) and torch.equal(v[-30:], small_v) and not bool(k[:-30].any())


# ---- append --------------------------------------------------------------------------------
def plain_turn(x, pos, theta):
    """x [heads][hd] in 64 bits, its rotation, and |x| + |partner|."""
    hd = x.shape[-1]
    x = x.double()
    if theta == 0:
        return x, torch.zeros_like(x)
    j = torch.arange(hd // 2, dtype=torch.float64)
    ang = pos * torch.pow(torch.tensor(theta, dtype=torch.float64), -2 * j / hd)
    c, s = torch.cos(ang), torch.sin(ang)
    a, b = x[..., :hd // 2], x[..., hd // 2:]
    both = a.abs() + b.abs()
    return torch.cat((a * c - b * s, b * c + a * s), -1), 2.0 ** -21 * torch.cat((both, both), -1)


def near(got, want, rough):
    return bool(((got.double() - want).abs() <= rough + torch.finfo(got.dtype).eps / 2 * want.abs() + 1e-37).all())


def check_append(lengths, new, hq, hkv, hd, dtype, rdtype, theta, seed=0, pad=0, misalign=0):
    print("append", lengths[:8], new[:8], hq, hkv, hd, dtype, rdtype, theta, pad, misalign, flush=True)
    k, v, table, K, V = make_cache(lengths, hkv, hd, dtype, seed, extra=max(new) if new else 0, fill=3.0)
    k0, v0 = k.cpu().clone(), v.cpu().clone()
    rows = sum(new)
    g = torch.Generator().manual_seed(seed + 5)
    width = (hq + 2 * hkv) * hd
    x = torch.randn((rows + pad, width + 2 * misalign), generator=g).to(rdtype)
    d = x.cuda()[:, misalign:misalign + width]
    x = x[:, misalign:misalign + width]
    q, kk, vv = d.split((hq * hd, hkv * hd, hkv * hd), 1) if hq else (None,) + d.split((hkv * hd, hkv * hd), 1)
    q_out = torch.full((rows + pad, hq * hd + misalign), 9.0, dtype=rdtype, device="cuda")[:, misalign:] if hq else None
    offs = [sum(new[:i]) for i in range(len(new) + 1)]
    ops.ts_kv_append(k, v, table, ints(lengths), ints(offs), q, kk, vv, theta, q_out)
    k, v = k.cpu(), v.cpu()
    touched_k, touched_v = k0.clone(), v0.clone()
    t = table.cpu().long()
    for s, (n, m) in enumerate(zip(lengths, new)):
        for i in range(m):
            row, pos = x[offs[s] + i], n + i
            page, slot = t[s, pos // 16], pos % 16
            want, rough = plain_turn(row[hq * hd:(hq + hkv) * hd].view(hkv, hd), pos, theta)
            assert near(k[page, :, slot], want, rough), ("k", s, i)
            assert torch.equal(v[page, :, :, slot], row[(hq + hkv) * hd:].view(hkv, hd).to(dtype)), ("v", s, i)
            touched_k[page, :, slot], touched_v[page, :, :, slot] = k[page, :, slot], v[page, :, :, slot]
            if hq:
                want, rough = plain_turn(row[:hq * hd].view(hq, hd), pos, theta)
                assert near(q_out[offs[s] + i].cpu().view(hq, hd), want, rough), ("q", s, i)
    assert torch.equal(k, touched_k) and torch.equal(v, touched_v)     # nothing else
    if hq and pad:
        assert bool((q_out[rows:] == 9.0).all())


@pytest.mark.parametrize("dtype,rdtype", TYPES)
def test_append_rows(dtype, rdtype):
    for hq, hkv, hd in ((8, 2, 64), (4, 4, 128), (0, 3, 64), (40, 8, 64)):
        check_append([0], [1], hq, hkv, hd, dtype, rdtype, 1e4)
        check_append([15, 16, 17, 0, 100], [1, 1, 1, 1, 1], hq, hkv, hd, dtype, rdtype, 5e5, seed=1, pad=2)
        check_append([0, 5, 31, 64], [40, 0, 17, 16], hq, hkv, hd, dtype, rdtype, 1e6, seed=2, pad=3)
        check_append([7, 7, 7], [0, 33, 0], hq, hkv, hd, dtype, rdtype, 0.0, seed=3)
    check_append([3, 40], [20, 2], 4, 2, 64, dtype, rdtype, 1e4, seed=4, pad=1, misalign=1)
    check_append([3, 40], [20, 2], 4, 2, 128, dtype, rdtype, 1e4, seed=4, misalign=3)


@pytest.mark.parametrize("hd", [8, 16, 32])
def test_append_small_heads(hd):
    check_append([0, 30], [19, 5], 6, 3, hd, torch.float32, torch.float32, 1e4)
    check_append([0, 30], [19, 5], 6, 3, hd, torch.float32, torch.bfloat16, 1e4, misalign=1)


def test_append_many_sequences():
    rng = np.random.default_rng(0)
    for n in (63, 64, 65, 200, 4097):
        new = [int(x) for x in rng.integers(0, 3, n)]
        new[0], new[-1] = 1, 1
        check_append([int(x) for x in rng.integers(0, 20, n)], new, 1, 1, 64, torch.bfloat16, torch.bfloat16, 1e4, seed=n, pad=1)


@pytest.mark.parametrize("dtype,rdtype", TYPES)
@pytest.mark.parametrize("most", [2, 6, 14, 30])
def test_append_many_sequences_of_many_heads(dtype, rdtype, most):
    rng = np.random.default_rng(most)
    for n, hq, hkv in ((127, 5, 2), (130, 31, 5)):
        new = [int(x) for x in rng.integers(most // 2, most + 1, n)]
        check_append([int(x) for x in rng.integers(0, 20, n)], new, hq, hkv, 64, dtype, rdtype, 1e4, seed=n + most, pad=1)


@pytest.mark.parametrize("new", [[300], [9, 700, 0, 260], [1100, 1030]])
def test_append_long_contexts(new):
    check_append([5 + 7 * i for i in range(len(new))], new, 3, 1, 64, torch.bfloat16, torch.bfloat16, 1e6, seed=len(new), pad=2)


def test_append_far_positions_keep_their_phase():
    """Positions up to 2^27 on one page each: the table points them all at a few pages."""
    hd, width = 64, (1 << 27) // 16 + 1
    table = torch.zeros((1, width), dtype=torch.int32, device="cuda")
    for pos in (1000003, 16777217, (1 << 27) - 1):
        k = torch.zeros((1, 1, 16, hd), device="cuda")
        v = torch.zeros((1, 1, hd, 16), device="cuda")
        x = torch.randn((1, 3 * hd), device="cuda")
        q, kk, vv = x.split((hd, hd, hd), 1)
        out = ops.ts_kv_append(k, v, table, ints([pos]), ints([0, 1]), q, kk, vv, 1e4)
        want, rough = plain_turn(q.cpu().view(1, hd), pos, 1e4)
        assert near(out.cpu().view(1, hd), want, rough), pos
        want, rough = plain_turn(kk.cpu().view(1, hd), pos, 1e4)
        assert near(k[0, :, pos % 16].cpu(), want, rough), pos


def test_append_leaves_what_has_no_place():
    hd, hkv, hq = 64, 2, 4
    for dtype in (torch.bfloat16, torch.float32):
        g = torch.Generator(device="cuda").manual_seed(3)
        rows = 40
        x = torch.randn((rows, (hq + 2 * hkv) * hd), generator=g, device="cuda").to(dtype)
        q, kk, vv = x.split((hq * hd, hkv * hd, hkv * hd), 1)

        def go(table, lengths, offs):
            k = torch.full((6, hkv, 16, hd), 3.0, dtype=dtype, device="cuda")
            v = torch.full((6, hkv, hd, 16), 3.0, dtype=dtype, device="cuda")
            out = torch.full((rows, hq * hd), 9.0, dtype=dtype, device="cuda")
            ops.ts_kv_append(k, v, ints(table), ints(lengths), ints(offs), q, kk, vv, 1e4, out)
            rows_written = [r for r in range(rows) if not bool((out[r] == 9.0).all())]
            places = (k != 3.0).any(3).any(1)
            assert torch.equal(places, (v != 3.0).any(2).any(1))
            return rows_written, int(places.sum())

        assert go([[0, 1, 2]], [0], [0, 40]) == (list(range(40)), 40)
        assert go([[0, -1, 2]], [0], [0, 40]) == (list(range(16)) + list(range(32, 40)), 24)          # a page that does not exist
        assert go([[0, 6, 2]], [0], [0, 40]) == (list(range(16)) + list(range(32, 40)), 24)
        assert go([[0, 1]], [0], [0, 40]) == (list(range(32)), 32)                                   # beyond the table
        assert go([[0, 1, 2]], [-3], [0, 40]) == (list(range(3, 40)), 37)                            # before the first position
        assert go([[0, 1, 2]], [1 << 30], [0, 40]) == ([], 0)
        assert go([[0, 1, 2]], [2147483647], [0, 40]) == ([], 0)
        assert go([[0, 1, 2]], [0], [5, 12]) == (list(range(5, 12)), 7)                              # rows of nobody in front and behind
        assert go([[0, 1], [2, 3], [4, 5]], [4, 9, 0], [2, 2, 30, 33]) == (list(range(2, 25)) + [30, 31, 32], 26)     # the second sequence's table ends
        assert go([[0, 1, 2]], [0], [0, 1000]) == (list(range(40)), 40)                              # offsets beyond the rows there are
        assert go([[0, 1, 2]], [0], [-7, 3]) == ([0, 1, 2], 3)                                       # ... and before


def test_append_in_place_queries():
    hd = 128
    k, v, table, _, _ = make_cache([10, 50], 2, hd, torch.bfloat16, 0, extra=20, fill=0.0)
    x = torch.randn((23, 8 * hd), device="cuda").bfloat16()
    y = x.clone()
    want = ops.ts_kv_append(k.clone(), v.clone(), table, ints([10, 50]), ints([0, 20, 23]), x[:, :4 * hd], x[:, 4 * hd:6 * hd], x[:, 6 * hd:], 1e4)
    ops.ts_kv_append(k, v, table, ints([10, 50]), ints([0, 20, 23]), y[:, :4 * hd], y[:, 4 * hd:6 * hd], y[:, 6 * hd:], 1e4, y[:, :4 * hd])
    assert torch.equal(y[:, :4 * hd], want) and torch.equal(y[:, 4 * hd:], x[:, 4 * hd:])


def test_queries_rows_and_pages_that_require_gradients_are_refused():
    k, v, table, _, _ = make_cache([20], 2, 64, torch.float32, 0, extra=4, fill=0.0)
    q, kk = torch.randn((1, 256), device="cuda"), torch.randn((1, 128), device="cuda")
    grad = lambda t: t.clone().requires_grad_()  # noqa: E731
    k0 = k.clone()
    for a, b, c, d in ((k, grad(q), kk, kk), (k, q, grad(kk), kk), (k, q, kk, grad(kk)), (grad(k), q, kk, kk)):
        with pytest.raises(ValueError, match="requires a gradient"):
            ops.ts_kv_append(a, v, table, ints([20]), ints([0, 1]), b, c, d, 1e4)
    for a, b in ((k, grad(q)), (grad(k), q)):
        with pytest.raises(ValueError, match="requires a gradient"):
            ops.ts_kv_attend(a, v, table, ints([20]), b, 20)
    with pytest.raises(ValueError, match="requires a gradient"):
        ops.ts_kv_attend(k, grad(v), table, ints([20]), q, 20)
    assert torch.equal(k, k0)
    with torch.no_grad():
        out, lse = ops.ts_kv_attend(k, v, table, ints([20]), grad(q), 20)
    want = ops.ts_kv_attend(k, v, table, ints([20]), q, 20)
    assert torch.equal(out, want[0]) and torch.equal(lse, want[1])


def test_lengths_and_windows_beyond_32_bits_are_refused():
    k, v, table, _, _ = make_cache([20], 2, 64, torch.bfloat16, 0)
    q = torch.zeros((1, 256), dtype=torch.bfloat16, device="cuda")
    for ws in (None, torch.empty(1 << 20, dtype=torch.uint8, device="cuda")):
        for top, window in ((1 << 31, 0), ((1 << 32) + 20, 0), (20, 1 << 31), (20, (1 << 32) + 4)):
            with pytest.raises(ValueError, match="32 bits|out of range"):
                ops.ts_kv_attend(k, v, table, ints([20]), q, top, window=window, workspace=ws)


def test_as_many_sequences_as_a_call_takes():
    """2^20 sequences of a page each, a row appended to every one, and attention of 15 heads: 2^24 - 2^20 of them."""
    n, hq, hd = 1 << 20, 15, 64
    if torch.cuda.mem_get_info()[0] < (40 << 30):
        pytest.skip("40 GB of device memory are needed")
    g = torch.Generator(device="cuda").manual_seed(4)
    k = torch.randn((n, 1, 16, hd), generator=g, device="cuda", dtype=torch.bfloat16)
    v = torch.randn((n, 1, hd, 16), generator=g, device="cuda", dtype=torch.bfloat16)
    table = torch.randperm(n, generator=g, device="cuda").to(torch.int32)[:, None]
    lens = torch.randint(0, 16, (n,), generator=g, device="cuda", dtype=torch.int32)
    x = torch.randn((n, (hq + 2) * hd), generator=g, device="cuda", dtype=torch.bfloat16)
    q, kk, vv = x.split((hq * hd, hd, hd), 1)
    sample = [0, 1, 63, 64, 4095, 65536, n // 2 + 1, n - 2, n - 1] + [int(i) for i in np.random.default_rng(0).integers(0, n, 60)]
    pages = table[sample, 0].long()
    K0, V0 = k[pages, 0].cpu(), v[pages, 0].cpu()
    turned = ops.ts_kv_append(k, v, table, lens, torch.arange(n + 1, dtype=torch.int32, device="cuda"), q, kk, vv, 1e4)
    out, lse = ops.ts_kv_attend(k, v, table, lens + 1, turned, 16)
    K1, V1, nums = k[pages, 0].cpu(), v[pages, 0].cpu(), lens[sample].tolist()
    for i, (s, m) in enumerate(zip(sample, nums)):
        want, rough = plain_turn(kk[s].cpu().view(1, hd), m, 1e4)
        assert near(K1[i, m:m + 1], want, rough) and torch.equal(V1[i, :, m], vv[s].cpu()), s
        want, rough = plain_turn(q[s].cpu().view(hq, hd), m, 1e4)
        assert near(turned[s].cpu().view(hq, hd), want, rough), s
        others = [p for p in range(16) if p != m]
        assert torch.equal(K1[i, others], K0[i, others]) and torch.equal(V1[i][:, others], V0[i][:, others]), s
        want, want_lse, rough, d, _ = plain_attend(turned[s].cpu(), K1[i, :m + 1, None], V1[i].t()[:m + 1, None], 1, hd, 0, hd ** -0.5)
        tol = (2 * d[:, None] + 2.0 ** -20 + 2 * 80 * 2.0 ** -24) * rough + torch.finfo(torch.bfloat16).eps / 2 * want.abs()
        assert bool(((out[s].double().cpu().view(hq, hd) - want).abs() <= tol).all()), s
        assert bool(((lse[s].double().cpu() - want_lse).abs() <= d + 2.0 ** -20 + 80 * 2.0 ** -24 + 2.0 ** -23 * want_lse.abs()).all()), s
    del k, v, x, q, kk, vv, turned, out, lse
    torch.cuda.empty_cache()


def test_captured_steps_replay_with_other_lengths():
    """Append, attend and the lengths' increment in one graph, replayed over a page border with eager work between."""
    hd, hq, hkv, n = 128, 8, 2, 3
    lengths = [13, 200, 0]
    k, v, table, _, _ = make_cache(lengths, hkv, hd, torch.bfloat16, 1, extra=40, fill=0.0)
    ek, ev = k.clone(), v.clone()
    x = torch.randn((n, (hq + 2 * hkv) * hd), device="cuda").bfloat16()
    lens, offs = ints(lengths), ints([0, 1, 2, 3])
    q_out = torch.empty((n, hq * hd), dtype=torch.bfloat16, device="cuda")
    out, lse = torch.empty_like(q_out), torch.empty((n, hq), device="cuda")
    ws = ops.ts_kv_attend_workspace(n, hq, hkv, hd, 600)

    def step(k, v, lens, q_out, out, lse, ws):
        q, kk, vv = x.split((hq * hd, hkv * hd, hkv * hd), 1)
        ops.ts_kv_append(k, v, table, lens, offs, q, kk, vv, 1e4, q_out)
        lens += 1
        return ops.ts_kv_attend(k, v, table, lens, q_out, 600, workspace=ws, out=out, lse=lse)

    elens = lens.clone()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step(k, v, lens, q_out, out, lse, ws)
    lens.copy_(elens)
    for i in range(20):
        x.copy_(torch.randn(x.shape, generator=torch.Generator(device="cuda").manual_seed(i), device="cuda"))
        want, want_lse = step(ek, ev, elens, torch.empty_like(q_out), None, None, None)
        g.replay()
        if i % 7 == 0:
            torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(lse, want_lse), i
        assert torch.equal(k, ek) and torch.equal(v, ev)


def test_two_streams_at_once():
    lengths = [3000, 100, 5000]
    k, v, table, _, _ = make_cache(lengths, 2, 128, torch.bfloat16, 1, fill=0.0)
    qs = [torch.randn((3, 8 * 128), device="cuda").bfloat16() for _ in range(2)]
    want = [ops.ts_kv_attend(k, v, table, ints(lengths), q, 5000) for q in qs]
    streams = [torch.cuda.Stream() for _ in qs]
    lens = ints(lengths)
    torch.cuda.synchronize()
    got = []
    for _ in range(5):
        for s, q in zip(streams, qs):
            with torch.cuda.stream(s):
                got.append(ops.ts_kv_attend(k, v, table, lens, q, 5000))
    torch.cuda.synchronize()
    for i, (o, l) in enumerate(got):
        assert torch.equal(o, want[i % 2][0]) and torch.equal(l, want[i % 2][1])


def test_extend_waits_for_the_stream_it_is_given():
    """Positions appended on a side stream behind other work are there once the length says so (one GPU here: a stream of
    another one is refused by the same check as in the other calls)."""
    cfg = wl.get_config("small_bf16")
    model = B.ts_model_load(cfg, wl.gen_weights(cfg, 1))
    kv = B.ts_kv_alloc(model, 64)
    try:
        hd, hkv = cfg.head_dim, cfg.n_kv_heads
        table = torch.from_numpy(ops.ts_kv_page_table(kv, 64)).cuda()[None]
        rows = torch.randn((5, 2 * hkv * hd), device="cuda").bfloat16()
        big = torch.randn((4096, 4096), device="cuda")
        lens, offs = ints([0]), ints([0, 5])
        torch.cuda.synchronize()
        side = torch.cuda.Stream()
        with torch.cuda.stream(side):
            for _ in range(20):
                big = big @ big * 1e-3
            for layer in range(cfg.n_layers):
                ops.ts_kv_append(ops.ts_kv_layer_pages(kv, layer), None, table, lens, offs, None, rows[:, :hkv * hd], rows[:, hkv * hd:], 0.0)
        ops.ts_kv_extend(kv, 5, stream=side)
        assert side.query() and B.ts_kv_len(kv) == 5
        gk, gv = B.ts_kv_export(kv, 0, 5, cfg)
        want = rows.view(torch.int16).cpu().numpy().view(np.uint16).reshape(5, 2, hkv, hd)
        for layer in range(cfg.n_layers):
            assert np.array_equal(gk[layer], want[:, 0]) and np.array_equal(gv[layer], want[:, 1])
    finally:
        B.ts_kv_free(kv)
        B.ts_model_free(model)


# ---- together, over a cache of the library -------------------------------------------------------
@pytest.mark.parametrize("cfg_name", ["small_bf16", "small_fp32"])
@pytest.mark.parametrize("pooled", [False, True])
def test_a_layer_step_over_a_library_cache(cfg_name, pooled):
    """What a program with decoder blocks of its own does: rows appended to every layer of a cache that the library ingested,
    attention over it, the length extended - then the library goes on.  Compared with the cache's exported contents."""
    cfg = wl.get_config(cfg_name)
    model = B.ts_model_load(cfg, wl.gen_weights(cfg, 1234))
    pool = B.ts_kv_pool_create(model, 40) if pooled else None
    cap, n0 = 150, 101
    kvs = [B.ts_kv_alloc_pooled(pool, cap) if pooled else B.ts_kv_alloc(model, cap) for _ in range(2)]
    try:
        dt = torch.float32 if cfg.dtype == 0 else torch.bfloat16
        if not pooled:
            B.ts_kv_set_page_table(kvs[1], np.random.default_rng(0).permutation(10).astype(np.int32))
        kv = kvs[1]
        K, V = wl.gen_context_kv(cfg, n0, seed=5)
        B.ts_kv_import(kv, K, V)
        table = torch.from_numpy(ops.ts_kv_page_table(kv, cap)).cuda()[None]
        hd, hkv, hq = cfg.head_dim, cfg.n_kv_heads, cfg.n_q_heads
        new = 7
        x = torch.randn((new, (hq + 2 * hkv) * hd), generator=torch.Generator(device="cuda").manual_seed(1), device="cuda").to(dt)
        q, kk, vv = x.split((hq * hd, hkv * hd, hkv * hd), 1)
        outs = []
        for layer in range(cfg.n_layers):
            pages = ops.ts_kv_layer_pages(kv, layer)
            assert (pages.n_kv_heads, pages.head_dim, pages.dtype) == (hkv, hd, cfg.dtype)
            turned = ops.ts_kv_append(pages, None, table, ints([n0]), ints([0, new]), q, kk, vv, cfg.rope_theta)
            outs.append((turned[-1:], ops.ts_kv_attend(pages, None, table, ints([n0 + new]), turned[-1:], n0 + new)[0]))
        with pytest.raises(B.TsError) as e:
            ops.ts_kv_extend(kv, cap)
        assert e.value.status == B.TS_ERR_KV_CAPACITY
        ops.ts_kv_extend(kv, new)
        assert B.ts_kv_len(kv) == n0 + new
        gk, gv = B.ts_kv_export(kv, 0, n0 + new, cfg)
        as_t = lambda a: torch.from_numpy(a.astype(np.int32)).to(torch.int16).view(torch.bfloat16) if a.dtype == np.uint16 else torch.from_numpy(a)  # noqa: E731
        assert np.array_equal(gk[:, :n0], K) and np.array_equal(gv[:, :n0], V)
        for layer in range(cfg.n_layers):
            lk, lv = as_t(gk[layer]), as_t(gv[layer])
            for i in range(new):
                want, rough = plain_turn(kk[i].cpu().view(hkv, hd), n0 + i, cfg.rope_theta)
                assert near(lk[n0 + i], want, rough)
            assert torch.equal(lv[n0:], vv.cpu().view(new, hkv, hd))
            want, _, rough, d, _ = plain_attend(outs[layer][0][0].cpu(), lk, lv, hkv, hd, 0, hd ** -0.5)
            tol = (2 * d[:, None] + 2.0 ** -16 + 400 * 2.0 ** -24) * rough + torch.finfo(dt).eps / 2 * want.abs()
            assert bool(((outs[layer][1].double().cpu().view(hq, hd) - want).abs() <= tol).all())
        # the library's own pass goes on from there: the same as over a cache that was given these contents
        B.ts_kv_import(kvs[0], gk, gv)
        for c in kvs:
            B.ts_set_pending(c, 5)
        assert B.ts_verify(model, kvs[0], [7, 8, 9], [-1, 0, 0]) == B.ts_verify(model, kvs[1], [7, 8, 9], [-1, 0, 0])
        with pytest.raises(B.TsError):
            ops.ts_kv_layer_pages(kv, cfg.n_layers)
    finally:
        for c in kvs:
            B.ts_kv_free(c)
        if pool:
            B.ts_kv_pool_free(pool)
        B.ts_model_free(model)
