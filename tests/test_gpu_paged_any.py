"""Rows into and out of paged caches of any type - norms of heads, rotations of every layout, 8-bit values - against plain 64-bit implementations,
and the calls over such caches together.

Tolerance of a normed value: hd squares summed in fp32 are good to (hd + 2) half steps, the root halves that, six roundings follow:
(hd / 2 + 8) 2^-24 of it.  Of a rotated one: the angle is reduced in 64 bits and rounded to 2^-26 of a turn (9e-8 radians), sine and cosine are
good to two steps, the magnitude and three fp32 roundings follow: 2^-21 (|x| + |y|) of the pair, and the errors of the two.  Then half a step
of the stored type; 8-bit values are within half a step of e4m3 of a value that near, at the scale that such a value gives."""
import math

import numpy as np
import pytest
import torch

import workloads as wl
from paged_any import BF16, E4M3, F32, cache_of, encode, ints, scale_exponents
from paper_2604_13519_amd import binding as B
from paper_2604_13519_amd import ops

pytestmark = pytest.mark.gpu

TYPES = [(BF16, BF16), (BF16, F32), (E4M3, BF16), (E4M3, F32), (F32, F32), (F32, BF16)]      # pages, rows


def plain_head(x, gain, eps, pos, rope):
    """[rows][heads][hd] in 64 bits, normed and turned: (values, tolerance)."""
    x = x.double()
    hd = x.shape[-1]
    tol = torch.zeros_like(x)
    if gain is not None:
        x = x / torch.sqrt(x.square().mean(-1, keepdim=True) + eps) * gain.double().cpu()
        tol = (hd / 2 + 8) * 2.0 ** -24 * x.abs()
    rd = rope.get("rope_dim")
    rd = hd if rd is None else rd
    theta, freqs = rope.get("rope_theta", 0.0), rope.get("rope_freqs")
    if rd == 0 or (theta == 0 and freqs is None):
        return x, tol
    f = freqs.double().cpu() if freqs is not None else torch.exp(-2.0 * torch.arange(rd // 2).double() / rd * math.log(np.float32(theta)))
    angle = pos.double()[:, None] * f
    mag = float(np.float32(rope.get("rope_magnitude", 1.0)))
    c, s = mag * torch.cos(angle)[:, None], mag * torch.sin(angle)[:, None]
    a_at, b_at = (slice(0, rd, 2), slice(1, rd, 2)) if rope.get("rope_pairs") else (slice(0, rd // 2), slice(rd // 2, rd))
    y, t = x.clone(), tol.clone()
    a, b, ta, tb = x[..., a_at], x[..., b_at], tol[..., a_at], tol[..., b_at]
    y[..., a_at], y[..., b_at] = a * c - b * s, b * c + a * s
    t[..., a_at] = t[..., b_at] = abs(mag) * ((ta + tb) + 2.0 ** -21 * (a.abs() + b.abs()))
    return y, t


def check_stored(got, want, tol, dtype, what):
    """Stored rows [..][hd] (8 bits: (values over the scale, bytes)) against 64-bit ones that are known to `tol`."""
    if dtype != E4M3:
        worst = ((got.double() - want).abs() / (tol + torch.finfo(dtype).eps / 2 * (want.abs() + tol) + 1e-40)).max()
        assert float(worst) <= 1.0, "%s: %.3g of the tolerance" % (what, float(worst))
        return
    codes, byte = got
    e = byte.long() - 127
    row_tol = tol.amax(-1, keepdim=True)
    low, high = scale_exponents((want.abs().amax(-1, keepdim=True) - row_tol).clamp(min=0)), scale_exponents(want.abs().amax(-1, keepdim=True) + row_tol)
    assert bool(((e >= low) & (e <= high)).all()), "%s: scales" % what
    y = torch.ldexp(want.abs() + tol, -e[..., None])
    _, m = torch.frexp(y)
    half = torch.ldexp(torch.ones_like(y), (m - 1).clamp(min=-6) - 4)
    off = (codes - torch.ldexp(want, -e[..., None])).abs() / (half + torch.ldexp(tol, -e[..., None]))
    assert float(off.max()) <= 1.0, "%s: %.3g half steps" % (what, float(off.max()))


def rows_of_pages(pages, table, seq, p0, n):
    """(keys, values) stored at positions, [n][hkv][hd]; of 8-bit pages each is (values over the scale, bytes)."""
    pos = torch.arange(p0, p0 + n)
    page, slot = table.cpu()[seq, pos // 16].long(), pos % 16
    k, v = (x.cpu() for x in pages.pages)
    if pages.scales is None:
        return k[page, :, slot], v[page, :, :, slot]
    ks, vs = (x.cpu() for x in pages.scales)
    return (k.double()[page, :, slot], ks[page, :, slot]), (v.double()[page, :, :, slot], vs[page, :, slot])


def check(before, new, hq, hkv, hd, dtype, rdtype, seed=0, norm=True, gain_dtype=None, eps=1e-6, positions=None, spare=0, fused=True, use_q=True, alias=False, **rope):
    print("append", before[:5], new[:5], hq, hkv, hd, dtype, rdtype, norm, {k: v if not isinstance(v, torch.Tensor) else "table" for k, v in rope.items()}, flush=True)
    pages, table, K, V = cache_of(before, hkv, hd, dtype, seed, extra=max(new))
    old = pages.clone()
    n, rows = len(new), sum(new) + spare
    g = torch.Generator().manual_seed(seed + 5)
    x = (torch.randn((rows, (hq + 2 * hkv) * hd), generator=g) * torch.exp(torch.randn((rows, 1), generator=g))).to(rdtype)
    q, k, v = x.split((hq * hd, hkv * hd, hkv * hd), 1)
    gains = [(1 + 0.2 * torch.randn(hd, generator=g)).to(gain_dtype or rdtype).cuda() if norm else None for _ in range(2)]
    offsets = [sum(new[:i]) for i in range(n + 1)]
    dq, dk, dv = (t.cuda() if not fused else None for t in (q, k, v))
    if fused:
        dq, dk, dv = x.cuda().split((hq * hd, hkv * hd, hkv * hd), 1)
    out = (dq if alias else torch.full((rows, hq * hd), 9.0, dtype=rdtype, device="cuda")) if use_q else None
    if not use_q:
        gains[0] = None
    at = None if positions is None else ints(positions + [3] * spare)
    got = ops.ts_kv_append_norm_rope(*pages.pages, table, ints(before), ints(offsets), dq if use_q else None, dk, dv, q_norm=gains[0], k_norm=gains[1], norm_eps=eps,
                                     positions=at, scales=pages.scales, q_out=out, **rope)
    assert got is out
    for i in range(n):
        a, b = offsets[i], offsets[i + 1]
        if a == b:
            continue
        pos = torch.arange(before[i], before[i] + new[i]) if positions is None else torch.tensor(positions[a:b])
        if use_q:
            want, tol = plain_head(q[a:b].reshape(b - a, hq, hd), gains[0], np.float32(eps).item(), pos, rope)
            check_stored(out[a:b].cpu().view(b - a, hq, hd), want, tol, rdtype, "queries of sequence %d" % i)
        ks, vs = rows_of_pages(pages, table, i, before[i], new[i])
        want, tol = plain_head(k[a:b].reshape(b - a, hkv, hd), gains[1], np.float32(eps).item(), pos, rope)
        check_stored(ks, want, tol, dtype, "keys of sequence %d" % i)
        want = v[a:b].reshape(b - a, hkv, hd)
        if dtype == E4M3:
            code, byte = encode(want.double())
            assert torch.equal(vs[1], byte) and torch.equal(vs[0], code), "values of sequence %d" % i
        else:
            assert torch.equal(vs, want.to(dtype)), "values of sequence %d" % i
        # everything else stays
        p = torch.arange(before[i], before[i] + new[i])
        page, slot = table.cpu()[i, p // 16].long().cuda(), (p % 16).cuda()
        for side in (pages, old):
            side.pages[0].view(torch.uint8 if dtype == E4M3 else dtype)[page, :, slot] = 0
            side.pages[1].view(torch.uint8 if dtype == E4M3 else dtype)[page, :, :, slot] = 0
            for s in side.scales or ():
                s[page, :, slot] = 0
    for x, y in zip(pages.pages + (pages.scales or []), old.pages + (old.scales or [])):
        assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))
    if use_q and spare and not alias:
        assert bool((out[sum(new):] == 9).all())


@pytest.mark.parametrize("dtype,rdtype", TYPES)
@pytest.mark.parametrize("hd", [64, 128])
def test_places_and_counts(dtype, rdtype, hd):
    for before, new in (([0], [1]), ([15], [1]), ([16], [17]), ([5], [11]), ([3], [12]), ([9], [60]), ([100, 0, 31, 7], [1, 1, 1, 1]), ([0, 40, 15, 2], [0, 33, 2, 5]), ([1], [300])):
        check(before, new, 4, 2, hd, dtype, rdtype, seed=sum(before) + sum(new), rope_theta=1e4, spare=len(new) % 3)


@pytest.mark.parametrize("dtype,rdtype", TYPES)
@pytest.mark.parametrize("hq,hkv", [(1, 1), (5, 5), (12, 3), (9, 9), (32, 8), (16, 1)])
def test_head_counts(dtype, rdtype, hq, hkv):
    check([30, 3], [7, 20], hq, hkv, 64, dtype, rdtype, seed=hq, rope_theta=5e5)
    check([30, 3, 0], [1, 1, 1], hq, hkv, 128, dtype, rdtype, seed=hq, rope_theta=5e5)


@pytest.mark.parametrize("rdtype", [F32, BF16])
@pytest.mark.parametrize("hd", [8, 16, 32, 64, 128])
def test_fp32_head_sizes(hd, rdtype):
    for rope in (dict(rope_theta=1e4), dict(rope_theta=1e4, rope_pairs=True), dict(rope_theta=1e4, rope_dim=hd // 2), dict(rope_theta=1e4, rope_dim=hd - 2)):
        check([10, 0], [9, 18], 6, 2, hd, F32, rdtype, seed=hd, **rope)


@pytest.mark.parametrize("dtype,rdtype", TYPES)
@pytest.mark.parametrize("pairs", [False, True])
def test_rotations(dtype, rdtype, pairs):
    for hd in (64, 128):
        for rd in (0, 2, 6, 16, 30, 32, hd // 2, hd - 2, hd):
            check([70, 5], [3, 19], 3, 1, hd, dtype, rdtype, seed=rd, rope_dim=rd, rope_pairs=pairs, rope_theta=1e4)
    f = torch.rand(24, generator=torch.Generator().manual_seed(1)).cuda() * 2
    check([70, 5], [3, 19], 3, 1, 64, dtype, rdtype, rope_dim=48, rope_pairs=pairs, rope_freqs=f, rope_magnitude=1.2079)
    check([70, 5], [3, 19], 3, 1, 64, dtype, rdtype, rope_dim=48, rope_pairs=pairs, rope_freqs=f, rope_theta=77.0, rope_magnitude=-0.5, norm=False)
    check([70, 5], [3, 19], 3, 1, 64, dtype, rdtype, rope_pairs=pairs, rope_theta=0.0)


@pytest.mark.parametrize("dtype,rdtype", TYPES)
def test_norms(dtype, rdtype):
    for kw in (dict(eps=0.0), dict(eps=1.0), dict(gain_dtype=F32), dict(gain_dtype=BF16), dict(norm=False), dict(use_q=False), dict(fused=False), dict(alias=True, fused=False), dict(alias=True)):
        check([33, 4], [5, 30], 4, 2, 128, dtype, rdtype, rope_theta=1e6, seed=3, **kw)
        check([33, 4], [1, 1], 4, 2, 64, dtype, rdtype, rope_theta=1e6, seed=4, **kw)


@pytest.mark.parametrize("dtype,rdtype", [(BF16, BF16), (E4M3, BF16), (F32, F32)])
def test_far_and_given_positions(dtype, rdtype):
    check([200, 7], [20, 3], 4, 2, 64, dtype, rdtype, rope_theta=1e4, positions=[200 + d for d in range(0, 40, 2)] + [7, 9, 9])
    check([200], [5], 4, 2, 64, dtype, rdtype, rope_theta=1e4, positions=[0, -5, 1 << 20, (1 << 31) - 1, -(1 << 31)])
    f = torch.tensor([1.0, 1e-3, 3.1], device="cuda")
    check([200], [5], 4, 2, 64, dtype, rdtype, rope_freqs=f, rope_dim=6, positions=[0, -5, 1 << 20, (1 << 31) - 1, -(1 << 31)])


@pytest.mark.parametrize("dtype,rdtype", [(BF16, BF16), (E4M3, BF16), (F32, F32), (E4M3, F32)])
def test_many_rows_and_sequences(dtype, rdtype):
    check([0], [1500], 2, 1, 64, dtype, rdtype, rope_theta=1e4)
    check([i % 37 for i in range(300)], [1 + i % 3 for i in range(300)], 2, 2, 64, dtype, rdtype, rope_theta=1e4, spare=5)


def test_eight_bit_borders():
    """Scales at their borders, subnormal values, zeros, the largest numbers, infinities and NaN, as values and (without norm and rotation) as keys."""
    hd = 64
    rows = []
    for top in (448.0, 448.0 * (1 + 2.0 ** -23), 449.0, 447.9, 256.0, 1.75, 1.7500001, 1.0, 2.0 ** -100, 2.0 ** -126, 2.0 ** -127, 2.0 ** -140, 2.0 ** -149, 2.0 ** 127, 1.75 * 2.0 ** 127, 0.0):
        x = torch.tensor([top * (1 - 1 / 64) ** (5 * j) * (-1) ** j for j in range(hd)], dtype=torch.float32)
        x[0] = top
        x[1] = -0.0
        rows.append(x)
    ties = torch.tensor([448.0] + [s * (m + 0.5) * 2.0 ** (e - 3) for e in range(-6, 8) for m in (8, 9, 14, 15) for s in (1, -1)][:hd - 1], dtype=torch.float32)
    small = torch.tensor([448.0] + [(j + 0.5) * 2.0 ** -9 for j in range(20)] + [j * 2.0 ** -10 for j in range(hd - 21)], dtype=torch.float32)
    rows += [ties, small, ties * 2.0 ** -130, small * 2.0 ** 100]
    finite = len(rows)
    for bad in (math.inf, -math.inf, math.nan):
        x = torch.randn(hd)
        x[13] = bad
        rows.append(x)
    x = torch.stack(rows)
    for first in (0, 3):
        pages, table, _, _ = cache_of([0], 1, hd, E4M3, 1, extra=len(rows) + first)
        pages.scales[0].zero_()
        ops.ts_kv_append_norm_rope(*pages.pages, table, ints([first]), ints([0, len(rows)]), None, x.cuda(), x.cuda(), scales=pages.scales)
        code, byte = encode(x[:finite].double())
        for got, got_byte in rows_of_pages(pages, table, 0, first, len(rows)):
            assert torch.equal(got_byte[:finite, 0], byte) and torch.equal(got[:finite, 0], code)
            assert bool((got_byte[finite:] == 255).all()) and bool(got[finite:].isnan().all())
        k, v = ops.ts_kv_read(*pages.pages, table, ints([first]), ints([0, len(rows)]), len(rows), dtype=F32, scales=pages.scales)
        for t in (k, v):
            t = t.cpu()
            assert torch.equal(t[:finite].double(), torch.ldexp(code, byte.long()[:, None] - 127)) and bool(t[finite:].isnan().all())


def test_numbers_that_norms_meet():
    hd = 64
    x = torch.zeros((4, hd))
    x[1] = 3e38                                                 # squares beyond fp32: zeros
    x[2, 5] = math.nan
    x[3] = 1e-30
    one = torch.ones(hd, device="cuda")
    pages, table, _, _ = cache_of([0], 1, hd, F32, 1, extra=4)
    out = ops.ts_kv_append_norm_rope(*pages.pages, table, ints([0]), ints([0, 4]), x.cuda(), x.cuda(), x.cuda(), q_norm=one, k_norm=one, norm_eps=0.0)
    out = out.cpu()
    assert bool(out[0].isnan().all()) and bool((out[1] == 0).all()) and bool(out[2].isnan().all()) and bool(out[3].isnan().logical_or(out[3].isinf()).all())
    out = ops.ts_kv_append_norm_rope(*pages.pages, table, ints([0]), ints([0, 4]), x.cuda(), x.cuda(), x.cuda(), q_norm=one, k_norm=one, norm_eps=1e-6).cpu()
    assert bool((out[:2] == 0).all()) and bool(out[2].isnan().all()) and float((out[3] - 1e-27).abs().max()) <= 1e-33


def test_rows_that_have_no_place_leave_everything_as_it_was():
    for dtype in (BF16, E4M3, F32):
        hd = 64
        pages, table, _, _ = cache_of([40], 2, hd, dtype, 4)
        old = pages.clone()
        x = torch.randn((20, 2 * hd), device="cuda").to(BF16)
        out = torch.full((20, 2 * hd), 9.0, dtype=BF16, device="cuda")
        call = lambda t, n, off: ops.ts_kv_append_norm_rope(*pages.pages, t, ints(n), ints(off), x, x, x, rope_theta=1e4, scales=pages.scales, q_out=out)  # noqa: E731
        bad = table.clone()
        for page in (-1, 1 << 30, -(1 << 31), pages.pages[0].shape[0]):
            bad[:] = page
            call(bad, [0], [0, 20])
        for n in (1 << 30, (1 << 31) - 1, -(1 << 31), -20, 16 * table.shape[1]):
            call(table, [n], [0, 20])
        for off in ((20, 20), (20, 0), (5, 3), ((1 << 31) - 1, -(1 << 31)), (1 << 30, (1 << 31) - 1)):
            call(table, [0], off)
        assert bool((out == 9).all())
        for a, b in zip(pages.pages + (pages.scales or []), old.pages + (old.scales or [])):
            assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
        for off in ((0, 1 << 30), (-(1 << 31), 20), (-3, 4), (0, 30, 2, 20)):               # stay in bounds
            call(torch.cat([table] * (len(off) - 1)), [0] * (len(off) - 1), off)
        call(table, [-8], [0, 20])                                # rows 8 .. have positions 0 ..
        (k, v) = rows_of_pages(pages, table, 0, 0, 12)
        want = x[8:].cpu().view(12, 2, hd)
        assert torch.equal(v if dtype != E4M3 else v[0], want.to(dtype) if dtype != E4M3 else encode(want.double())[0])


@pytest.mark.parametrize("dtype", [BF16, F32, E4M3])
@pytest.mark.parametrize("to", [BF16, F32])
def test_read(dtype, to):
    for hd, hkv in ((64, 1), (128, 3), (64, 9)) + (((8, 2), (16, 5), (32, 1)) if dtype == F32 else ()):
        lengths, starts, new = [40, 300, 1, 17, 64], [3, 0, 0, 16, 5], [30, 290, 1, 0, 20]
        pages, table, K, V = cache_of(lengths, hkv, hd, dtype, hd + hkv)
        off = [sum(new[:i]) for i in range(6)]
        k, v = (torch.full((off[-1] + 2, hkv * hd + 8), 5.0, dtype=to, device="cuda") for _ in range(2))
        got = ops.ts_kv_read(*pages.pages, table, ints(starts), ints(off), off[-1] + 2, dtype=to, scales=pages.scales, k_out=k[:, 3:3 + hkv * hd], v_out=v[:, 5:5 + hkv * hd])
        for i in range(5):
            for g, X in zip(got, (K, V)):
                assert torch.equal(g[off[i]:off[i + 1]].cpu(), X[i][starts[i]:starts[i] + new[i]].flatten(1).to(to)), (hd, i)
        assert bool((got[0][off[-1]:] == 5).all()) and bool((k[:, :3] == 5).all()) and bool((k[:, 3 + hkv * hd:] == 5).all()) and bool((v[:, :5] == 5).all())
        a, b = ops.ts_kv_read(*pages.pages, table, None, ints([0] + [sum(lengths[:i + 1]) for i in range(5)]), sum(lengths) + 1, dtype=to, scales=pages.scales)
        assert torch.equal(a[:-1].cpu(), torch.cat(K).reshape(sum(lengths), -1).to(to)) and torch.equal(b[:-1].cpu(), torch.cat(V).reshape(sum(lengths), -1).to(to))
        assert bool((a[-1] == 0).all())
        only = torch.zeros_like(b)
        none, same = ops.ts_kv_read(*pages.pages, table, None, ints([0] + [sum(lengths[:i + 1]) for i in range(5)]), sum(lengths) + 1, dtype=to, scales=pages.scales, v_out=only)
        assert none is None and same is only and torch.equal(only, b)


def test_read_of_places_that_are_none():
    for dtype in (BF16, E4M3, F32):
        pages, table, K, V = cache_of([64], 2, 64, dtype, 4)
        k, v = (torch.full((20, 128), 9.0, device="cuda") for _ in range(2))
        call = lambda t, start, off: ops.ts_kv_read(*pages.pages, t, ints(start), ints(off), 20, dtype=F32, scales=pages.scales, k_out=k, v_out=v)  # noqa: E731
        bad = table.clone()
        for page in (-1, 1 << 30, -(1 << 31), pages.pages[0].shape[0]):
            bad[:] = page
            call(bad, [0], [0, 20])
        for n in (1 << 30, (1 << 31) - 1, -(1 << 31), -20, 16 * table.shape[1]):
            call(table, [n], [0, 20])
        for off in ((20, 20), (20, 0), (5, 3), ((1 << 31) - 1, -(1 << 31))):
            call(table, [0], off)
        assert bool((k == 9).all()) and bool((v == 9).all())
        for off in ((0, 1 << 30), (-(1 << 31), 20), (-3, 4), (0, 30, 2, 20)):               # stay in bounds
            call(torch.cat([table] * (len(off) - 1)), [0] * (len(off) - 1), off)
        call(table, [-8], [0, 20])
        assert torch.equal(k[8:].cpu().double(), K[0][:12].reshape(12, -1).double())


@pytest.mark.parametrize("dtype", [BF16, E4M3, F32])
def test_a_prompt_in_pieces_then_tokens_then_a_tree(dtype):
    """The calls as a program uses them: chunks of a prompt, single tokens (a captured step, replayed), a draft tree whose rows are turned by their depths;
    all against one plain pass over what the cache holds."""
    hq, hkv, hd, rd = 8, 2, 64, 48
    rdtype = F32 if dtype == F32 else BF16
    g = torch.Generator().manual_seed(3)
    total, pieces = 200, [90, 64, 1, 45]
    pages, table, _, _ = cache_of([0], hkv, hd, dtype, 2, extra=total + 40)
    x = torch.randn((total + 34, (hq + 2 * hkv) * hd), generator=g).to(rdtype).cuda()
    gains = [(1 + 0.2 * torch.randn(hd, generator=g)).to(rdtype).cuda() for _ in range(2)]
    kw = dict(rope_theta=1e4, rope_dim=rd, q_norm=gains[0], k_norm=gains[1], scales=pages.scales)
    split = (hq * hd, hkv * hd, hkv * hd)
    outs, queries, at = [], [], 0
    for n in pieces:
        q, k, v = x[at:at + n].split(split, 1)
        queries.append(ops.ts_kv_append_norm_rope(*pages.pages, table, ints([at]), ints([0, n]), q, k, v, **kw))
        outs.append(ops.ts_kv_attend_rows(*pages.pages, table, ints([at]), ints([0, n]), queries[-1], total + 40, scales=pages.scales)[0])
        at += n
    # ten tokens, one captured step
    length, row, one = ints([at]), x[at:at + 1].clone(), ints([0, 1])
    q, k, v = row.split(split, 1)
    q_out, out, lse = torch.zeros_like(q).contiguous(), torch.zeros((1, hq * hd), dtype=rdtype, device="cuda"), torch.zeros((1, hq), device="cuda")
    ws = ops.ts_kv_attend_rows_workspace(1, 1, hq, hkv, hd, total + 40)

    def step():
        ops.ts_kv_append_norm_rope(*pages.pages, table, length, one, q, k, v, q_out=q_out, **kw)
        ops.ts_kv_attend_rows(*pages.pages, table, length, one, q_out, total + 40, scales=pages.scales, workspace=ws, out=out, lse=lse)
    step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(10):
        row.copy_(x[at:at + 1])
        length.fill_(at)
        graph.replay()
        torch.cuda.synchronize()
        queries.append(q_out.clone())
        outs.append(out.clone())
        at += 1
    # a tree: two branches behind a root
    depth = [0] + list(range(1, 13)) + list(range(1, 12))
    sets, branch = [0], [0, 0]
    for j in range(1, 24):
        b = 0 if j <= 12 else 1
        branch[b] |= 1 << (j - 1)
        sets.append(branch[b])
    q, k, v = x[at:at + 24].split(split, 1)
    queries.append(ops.ts_kv_append_norm_rope(*pages.pages, table, ints([at]), ints([0, 24]), q, k, v, positions=ints([at + d for d in depth]), **kw))
    outs.append(ops.ts_kv_attend_rows(*pages.pages, table, ints([at]), ints([0, 24]), queries[-1], total + 40, scales=pages.scales,
                                      ancestors=torch.tensor(sets, device="cuda"))[0])
    n = at + 24
    stored = ops.ts_kv_read(*pages.pages, table, None, ints([0, n]), n, dtype=F32, scales=pages.scales)
    K, V = (t.cpu().view(n, hkv, hd) for t in stored)
    pos = torch.tensor(list(range(at)) + [at + d for d in depth])
    want, tol = plain_head(x[:n, :hq * hd].cpu().reshape(n, hq, hd), gains[0], 1e-6, pos, dict(rope_theta=1e4, rope_dim=rd))
    check_stored(torch.cat(queries).cpu().view(n, hq, hd), want, tol, rdtype, "queries")
    want, tol = plain_head(x[:n, hq * hd:(hq + hkv) * hd].cpu().reshape(n, hkv, hd), gains[1], 1e-6, pos, dict(rope_theta=1e4, rope_dim=rd))
    ks = rows_of_pages(pages, table, 0, 0, n)[0]
    check_stored(ks, want, tol, dtype, "keys")
    from test_gpu_paged_rows import plain, seen_of, tolerance
    seen = torch.zeros((n, n), dtype=torch.bool)
    seen[:at, :at] = seen_of(0, at)
    seen[at:] = seen_of(at, 24, sets=sets)
    want, _, rough, d = plain(torch.cat(queries).cpu().view(n, hq, hd), K, V, seen, hd ** -0.5)
    assert bool(((torch.cat(outs).double().cpu().view(n, hq, hd) - want).abs() <= tolerance(want, rough, d, n, dtype, rdtype, 1000)).all())


def test_over_a_library_cache():
    """The pages of the library's own caches, and its passes after rows that these calls wrote."""
    cfg = wl.get_config("small_bf16")
    model = B.ts_model_load(cfg, wl.gen_weights(cfg, 1234))
    kv = B.ts_kv_alloc(model, 200)
    try:
        g = torch.Generator().manual_seed(3)
        table = torch.from_numpy(ops.ts_kv_page_table(kv, 200))[None].cuda()
        hq, hkv, hd, n = cfg.n_q_heads, cfg.n_kv_heads, cfg.head_dim, 50
        for layer in range(cfg.n_layers):
            x = torch.randn((n, (hq + 2 * hkv) * hd), generator=g).to(BF16).cuda()
            q, k, v = x.split((hq * hd, hkv * hd, hkv * hd), 1)
            pages = ops.ts_kv_layer_pages(kv, layer)
            q = ops.ts_kv_append_norm_rope(pages, None, table, ints([0]), ints([0, n]), q, k, v, rope_theta=cfg.rope_theta)
            out, lse = ops.ts_kv_attend_rows(pages, None, table, ints([0]), ints([0, n]), q, 200)
            last, last_lse = ops.ts_kv_attend(pages, None, table, ints([n]), q[-1:], 200)
            assert float((out[-1:].double() - last.double()).abs().max()) <= 2.0 ** -6 and float((lse[-1:] - last_lse).abs().max()) <= 1e-5
            kr, vr = ops.ts_kv_read(pages, None, table, None, ints([0, n]), n)
            assert torch.equal(vr, v)
        ops.ts_kv_extend(kv, n)
        ks, vs = B.ts_kv_export(kv, 0, n, cfg)
        assert np.array_equal(np.asarray(ks[-1]).reshape(n, -1), kr.view(torch.int16).cpu().numpy().view(np.uint16).reshape(n, -1))
        B.ts_set_pending(kv, 5)
        assert B.ts_verify(model, kv, [7, 8], [-1, 0])[0] >= 0
    finally:
        B.ts_kv_free(kv)
        B.ts_model_free(model)
