"""Attention of chunks with a scale of zero; and over 8-bit pages whose value scales a program wrote itself, at both ends of their range: a value stands for its e4m3 value times 2^e, infinite
from 2^128 on, whatever its probability, in calls of few columns and of many; against 64 bits with the tolerances of test_gpu_paged_rows."""
import math

import pytest
import torch

from paged_any import BF16, E4M3, F32, cache_of, ints
from paper_2604_13519_amd import ops
from test_gpu_paged_rows import plain, tolerance

pytestmark = pytest.mark.gpu


def stored(pages, table, n, which):
    """Keys or values of positions 0 .. n - 1 of sequence 0 in 64 bits, [n][kv heads][hd]: infinite from 2^128 on."""
    pos = torch.arange(n)
    page, slot = table.cpu()[0, pos // 16].long(), pos % 16
    x = pages.pages[which].cpu().float()
    x = (x[page, :, slot] if which == 0 else x[page, :, :, slot]).double()
    byte = pages.scales[which].cpu()[page, :, slot].long()
    x = torch.ldexp(x, byte[..., None] - 127)
    return torch.where(x.abs() >= 2.0 ** 128, torch.sign(x) * math.inf, x)


def set_values(pages, table, position, codes, byte):
    page, slot = int(table[0, position // 16]), position % 16
    pages.pages[1].view(torch.uint8)[page, :, :, slot] = codes
    pages.scales[1][page, :, slot] = byte


@pytest.mark.parametrize("qdtype", [BF16, F32])
@pytest.mark.parametrize("rows,n", [(1, 40), (1, 200), (1, 3000), (20, 40), (20, 3000)])
@pytest.mark.parametrize("byte,at", [(254, 3), (253, 35), (248, 3), (247, 17), (246, 20), (240, 0), (239, 1), (64, 2), (63, 18), (36, 2), (33, 3), (30, 3), (27, 1), (8, 33), (1, 5), (0, 6)])
def test_scales_at_their_ends(qdtype, rows, n, byte, at):
    """One position holds values of a far scale with a small probability, the others zeros (a far small scale) or ordinary values (a far large one)."""
    hq, hkv, hd = 4, 2, 64
    pages, table, _, _ = cache_of([n + rows], hkv, hd, E4M3, byte + n)
    total = n + rows
    if byte < 127:                                               # nothing but that position's values
        pages.pages[1].view(torch.uint8).zero_()
    codes = torch.arange(hd, dtype=torch.uint8) % 64 + 0x3f      # 1.875 .. 448, NaN left out below
    codes[codes == 0x7f] = 0x7e
    codes[1::3] |= 0x80
    set_values(pages, table, at, codes.cuda(), byte)
    # scores: the far position some 26 below the others, 2^-37 of the sum
    page, slot = int(table[0, at // 16]), at % 16
    pages.pages[0].view(torch.uint8)[:, :, :, 0] = 0x38          # 1
    pages.pages[0].view(torch.uint8)[page, :, slot, 0] = 0xb8    # -1
    pages.scales[0][page, :, slot] = 127
    pos = torch.arange(total)
    pages.scales[0][table.cpu()[0, pos // 16].long().cuda(), :, (pos % 16).cuda()] = 127
    q = torch.zeros((rows, hq, hd))
    q[..., 0] = 13.0
    K, V = stored(pages, table, total, 0), stored(pages, table, total, 1)
    out, lse = ops.ts_kv_attend_rows(*pages.pages, table, ints([n]), ints([0, rows]), q.to(qdtype).flatten(1).cuda(), total, scale=1.0, scales=pages.scales)
    out = out.double().cpu().view(rows, hq, hd)
    seen = torch.arange(total)[None] <= n + torch.arange(rows)[:, None]
    inf = V[at].isinf()                                          # [kv heads][hd]
    want, _, rough, d = plain(q.to(qdtype), K, torch.where(V.isinf(), 0.0, V), seen, 1.0)
    # bits of products below 2^-133 are lost, of up to three terms; a tiny output is rounded to the steps of its type there
    tol = tolerance(want, rough, d, total, E4M3, qdtype, rows * 2) - 1e-30 + 4 * 2.0 ** -133
    off = (out - want).abs() / tol
    for h in range(hq):
        i = inf[h // 2]
        assert bool((out[:, h, i] == V[at, h // 2, i]).all()), "infinite values: %s" % out[0, h, i]
        assert float(off[:, h, ~i].max() if bool((~i).any()) else 0) <= 1.0, off[:, h, ~i].max()


@pytest.mark.parametrize("dtype,qdtype", [(BF16, BF16), (BF16, F32), (F32, F32)])
@pytest.mark.parametrize("rows", [1, 20])
def test_an_infinite_product_with_a_scale_of_zero(dtype, qdtype, rows):
    """Zero times either infinity is no number: the heads that see such a score are NaN, the others the mean of what they see."""
    hq, hkv, hd, n = 4, 2, 64, 50
    pages, table, K, V = cache_of([n + rows], hkv, hd, dtype, 4)
    q = (torch.rand((rows, hq * hd), generator=torch.Generator().manual_seed(3)) + 0.01).to(qdtype).cuda()
    for at, bad in ((7, -math.inf), (7, math.inf), (n + rows - 1, -math.inf), (n + rows // 2, -math.inf)):
        other = pages.clone()
        other.pages[0][int(table[0, at // 16]), 1, at % 16] = bad
        for scale in (0.0, -0.0):
            out, lse = ops.ts_kv_attend_rows(*other.pages, table, ints([n]), ints([0, rows]), q, n + rows, scale=scale)
            out, lse = out.double().cpu().view(rows, hq, hd), lse.cpu()
            for r in range(rows):
                sees = n + r >= at
                assert bool(out[r, 2:].isnan().all()) == sees and bool(lse[r, 2:].isnan().all()) == sees, (at, bad, r)
                want = V[0][:n + r + 1].double().mean(0)
                for h in range(2 if sees else 4):
                    # equal weights: their sum, the values' sum and its rounding
                    tol = (2.0 ** -8 if qdtype == BF16 and rows > 8 else 2.0 ** -20) * V[0][:n + r + 1, h // 2].double().abs().mean(0) + torch.finfo(qdtype).eps / 2 * want[h // 2].abs() + 1e-6
                    assert bool(((out[r, h] - want[h // 2]).abs() <= tol).all()), (at, bad, r, h)
