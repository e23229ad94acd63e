"""Paged caches of any type for tests: pages in random order, what they hold in 64 bits, and 8-bit values from their definition."""
import math

import torch

BF16, F32, E4M3 = torch.bfloat16, torch.float32, torch.float8_e4m3fn


def ints(x):
    return torch.tensor(list(x), dtype=torch.int32, device="cuda")


def scale_exponents(x):
    """[...][hd] in 64 bits -> the least e >= -127 with the largest magnitude at most 448 * 2^e (zeros: -127)."""
    top = x.abs().amax(-1)
    m, e = torch.frexp(top)                                    # top = m 2^e, 1/2 <= m < 1; 448 = 7/8 * 2^9
    e = e.long() - 9 + (m > 0.875)
    return torch.where(top > 0, e, -127).clamp(min=-127)


def round_e4m3(y):
    """The nearest e4m3 values (ties to even) of numbers of at most 448, in 64 bits."""
    _, e = torch.frexp(y.abs())
    step = torch.ldexp(torch.ones_like(y), (e - 1).clamp(min=-6) - 3)
    return torch.round(y / step) * step


def encode(x):
    """[...][hd] finite, in 64 bits -> (values over the scale, bytes of the scales)."""
    e = scale_exponents(x)
    return round_e4m3(torch.ldexp(x, -e[..., None])), (e + 127).to(torch.uint8)


class Pages:
    """pages = [k, v]; scales = [k_scales, v_scales] or None."""

    def __init__(self, pages, scales):
        self.pages, self.scales = pages, scales

    def clone(self):
        return Pages([x.clone() for x in self.pages], self.scales and [x.clone() for x in self.scales])


def cache_of(lengths, hkv, hd, dtype, seed, spare_pages=2, identity=False, extra=0):
    """(Pages, table, keys, values): keys[s] and values[s] are [n][hkv][hd] as the cache holds them (8 bits: in 64 bits).  Places without a
    position are NaN."""
    g = torch.Generator().manual_seed(seed)
    need = [max(1, -(-(n + extra) // 16)) for n in lengths]
    total = sum(need) + spare_pages
    order = torch.arange(total) if identity else torch.randperm(total, generator=g)
    table = torch.full((len(lengths), max(need) + 1), -1, dtype=torch.int32)
    eight = dtype == E4M3
    k = torch.full((total, hkv, 16, hd), math.nan, dtype=F32 if eight else dtype)
    v = torch.full((total, hkv, hd, 16), math.nan, dtype=F32 if eight else dtype)
    ks, vs = (torch.full((total, hkv, 16), 255, dtype=torch.uint8) for _ in range(2))
    at, K, V = 0, [], []
    for i, n in enumerate(lengths):
        pages = order[at:at + need[i]]
        at += need[i]
        table[i, :need[i]] = pages.to(torch.int32)
        p, s = pages[torch.arange(n) // 16], torch.arange(n) % 16
        a, b = (torch.randn((n, hkv, hd), generator=g) for _ in range(2))
        if eight:
            (ac, ab), (bc, bb) = encode(a.double() * torch.exp(torch.randn((n, hkv, 1), generator=g)).clamp(max=3)), encode(b.double())
            ks[p, :, s], vs[p, :, s] = ab, bb
            k[p, :, s], v[p, :, :, s] = ac.float(), bc.float()
            K.append(torch.ldexp(ac, ab.long()[..., None] - 127))
            V.append(torch.ldexp(bc, bb.long()[..., None] - 127))
        else:
            K.append(a.to(dtype))
            V.append(b.to(dtype))
            k[p, :, s], v[p, :, :, s] = K[i], V[i]
    if eight:
        k, v = k.to(E4M3), v.to(E4M3)
    return Pages([k.cuda(), v.cuda()], [ks.cuda(), vs.cuda()] if eight else None), table.cuda(), K, V


def store(pages, table, position, value):
    """Every key and value of a position of sequence 0 (all heads) becomes `value`; in 8-bit pages NaN is a scale, and codes of NaN."""
    page, slot = int(table[0, position // 16]), position % 16
    if pages.scales is None:
        pages.pages[0][page, :, slot] = value
        pages.pages[1][page, :, :, slot] = value
    else:
        pages.pages[0].view(torch.uint8)[page, :, slot] = 0x7f
        pages.pages[1].view(torch.uint8)[page, :, :, slot] = 0xff
        pages.scales[0][page, :, slot] = 255
        pages.scales[1][page, :, slot] = 255
