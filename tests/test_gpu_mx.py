"""4-bit microscaled values on the GPU against their definition in 64 bits.

Quantising divides by a power of two and rounds once, so it is compared exactly.  The product has exact terms (a weight
has two significant bits, fp32 rows are three bf16 terms) and fp32 sums: n additions in any order err by less than
n 2^-24 times the sum of the magnitudes, n = K (three times that for fp32 rows) + 16 for the groups of waves; the result
is rounded once to its type, half a step of it more."""
import math

import pytest
import torch

from paper_2604_13519_amd import binding as B
from paper_2604_13519_amd import ops

pytestmark = pytest.mark.gpu
GRID = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64)


def definition(x):
    """Values (64 bits) and scale bytes of rows of any float type, on the CPU, straight from the definition."""
    x = x.detach().cpu().double()
    rows, cols = x.shape
    blocks = -(-cols // 32)
    pad = torch.zeros((rows, blocks * 32), dtype=torch.float64)
    pad[:, :cols] = x
    b = pad.view(rows, blocks, 32)
    bad = ~torch.isfinite(b).all(2)
    b = torch.where(bad[..., None], 0.0, b)
    a = b.abs().amax(2)
    e = torch.where(a > 0, torch.frexp(a).exponent - 1 - 2, -127).clamp(-127, 127)
    scale = torch.pow(torch.tensor(2.0, dtype=torch.float64), e.double())
    v = b.abs() / scale[..., None]
    d = (v[..., None] - GRID).abs()
    best = d.amin(-1, keepdim=True)
    near = d == best                                           # one code, or two at a tie: then the even one
    code = torch.arange(8)
    pick = torch.where(near, torch.where(code % 2 == 0, 0, 1), 2).argmin(-1)
    val = torch.sign(b) * GRID[pick] * scale[..., None]
    val[bad] = math.nan
    return val.view(rows, -1)[:, :cols], torch.where(bad, 255, e + 127).to(torch.uint8)


def same(a, b):
    a, b = a.double().cpu(), b.double().cpu()
    return bool(((a == b) | (a.isnan() & b.isnan())).all())


def check_quantize(x, tag):
    print("quantize", tag, tuple(x.shape), x.dtype, flush=True)
    codes, scales = ops.ts_mx_quantize(x)
    want, want_scales = definition(x)
    for dt in (torch.float32, torch.bfloat16):
        assert same(ops.ts_mx_dequantize(codes, scales, x.shape[1], dt), want), tag
    assert torch.equal(scales.cpu(), want_scales), tag
    if x.shape[1] % 32:                                        # behind the row's end: zeros
        tail = codes.view(x.shape[0], -1, 16)[:, -1]
        nib = torch.stack((tail & 15, tail >> 4), 2).view(x.shape[0], 32)
        assert int(nib[:, x.shape[1] % 32:].max()) == 0
    return codes, scales


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_quantize_every_grid_point_and_tie(dtype):
    """All magnitudes around the grid in steps of 1/64, both signs, under scales from the smallest to the largest."""
    steps = torch.arange(0, 512).double() / 64                 # up to 8
    for e in (-126, -100, -3, 0, 1, 60, 124):
        vals = torch.cat([steps, -steps]) * 2.0 ** e
        rows = vals.view(-1, 1).repeat(1, 32)
        rows[:, 0] = 7.875 * 2.0 ** e                          # fixes the scale: 2^e
        check_quantize(rows.to(dtype).cuda(), "grid 2^%d" % e)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 31), (3, 32), (5, 33), (2, 64), (7, 1000), (1, 4096), (129, 257), (33, 8), (300, 96)])
def test_quantize_shapes_strides_alignment(dtype, rows, cols):
    g = torch.Generator(device="cuda").manual_seed(rows * 1000 + cols)
    x = torch.randn((rows, cols), generator=g, device="cuda") * torch.exp(3 * torch.randn((rows, 1), generator=g, device="cuda"))
    check_quantize(x.to(dtype), "dense")
    for off, extra in ((0, 5), (1, 8), (3, 13)):
        wide = torch.full((rows, cols + off + extra), math.nan, dtype=dtype, device="cuda")
        wide[:, off:off + cols] = x.to(dtype)
        check_quantize(wide[:, off:off + cols], "offset %d, stride + %d" % (off, off + extra))


def test_quantize_special_values():
    x = torch.zeros((12, 64), device="cuda")
    x[1, 3], x[2, 40], x[3, 5] = math.inf, -math.inf, math.nan
    x[4] = -0.0
    x[5, 0] = 1e-45                                            # the smallest fp32
    x[6, :40] = 2.0 ** -127                                    # subnormal throughout
    x[7, 0], x[7, 1] = 3.4e38, -3.3e38
    x[8, 0], x[8, 33] = 2.0 ** -125, 2.0 ** -126
    x[9] = torch.linspace(-1, 1, 64, device="cuda") * 2.0 ** -126
    x[10, 0], x[10, 1:] = 1.0, 2.0 ** -3 * 1.0000001           # a hair above a tie
    x[11, 0], x[11, 1:] = 1.0, 2.0 ** -4
    check_quantize(x, "special")
    check_quantize(x.bfloat16(), "special bf16")


def test_quantize_is_idempotent():
    x = torch.randn((64, 512), device="cuda") * torch.exp2(torch.randint(-20, 20, (64, 512), device="cuda").float())
    c, s = ops.ts_mx_quantize(x)
    v = ops.ts_mx_dequantize(c, s, 512)
    assert torch.equal(ops.ts_mx_dequantize(*ops.ts_mx_quantize(v), 512), v)


def test_dequantize_every_code_and_scale():
    codes = torch.arange(256, dtype=torch.uint8, device="cuda").view(16, 16)
    for s in (0, 1, 2, 126, 127, 128, 250, 252, 255):
        scales = torch.full((16, 1), s, dtype=torch.uint8, device="cuda")
        c = codes.cpu().int()
        nib = torch.stack((c & 15, c >> 4), 2).view(16, 32)
        want = GRID[nib % 8] * torch.where(nib >= 8, -1.0, 1.0).double() * 2.0 ** (s - 127) if s != 255 else torch.full((16, 32), math.nan)
        for dt in (torch.float32, torch.bfloat16):
            assert same(ops.ts_mx_dequantize(codes, scales, 32, dt), want), (s, dt)


def test_scales_whose_values_pass_fp32():
    """Scale bytes that quantising never writes: values up to 2^128 - 1 step as they are, infinities beyond, in both types and in the product."""
    codes = torch.zeros((16, 16), dtype=torch.uint8, device="cuda")
    codes[:, 0] = torch.arange(16, dtype=torch.uint8, device="cuda")
    for s in (252, 253, 254):
        scales = torch.full((16, 1), s, dtype=torch.uint8, device="cuda")
        want = GRID[torch.arange(16) % 8] * torch.where(torch.arange(16) >= 8, -1.0, 1.0).double() * 2.0 ** (s - 127)
        want = torch.where(want.abs() >= 2.0 ** 128, torch.sign(want) * math.inf, want)
        for dt in (torch.float32, torch.bfloat16):
            assert same(ops.ts_mx_dequantize(codes, scales, 32, dt)[:, 0], want), (s, dt)
            x = torch.zeros((3, 32), dtype=dt, device="cuda")
            x[:, 0] = 0.125
            y = ops.ts_mx_project(ops.ts_mx_pack(codes, scales, 32), 16, x).double().cpu()
            finite = torch.isfinite(want)
            assert bool((y[:, finite] == want[finite] / 8).all()) and not bool(torch.isfinite(y[:, ~finite]).any()), (s, dt)


def weights(n_out, n_in, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    w = torch.randn((n_out, n_in), generator=g, device="cuda") * torch.exp2(torch.randint(-6, 6, (n_out, 1), generator=g, device="cuda").float())
    codes, scales = ops.ts_mx_quantize(w)
    return ops.ts_mx_pack(codes, scales, n_in), ops.ts_mx_dequantize(codes, scales, n_in).double()


def bound(x, w, y, dtype):
    k = x.shape[1] * (3 if dtype == torch.float32 else 1) + 16
    return k * 2.0 ** -24 * (x.abs() @ w.abs().t().contiguous()) + torch.finfo(dtype).eps / 2 * y.abs()


def check_project(packed, w, x, tag, out=None):
    print("project", tag, tuple(x.shape), x.dtype, w.shape[0], flush=True)
    y = ops.ts_mx_project(packed, w.shape[0], x, out)
    x64 = x.double().contiguous()
    want = x64 @ w.t().contiguous()
    tol = bound(x64, w, want, x.dtype) * 1.01
    worst = ((y.double() - want).abs() / tol.clamp(min=1e-300)).max().item()
    assert worst <= 1.0, "%s: %.3g of the tolerance" % (tag, worst)
    return y


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("n_in,n_out", [(1, 1), (31, 3), (32, 16), (33, 17), (127, 15), (128, 64), (129, 130), (256, 33), (1000, 200), (1024, 1031), (4100, 96)])
def test_project_shapes(dtype, n_in, n_out):
    packed, w = weights(n_out, n_in, n_in + n_out)
    g = torch.Generator(device="cuda").manual_seed(7)
    for rows in (1, 2, 15, 16, 17, 32, 33, 48, 49, 64, 65, 80, 81, 128, 129, 300):
        x = torch.randn((rows, n_in), generator=g, device="cuda").to(dtype)
        check_project(packed, w, x, "dense")


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows", [1, 19, 77, 150])
def test_project_strides_and_neighbours(dtype, rows):
    """Rows inside wider ones filled with NaN: nothing outside is read into a result or written."""
    for n_in, n_out, off in ((96, 40, 0), (200, 50, 1), (513, 131, 3), (640, 256, 8)):
        packed, w = weights(n_out, n_in, 3)
        g = torch.Generator(device="cuda").manual_seed(rows)
        wide = torch.full((rows, n_in + off + 8), math.nan, dtype=dtype, device="cuda")
        wide[:, off:off + n_in] = torch.randn((rows, n_in), generator=g, device="cuda").to(dtype)
        out = torch.full((rows + 2, n_out + off + 8), 7.0, dtype=dtype, device="cuda")
        view = out[1:1 + rows, off:off + n_out]
        check_project(packed, w, wide[:, off:off + n_in], "strided %d" % off, view)
        out[1:1 + rows, off:off + n_out] = 7.0
        assert bool((out == 7.0).all())


def test_project_infinities_stay_in_their_rows_and_columns():
    packed, w = weights(96, 256, 5)
    for dtype in (torch.bfloat16, torch.float32):
        for rows in (5, 70, 200):
            x = torch.randn((rows, 256), device="cuda").to(dtype)
            clean = ops.ts_mx_project(packed, 96, x)
            x[2, 7], x[4, 100] = math.inf, math.nan
            y = ops.ts_mx_project(packed, 96, x)
            keep = [r for r in range(rows) if r not in (2, 4)]
            assert torch.equal(y[keep], clean[keep])
            assert bool(y[4].isnan().all())
            want = x.double()[2:3] @ w.t().contiguous()
            assert same(y[2:3].isinf(), want.isinf()) and same(y[2:3].isnan(), want.isnan())
    codes, scales = ops.ts_mx_quantize(torch.randn((40, 160), device="cuda"))
    scales[3, 2] = 255
    y = ops.ts_mx_project(ops.ts_mx_pack(codes, scales, 160), 40, torch.ones((9, 160), device="cuda"))
    assert bool(y[:, 3].isnan().all()) and int(y.isnan().sum()) == 9


@pytest.mark.parametrize("rows", [1, 5, 33, 100, 600])
def test_project_finite_rows_give_finite_sums(rows):
    """fp32 rows with one value each, of 24 bits and of any size up to the largest, over weights of any code: what does not
    overflow is finite, and a code of zero gives zero.  An output is the sum of three exact products of one sign: two additions."""
    n_out, n_in = 96, 300
    gen = torch.Generator(device="cuda").manual_seed(rows)
    codes = torch.randint(0, 256, (n_out, 160), dtype=torch.uint8, device="cuda", generator=gen)
    scales = torch.randint(40, 124, (n_out, 10), dtype=torch.uint8, device="cuda", generator=gen)
    w = ops.ts_mx_dequantize(codes, scales, n_in).double()
    top = torch.finfo(torch.float32).max
    for value in (top, -top, 3.397e38, 1.9999999 * 2.0 ** 100, -1.5 * 2.0 ** 127, 1.0000001):
        x = torch.zeros((rows, n_in), device="cuda")
        at = torch.randint(0, n_in, (rows,), device="cuda", generator=gen)
        x[torch.arange(rows, device="cuda"), at] = value
        y = ops.ts_mx_project(ops.ts_mx_pack(codes, scales, n_in), n_out, x).double()
        want = float(torch.tensor(value, dtype=torch.float32)) * w[:, at].t()
        assert bool(torch.isfinite(y).all()), (rows, value)
        assert bool(((y - want).abs() <= 2.0 ** -22 * want.abs()).all()), (rows, value)


def test_project_extreme_scales():
    """fp32 sums of the smallest and the largest weights; scales down to 2^-127."""
    for e in (0, 1, 40, 200, 230):
        codes = torch.randint(0, 256, (33, 64), dtype=torch.uint8, device="cuda")
        scales = torch.full((33, 4), e, dtype=torch.uint8, device="cuda")
        w = ops.ts_mx_dequantize(codes, scales, 128).double()
        x = torch.randn((5, 128), device="cuda").bfloat16() * (2.0 ** 20 if e < 2 else 1.0)
        y = ops.ts_mx_project(ops.ts_mx_pack(codes, scales, 128), 33, x.bfloat16()).double()
        want = x.double() @ w.t().contiguous()
        tol = bound(x.double(), w, want, torch.bfloat16) + 2.0 ** -133
        assert bool(((y - want).abs() <= tol).all()), e


def test_project_repeats_bit_for_bit_and_rows_are_independent():
    packed, _ = weights(1031, 999, 11)
    for dtype in (torch.bfloat16, torch.float32):
        for rows in (1, 16, 40, 70, 260):
            x = torch.randn((rows, 999), device="cuda").to(dtype)
            y = ops.ts_mx_project(packed, 1031, x)
            for _ in range(3):
                assert torch.equal(ops.ts_mx_project(packed, 1031, x), y)
            z = x.flip(0).contiguous()
            assert torch.equal(ops.ts_mx_project(packed, 1031, z).flip(0), y)


def test_on_another_stream_and_captured():
    packed, w = weights(256, 512, 21)
    x = torch.randn((33, 512), device="cuda").bfloat16()
    want = ops.ts_mx_project(packed, 256, x)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        y = ops.ts_mx_project(packed, 256, x)
    s.synchronize()
    assert torch.equal(y, want)
    out = torch.zeros_like(want)
    codes = torch.empty((33, 256), dtype=torch.uint8, device="cuda")
    scales = torch.empty((33, 16), dtype=torch.uint8, device="cuda")
    g = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g):
        ops.ts_mx_project(packed, 256, x, out)
        ops.ts_mx_quantize(x, codes, scales)
    for seed in range(4):
        x.copy_(torch.randn((33, 512), generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda"))
        out.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, ops.ts_mx_project(packed, 256, x))
        c, e = ops.ts_mx_quantize(x)
        assert torch.equal(codes, c) and torch.equal(scales, e)


def test_pack_more_records_than_one_launch_counts():
    n_out, n_in = (1 << 24) - 24, 4224                      # 33 records a row tile: 2^25 records end inside the matrix
    blocks = n_in // 32
    if torch.cuda.mem_get_info()[0] < (100 << 30):
        pytest.skip("100 GB of device memory are needed")
    codes = torch.zeros((n_out, 16 * blocks), dtype=torch.uint8, device="cuda")
    scales = torch.full((n_out, blocks), 127, dtype=torch.uint8, device="cuda")
    edge = (1 << 25) // 33 * 16
    spans = [(0, 48), (edge - 32, edge + 32), (n_out - 40, n_out)]
    gen = torch.Generator(device="cuda").manual_seed(5)
    for lo, hi in spans:
        codes[lo:hi] = torch.randint(0, 256, (hi - lo, 16 * blocks), dtype=torch.uint8, device="cuda", generator=gen)
        scales[lo:hi] = torch.randint(0, 255, (hi - lo, blocks), dtype=torch.uint8, device="cuda", generator=gen)
    packed = ops.ts_mx_pack(codes, scales, n_in).view(-1, 33, 1088)
    for lo, hi in spans:
        want = ops.ts_mx_pack(codes[lo:hi].contiguous(), scales[lo:hi].contiguous(), n_in).view(-1, 33, 1088)
        assert lo % 16 == 0 and torch.equal(packed[lo // 16:lo // 16 + want.shape[0]], want)
    del codes, scales, packed
    torch.cuda.empty_cache()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_quantize_more_values_than_one_launch_counts(dtype):
    cols = 40                                                  # two blocks a row: 2^27 rows a launch
    rows = (1 << 27) + 300
    if torch.cuda.mem_get_info()[0] < (80 << 30):
        pytest.skip("80 GB of device memory are needed")
    x = torch.zeros((rows, cols), dtype=dtype, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(2)
    spans = [(0, 40), ((1 << 27) - 30, (1 << 27) + 30), (rows - 40, rows)]
    for lo, hi in spans:
        x[lo:hi] = torch.randn((hi - lo, cols), generator=g, device="cuda")
    codes, scales = ops.ts_mx_quantize(x)
    back = ops.ts_mx_dequantize(codes, scales, cols, dtype)
    for lo, hi in spans:
        want, want_scales = definition(x[lo:hi])
        assert same(back[lo:hi], want) and torch.equal(scales[lo:hi].cpu(), want_scales)
    assert not bool(back[100:200].any()) and not bool(codes[100:200].any())
    del x, codes, scales, back
    torch.cuda.empty_cache()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_project_rows_and_outputs_beyond_32_bits(dtype):
    """As many rows as a call takes, inside wider ones: inputs and outputs of more than 2^32 elements."""
    rows, n_in, n_out, width = 1 << 19, 200, 40, 8448
    if torch.cuda.mem_get_info()[0] < (100 << 30):
        pytest.skip("100 GB of device memory are needed")
    packed, w = weights(n_out, n_in, 9)
    X = torch.zeros((rows, width), dtype=dtype, device="cuda")
    Y = torch.full((rows, width), 3.0, dtype=dtype, device="cuda")
    x, y = X[:, 8248:8448], Y[:, 8400:8440]
    x.copy_(torch.randn((rows, n_in), generator=torch.Generator(device="cuda").manual_seed(1), device="cuda"))
    ops.ts_mx_project(packed, n_out, x, y)
    for lo in (0, 1000, 254100, rows - 300):
        xs = x[lo:lo + 300].double().contiguous()
        want = xs @ w.t().contiguous()
        assert bool(((y[lo:lo + 300].double() - want).abs() <= bound(xs, w, want, dtype) * 1.01).all()), lo
        assert bool((Y[lo:lo + 300, :8400] == 3.0).all()) and bool((Y[lo:lo + 300, 8440:] == 3.0).all())
    del X, Y, x, y
    torch.cuda.empty_cache()


def test_weights_of_other_sizes_are_refused():
    """Also sizes that take the same bytes: whole records of 16 rows and 128 columns."""
    packed, w = weights(200, 1000, 4)
    x = torch.randn((3, 1024), device="cuda")
    for n_out, n_in in ((200, 1001), (200, 999), (200, 1024), (199, 1000), (208, 1000), (200, 900), (184, 1000)):
        with pytest.raises(ValueError, match="packed"):
            ops.ts_mx_project(packed, n_out, x[:, :n_in])
    check_project(packed, w, x[:, :1000], "its own size")
    codes, scales = ops.ts_mx_quantize(torch.randn((200, 1001), device="cuda"))
    ops.ts_mx_pack(codes, scales, 1001, packed)                # other weights in the same place: their size counts
    check_project(packed, ops.ts_mx_dequantize(codes, scales, 1001).double(), x[:, :1001], "packed over")
    with pytest.raises(ValueError, match="packed"):
        ops.ts_mx_project(packed, 200, x[:, :1000])
    check_project(packed.clone(), ops.ts_mx_dequantize(codes, scales, 1001).double(), x[:, :1001], "a copy")


def test_pointers_of_the_host_are_refused():
    lib = ops._load()
    x = torch.zeros((4, 64), device="cuda")
    h = torch.zeros((4, 64))
    c = torch.zeros((4, 32), dtype=torch.uint8, device="cuda")
    assert lib.ts_mx_quantize(h.data_ptr(), 0, 4, 64, 64, c.data_ptr(), c.data_ptr(), None) == B.TS_ERR_INVALID_ARG
    assert lib.ts_mx_quantize(x.data_ptr(), 0, 4, 64, 64, h.pin_memory().data_ptr(), c.data_ptr(), None) == B.TS_ERR_INVALID_ARG
    with pytest.raises(ValueError):
        ops.ts_mx_project(c.view(-1), 16, x)
    torch.cuda.synchronize()
