"""Every compiled variant of the product with 4-bit weights against 64-bit sums, by plans that the test chooses: the planner
picks a part of them for the sizes that other tests have.  Blocks of rows that are full, ragged, and a single row; columns
that end inside a tile and, for pairs of tiles, in an odd one; chunks of 128 inputs of every count up to several rounds, the
last one short; rows and outputs inside wider ones.

Tolerances.  The terms are exact, and n additions in fp32 in any order err by less than n 2^-24 times the sum of the magnitudes:
n = K (two planes: 2 K, fp32 rows: 3 K) + 16 for the groups of waves; then half a step of the output.  A term that is lost or meets
the wrong weight hides in that for fp32 rows and planes, so both also get rows of one value, all bits of it set: its products are
one sum of three (two) exact terms, off by at most a step of each of two additions, 2^-22."""
import ctypes as C
import math

import pytest
import torch

import hooks as H
from paper_2604_13519_amd import ops

pytestmark = pytest.mark.gpu

ALL = [(kind, out, shape, rt) for kind, out in ((H.MX_BF16, H.MX_ROWS), (H.MX_F32, H.MX_ROWS), (H.MX_PLANES, H.MX_ROWS), (H.MX_PLANES, H.MX_SWIGLU))
       for shape, rt in H.mx_variants(kind, out)]
PLANES_K, ANY_K = (128, 256, 384, 640, 1152), (20, 100, 128, 129, 300, 512, 1155)


def sizes(shape, rt):
    """Rows and columns of a workgroup."""
    return {H.DIRECT: (16, 16), H.DIRECT2: (16, 32), H.N32: (16 * rt, 32), H.N64: (16 * rt, 64), H.N128: (16 * rt, 128), H.N256: (64, 256)}[shape]


def weights(n_out, n_in, g):
    w = 0.05 * torch.randn((n_out, n_in), generator=g, device="cuda") * torch.exp2(torch.randint(-3, 3, (n_out, 1), generator=g, device="cuda").float())
    codes, scales = ops.ts_mx_quantize(w)
    return ops.ts_mx_pack(codes, scales, n_in), ops.ts_mx_dequantize(codes, scales, n_in).double()


def rows_of(kind, R, K, single, g):
    """The rows as 64-bit numbers, the sum of the terms' magnitudes, and the buffer, strides and offset that the launch gets."""
    x = torch.randn((R, K), generator=g, device="cuda")
    if single:                                             # one value a row, with every significant bit that the kind holds
        bits = 21 if kind == H.MX_PLANES else 24
        v = ((2.0 ** bits - 1) - 2 * torch.randint(0, 1 << (bits - 2), (R,), generator=g, device="cuda").double()) * 2.0 ** (1 - bits)
        at = torch.randint(0, K, (R,), generator=g, device="cuda")
        x = torch.zeros((R, K), device="cuda")
        x[torch.arange(R, device="cuda"), at] = v.float()
    if kind == H.MX_PLANES:
        hi = x.half()
        lo = (x - hi.float()).half()
        X = torch.full((2, R + 3, K + 64), math.nan, dtype=torch.float16, device="cuda")
        X[0, :R, :K], X[1, :R, :K] = hi, lo
        return hi.double() + lo.double(), hi.double().abs() + lo.double().abs(), X, K + 64, (R + 3) * (K + 64), 0
    dt = torch.bfloat16 if kind == H.MX_BF16 else torch.float32
    x = x.to(dt)
    off = 3                                                # rows at any element's place, NaN around them
    X = torch.full((R + 1, K + off + 5), math.nan, dtype=dt, device="cuda")
    X[:R, off:off + K] = x
    return x.double(), x.double().abs(), X, K + off + 5, 0, off


def check(kind, out, shape, rt, R, N, K, splits=1, single=False, seed=0):
    print("product: kind %d to %d, shape %d rt %d: %d rows x %d columns, K %d in %d%s" % (kind, out, shape, rt, R, N, K, splits, ", single values" if single else ""), flush=True)
    g = torch.Generator(device="cuda").manual_seed(seed)
    packed, w = weights(N, K, g)
    x, mag, X, xs, xp, off = rows_of(kind, R, K, single, g)
    want = x @ w.t().contiguous()
    if single:
        err = 2.0 ** -22 * want.abs()
    else:
        err = ({H.MX_BF16: 1, H.MX_F32: 3, H.MX_PLANES: 2}[kind] * K + 16) * 2.0 ** -24 * (mag @ w.abs().t().contiguous())
    sat = torch.zeros(1, dtype=torch.int64, device="cuda")
    y_off, yp = 0, 0
    if out == H.MX_SWIGLU:
        Y = torch.full((2, R + 2, N // 2 + 64), 3.0, dtype=torch.float16, device="cuda")
        ys, yp = N // 2 + 64, (R + 2) * (N // 2 + 64)
    elif kind == H.MX_PLANES:                              # partial sums follow each other
        Y = torch.full((splits + 1, R, N), 3.0, device="cuda")
        ys = N
    else:
        y_off, ys = 2, N + 7
        Y = torch.full((R + 2, ys), 3.0, dtype=X.dtype, device="cuda")
    torch.cuda.synchronize()
    rc = H.lib().hook_mx_project(C.c_void_p(packed.data_ptr()), C.c_void_p(X.data_ptr() + off * X.element_size()), C.c_long(xs), C.c_long(xp),
                                 C.c_void_p(Y.data_ptr() + y_off * Y.element_size()), C.c_long(ys), C.c_long(yp), int(Y.dtype == torch.float32),
                                 C.c_void_p(sat.data_ptr()), kind, out, R, N, K, shape, rt, splits)
    assert rc == 0, "launch failed with %d" % rc
    assert int(sat) == 0
    if out == H.MX_SWIGLU:                                 # tiles of 16 alternate: gate and up of the same features
        f = lambda t: t.view(R, -1, 2, 16).permute(2, 0, 1, 3).reshape(2, R, N // 2)  # noqa: E731
        (gv, uv), (ge, ue) = f(want), f(err)
        ref = gv * torch.sigmoid(gv) * uv
        tol = 1.1 * uv.abs() * ge + (gv * torch.sigmoid(gv)).abs() * ue + 1.2 * ge * ue + 2.0 ** -20 * ref.abs() + 2.0 ** -24      # d silu <= 1.1; expf, division, hi + lo
        got = Y[:, :R, :N // 2].double().sum(0)
        rest = (Y[:, R:] == 3.0).all() and (Y[:, :, N // 2:] == 3.0).all()
    elif kind == H.MX_PLANES:
        ref, tol, got = want, err, Y[:splits].double().sum(0)
        rest = (Y[splits] == 3.0).all()
    else:
        ref, tol, got = want, err + torch.finfo(Y.dtype).eps / 2 * want.abs(), Y[:R, y_off:y_off + N].double()
        rest = (Y[R:] == 3.0).all() and (Y[:, :y_off] == 3.0).all() and (Y[:, y_off + N:] == 3.0).all()
    bad = (got - ref).abs() > tol
    assert not bool(bad.any()), "%d outputs, worst %.3g of the tolerance" % (int(bad.sum()), float(((got - ref).abs() / tol.clamp(min=1e-300)).max()))
    assert bool(rest), "written beside the outputs"


@pytest.mark.parametrize("kind,out,shape,rt", ALL)
def test_every_variant(kind, out, shape, rt):
    mt, nt = sizes(shape, rt)
    for R in (1, mt - 1, mt, 2 * mt + 3):
        for i, K in enumerate(PLANES_K if kind == H.MX_PLANES else ANY_K):
            N = nt + 96 if out == H.MX_SWIGLU else nt + (37, 53)[i % 2]
            check(kind, out, shape, rt, R, N, K, seed=K + R)
    if out == H.MX_ROWS and kind != H.MX_BF16:
        for K in (128, 1152) if kind == H.MX_PLANES else (129, 1155):
            for seed in range(3):
                check(kind, out, shape, rt, 2 * mt + 3, nt + 37, K, single=True, seed=seed)
    if out == H.MX_ROWS and kind == H.MX_PLANES and shape not in (H.DIRECT, H.DIRECT2):      # which take all of K
        for splits, K in ((2, 256), (2, 384), (3, 1152), (5, 1152)):
            check(kind, out, shape, rt, mt + 5, nt + 37, K, splits=splits, seed=splits)


@pytest.mark.parametrize("dtype,rows,n_out,plan", [
    (torch.bfloat16, 20, 28672, (H.N128, 2)), (torch.bfloat16, 33, 28672, (H.N128, 3)), (torch.bfloat16, 64, 28672, (H.N128, 4)), (torch.bfloat16, 65, 28672, (H.N128, 5)),
    (torch.bfloat16, 200, 14336, (H.N256, 0)), (torch.bfloat16, 40, 14336, (H.N64, 3)), (torch.bfloat16, 161, 5408, (H.N64, 4)), (torch.bfloat16, 70, 14336, (H.N64, 5)),
    (torch.float32, 20, 28672, (H.N128, 2)), (torch.float32, 33, 28672, (H.N128, 3)), (torch.float32, 64, 28672, (H.N128, 4)), (torch.float32, 65, 28672, (H.N128, 5)),
    (torch.float32, 600, 14336, (H.N256, 0)), (torch.float32, 161, 5408, (H.N64, 4)), (torch.float32, 20, 14336, (H.N64, 2))])
def test_calls_that_take_the_wide_variants(dtype, rows, n_out, plan):
    """Through ts_mx_project, at sizes for which it takes them."""
    for n_in, off in ((4096, 0), (4101, 1)):
        assert H.mx_plan(H.MX_BF16 if dtype == torch.bfloat16 else H.MX_F32, H.MX_ROWS, rows, n_out, n_in) == plan
        print("call", dtype, rows, n_in, n_out, flush=True)
        g = torch.Generator(device="cuda").manual_seed(rows)
        codes = torch.randint(0, 256, (n_out, 16 * -(-n_in // 32)), dtype=torch.uint8, device="cuda", generator=g)
        scales = torch.randint(110, 120, (n_out, -(-n_in // 32)), dtype=torch.uint8, device="cuda", generator=g)
        X = torch.full((rows, n_in + off), math.nan, dtype=dtype, device="cuda")
        X[:, off:] = torch.randn((rows, n_in), generator=g, device="cuda")
        Y = torch.full((rows, n_out + off), 3.0, dtype=dtype, device="cuda")
        ops.ts_mx_project(ops.ts_mx_pack(codes, scales, n_in), n_out, X[:, off:], Y[:, off:])
        w, x, y = ops.ts_mx_dequantize(codes, scales, n_in).double(), X[:, off:].double(), Y[:, off:].double()
        want, mag = x @ w.t().contiguous(), x.abs() @ w.abs().t().contiguous()
        tol = ((n_in if dtype == torch.bfloat16 else 3 * n_in) + 16) * 2.0 ** -24 * mag + torch.finfo(dtype).eps / 2 * want.abs()
        assert bool(((y - want).abs() <= tol).all()) and bool((Y[:, :off] == 3.0).all())
        if dtype == torch.float32:                         # what a term is worth shows in rows of one value
            X = torch.zeros((rows, n_in), device="cuda")
            at = torch.randint(0, n_in, (rows,), device="cuda", generator=g)
            X[torch.arange(rows, device="cuda"), at] = 1.9999999
            want = X.max().double() * w[:, at].t()
            assert bool(((ops.ts_mx_project(ops.ts_mx_pack(codes, scales, n_in), n_out, X).double() - want).abs() <= 2.0 ** -22 * want.abs()).all())
