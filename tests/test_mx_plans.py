"""Planner of the products with 4-bit weights: what it picks is a compiled variant (all of which are run against 64-bit sums on a
GPU), and a model's sums fit where they go."""
import random

import hooks as H

SIZES = [(r, n, k) for r in (1, 5, 16, 17, 33, 48, 65, 80, 81, 129, 161, 260, 520, 2048) for n in (1, 31, 96, 512, 1024, 4096, 5408, 6144, 14336, 28672, 128256)
         for k in (32, 128, 1000, 4096, 14336)]


def drawn(n):
    rng = random.Random(3)
    return [(int(2 ** rng.uniform(0, 19)), int(2 ** rng.uniform(0, 20)), int(2 ** rng.uniform(0, 16))) for _ in range(n)]


def test_picks_are_compiled_variants():
    for kind, out in ((H.MX_BF16, H.MX_ROWS), (H.MX_F32, H.MX_ROWS), (H.MX_PLANES, H.MX_ROWS), (H.MX_PLANES, H.MX_SWIGLU)):
        compiled, picked = set(H.mx_variants(kind, out)), set()
        # the last three: many rows and few columns, where alone bf16 blocks of 48 and more rows by 32 columns are taken
        for r, n, k in SIZES + drawn(3000) + [(22904, 1, 890), (143145, 1, 128), (12924, 14, 46383), (20971, 63, 5), (162352, 34, 106504)]:
            if out == H.MX_SWIGLU:
                n = -(-n // 32) * 32
            picked.add(H.mx_plan(kind, out, r, n, k))
        assert picked == compiled, (kind, out, picked ^ compiled)


def test_sums_of_a_model_fit():
    compiled = set(H.mx_variants(H.MX_PLANES, H.MX_ROWS))
    rng = random.Random(4)
    for r, n, k in SIZES + drawn(3000):
        k = -(-k // 128) * 128
        room = int(r * n * rng.choice((1, 1.5, 2, 7, 16, 40)))
        shape, rt, splits = H.mx_plan_model(r, n, k, room)
        assert (shape, rt) in compiled and 1 <= splits <= 16 and splits * r * n <= room
        assert splits == 1 or shape not in (H.DIRECT, H.DIRECT2)
        assert splits <= k // 128 and (k // 128 + splits - 1) // splits * (splits - 1) < k // 128      # no split is empty
