"""Which kernel takes a projection, without a GPU: every form that products of the supported sizes are given to is
on a list of the GPU tests, and every plan covers its product and fits the workspace. A change of the modelled times
that leaves a form without a test fails here."""
import math
import random

import pytest

from tests import test_gpu_linear as lists
from tests.linear_plans import FORMS, TILE, TILES, Plan

WORKSPACE, SYNC = 64 << 20, 4096  # bytes of slices' sums, tiles of a product in slices


def draws(n, seed):
    """Sizes spread over their logarithm, some with whole steps of K, and row paddings."""
    rng = random.Random(seed)
    size = lambda hi: min(hi, int(math.exp(rng.uniform(0.0, math.log(hi + 1)))))
    out = []
    while len(out) < n:
        M, K, N = size(8192), size(16384), size(32768)
        if rng.random() < 0.3:
            K = -(-K // 64) * 64
        if M * K * N < 2 ** 41:
            out.append((M, K, N, rng.choice([0, 8, 16, 64, "lines"])))
    return out


@pytest.mark.parametrize("gated", [False, True])
def test_every_form_is_on_a_list(gated):
    tested = {Plan(M, K, N, gated, pad, shift).form() for M, K, N in lists.SHAPES
              for pad, shift in ((8, 0), ("lines", 0), ("lines", 40), (16, 8))}
    tested |= {Plan(M, K, N, gated, pad).form() for M, K, N in lists.COLD for pad in (0, 8, 24, 48)}
    tested |= {Plan(M, K, N, gated, pad).form() for M, K, N, pad in FORMS}
    missing = {}
    for c in draws(60000, 1):
        form = Plan(*c[:3], gated, c[3]).form()
        if form not in tested:
            missing.setdefault(form, c)
    assert not missing, missing


@pytest.mark.parametrize("gated", [False, True])
def test_every_epilogue_is_on_a_list(gated):
    """With activation, bias and residual: each kernel, whole and in slices."""
    tested = {Plan(M, min(K, 4200), N, gated).epilogue() for M, K, N in lists.LARGE + [(1, 200, 140), (40, 200, 140)]}
    tested |= {Plan(M, K, N, gated, pad).epilogue() for M, K, N, pad in FORMS}
    missing = {}
    for c in draws(20000, 2):
        e = Plan(*c[:3], gated, c[3]).epilogue()
        if e not in tested:
            missing.setdefault(e, c)
    assert not missing, missing
    assert len(tested) == 2 * TILE + 1  # the tile kernel takes no slices


@pytest.mark.parametrize("gated", [False, True])
def test_plans_cover_their_products(gated):
    """Every slice has steps, together they are all of K; the columns are all features; sums of slices fit."""
    extremes = [(1, 1, 1, 8), (1 << 20, 64, 4, 8), (1, (1 << 22) - 8, 8, 0), (16, 1 << 22, 1, "lines"), (17, 1, 1 << 24, 8),
                (1, 5, 1 << 25, 8), (1 << 20, 1, 1, 8), (300, 1 << 22, 300, 0)]
    for M, K, N, pad in draws(20000, 3) + extremes:
        p = Plan(M, K, N, gated, pad)
        at, all_steps, rows = (M, K, N, pad), -(-K // 64), TILES[p.kernel][0]
        assert (p.slices - 1) * p.steps < all_steps <= p.slices * p.steps, at
        weights = TILES[p.kernel][1]  # rows of them in a tile
        if p.kernel == TILE:
            features = (p.wide * 256 + p.columns * 128) // (2 if gated else 1)
            assert p.slices == 1 and not p.lines and features >= N > features - (128 if p.columns else 256), at
            continue
        assert p.wide == 0
        if p.kernel == 0:
            of, weights = 16, 32 if gated else 16
            assert M <= 16 and not p.lines
        else:
            of = weights // 2 if gated else weights
        assert p.columns * of >= N > (p.columns - 1) * of, at
        if p.slices > 1:
            tiles = -(-M // rows) * p.columns
            assert tiles <= SYNC and tiles * p.slices * rows * weights * 4 <= WORKSPACE, at
