"""The plan of the 8-bit products (CPU: its source compiled by itself): every form of a kernel that it picks for any call is one that a GPU test
runs, so that a plan that is fitted anew cannot leave one untested unseen."""
import math
import random

import pytest

from tests import fp8_plan
from tests.test_gpu_fp8 import LARGE, RUNS, SHAPES
from tests.test_gpu_fp8_forms import CASES

if not fp8_plan.available():
    pytest.skip("no C++ compiler", allow_module_level=True)


def covered():
    """The forms that the GPU tests' calls run."""
    calls = [(M, N, K, e, 16, s) for M, N, K in SHAPES for e in (0, 1) for s in (1, 2)]
    calls += [(M, N, K, 2, b, s) for M, N, K in SHAPES for b, s in ((8, 0), (8, 1), (16, 0), (16, 2))]
    calls += [(M, N, K, e, b, s) for M, N, K in LARGE for e, b in ((1, 16), (2, 16), (2, 8)) for s in (1, 2)]
    calls += [(M, N, K, e, b, s) for M, N, K in RUNS for e, b in ((0, 16), (1, 16), (2, 16), (2, 8)) for s in (1, 2)]
    out = set()
    for M, N, K, e, b, s in calls + CASES:
        out |= fp8_plan.forms(M, N + -N % 32 if b == 8 else N + N % 2 if e == 2 else N, K, e, b, s)
    return out


@pytest.mark.parametrize("seed", [1, 2])
def test_every_form_that_the_plan_picks_is_tested(seed):
    have, rng, missing = covered(), random.Random(seed), {}
    log = lambda lo, hi: int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))   # noqa: E731
    for _ in range(25_000):
        M, N, K = log(1, 45_000), log(16, 30_000), 16 * log(1, 1024)
        if rng.random() < 0.5:
            N += -N % 8
        for e, b in ((0, 16), (1, 16), (2, 16), (2, 8)):
            n = N + -N % 32 if b == 8 else N + N % 2 if e == 2 else N
            for s in (1, 2):
                for f in fp8_plan.forms(M, n, K, e, b, s) - have:
                    missing.setdefault(f, (M, n, K, e, b, s))
    assert not missing, missing


def test_every_tile_is_picked_and_taken_in_turn_where_it_can_be():
    have = covered()
    for t, (_, _, _, _, wide, run) in enumerate(fp8_plan.tiles()):
        assert any(f[0] == t for f in have)
        if run:
            for name in ("bias", "swiglu"):
                assert (t, "in turn", name, "several tiles") in have


def test_plans_by_hand():
    """Few rows take no tile, rows are dealt out whole, parts of K only where there are blocks enough, nothing past 2^32 threads."""
    tiles = fp8_plan.tiles()
    assert fp8_plan.launches(1, 4608, 3584, False, False) == [(-1, 1, 1, 0)]
    rng = random.Random(3)
    for _ in range(3000):
        M, N, K = int(2 ** rng.uniform(0, 17)), int(2 ** rng.uniform(4, 17)), 16 * int(2 ** rng.uniform(0, 12))
        for eight in (False, True):
            for wide in (False, True):
                runs = fp8_plan.launches(M, N, K, eight, wide)
                assert 1 <= len(runs) <= 2 and sum(r for _, r, _, _ in runs) == M
                for t, rows, splits, part in runs:
                    assert rows >= 1 and (t >= 0 or rows <= 16) and (splits == 1 or (part and 2 * splits <= -(-K // 128)))
                    if t >= 0:
                        assert bool(tiles[t][4]) == wide and (part or not eight or tiles[t][1] == 256)
                if len(runs) == 2:
                    assert not runs[0][3] and runs[0][2] == 1 and runs[0][1] % tiles[runs[0][0]][0] == 0
    assert fp8_plan.launches(1 << 22, 1 << 22, 256, False, False) == []
