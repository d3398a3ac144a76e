"""The launch rules of the packed products, on the host: every launch stays within what a grid and a
compute unit's LDS hold, and all row groups of a call are launched."""
import random

import pytest

from tests.matvec_cases import VARIANTS, instances, sizes
from tests.matvec_plan import Rules

BLOCK = {"nvfp4": 16, "mxfp4": 32, "q4k": 256}
LDS = 160 * 1024


@pytest.fixture(scope="module")
def rules(tmp_path_factory):
    return Rules(str(tmp_path_factory.mktemp("plan")))


def _launch_fits(p, fmt):
    assert 1 <= p.waves <= 8 and p.tiles_each in (1, 2) and 1 <= p.xmax <= 16
    assert p.xrows == p.xmax or (p.xrows == 8 and p.rows == "twice")
    assert p.per_launch >= 1
    assert p.tiles * min(p.per_launch, p.items) * 64 * p.waves < 1 << 32
    codes = 5120 if fmt == "q4k" else 4096
    lds = p.waves * (p.tiles_each * codes + p.xrows * 1024)
    assert p.waves * p.tiles_each * 1024 <= lds <= LDS             # the partial sums reuse the region


def test_launches_of_any_size(rules):
    rng = random.Random(0)
    for _ in range(20000):
        fmt = rng.choice(list(BLOCK))
        grouped = rng.random() < 0.6
        E = rng.choice([1, 2, 8, 60, 128, 1024]) if grouped else 1
        N = int(2 ** rng.uniform(0, 30))
        K = int(2 ** rng.uniform(0, 30)) // BLOCK[fmt] * BLOCK[fmt]
        R = max(1, int(2 ** rng.uniform(0, 30))) if grouped else rng.randint(1, 64)
        p = rules.plan(fmt, grouped, E, N, K, R)
        _launch_fits(p, fmt)
        assert p.tiles * 16 * p.tiles_each >= N
        assert grouped or p.items * p.xmax >= R
    for N in (1 << 26, (1 << 29) + 1, (1 << 30) - 17, (1 << 30) - 1):
        for K in (0, 256, 4096, 1 << 20):
            for M in (1, 64):
                _launch_fits(rules.plan("mxfp4", False, 1, N, K, M), "mxfp4")


def test_row_groups_of_experts_are_enough(rules):
    rng = random.Random(1)
    for _ in range(2000):
        E = rng.choice([1, 3, 16, 128])
        counts = [rng.choice([0, 0, 1, 3, 8, 9, 16, 17, 200]) for _ in range(E)]
        R = sum(counts) + rng.randint(0, 3)
        if R == 0:
            continue
        p = rules.plan(rng.choice(list(BLOCK)), True, E, 512, 512, R)
        assert p.items >= sum((c + p.xmax - 1) // p.xmax for c in counts)


def test_more_row_groups_than_one_launch_holds(rules):
    """9 million rows of 4096 columns, and the two calls that the device runs (test_gpu_matvec)."""
    for fmt, grouped, E, N, K, R in (("nvfp4", True, 128, 4096, 4096, 9000000), ("mxfp4", True, 1, 1 << 20, 32, 33000),
                                     ("mxfp4", False, 1, (1 << 29) + 40, 32, 64)):
        p = rules.plan(fmt, grouped, E, N, K, R)
        _launch_fits(p, fmt)
        assert p.per_launch < p.items


def test_device_cases_reach_every_instance(rules):
    seen = set()
    for fmt, instance, rows, N, K in VARIANTS:
        grouped, E, R = sizes(rows)
        assert tuple(rules.plan(fmt, grouped, E, N, K, R)[:3]) == instance, (fmt, rows, N, K)
        seen.add((fmt, instance))
    assert seen == instances()
