"""Every division of a launch over caches in 4 and 8 bits that a call can get is run by a
GPU test: shapes drawn over the whole range, of up to 2^24 rows, ask the planner for theirs.
A change of the planner that brings a division in which no test runs fails here; a shape of
it then belongs into quant_divisions.CASES."""
import math
import random
import shutil

import pytest

from tests import quant_divisions as qd
from tests import test_quant_plans_gpu as plans


@pytest.fixture(scope="module")
def planner(tmp_path_factory):
    if not shutil.which("g++"):
        pytest.skip("no host compiler")
    return qd.Planner(str(tmp_path_factory.mktemp("plan")))


def of(planner, shape, kw):
    return qd.divisions(planner(*shape, **kw), shape[5], "k_max" in kw)


def run_by_tests(planner):
    """Of the shapes of test_quant_plans_gpu.py (three calls each), and of CASES."""
    shapes = [(s, G) for s in plans.SHAPES for G in (2, 6, 16)]
    shapes += [(s, G) for s in [(1, 1, 200, 3), (1, 16, 700, 8), (4, 64, 96, 4), (8, 3, 8192, 2)]
               for G in (1, 17, 20, 48)]
    have = set()
    for (n, B, L, H_kv), G in shapes:
        for bits in (4, 8):
            for kw in ({}, dict(window=max(1, L // 2), n_sink=33), dict(k_max=L)):
                have |= of(planner, (n, B, L + 5, H_kv, G, bits), kw)
    for case in qd.CASES:
        have |= of(planner, *qd.arguments(case))
    return have


def drawn(rng):
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    while True:
        n, B, L = log(1, 64), log(1, 100), log(1, 131072)
        H_kv, bits = rng.choice([1, 2, 3, 4, 6, 8, 16]), rng.choice([4, 8])
        G = rng.choice([1, 2, 3, 4, 5, 6, 7, 8, 12, 16, 17, 20, 32, 48])
        kw = rng.choice([{}, dict(window=log(1, L), n_sink=rng.choice([0, 4, 64])),
                         dict(k_max=log(1, L))])
        if n * B * L * H_kv <= 1 << 24:
            return (n, B, L, H_kv, G, bits), kw


def test_every_division_is_run(planner):
    have, rng, missing = run_by_tests(planner), random.Random(20), {}
    for _ in range(60000):
        shape, kw = drawn(rng)
        for d in of(planner, shape, kw) - have:
            missing.setdefault(d, (shape, kw))
    assert not missing, missing


def test_the_divisions_that_the_tests_are_named_for(planner):
    """4 and 8 wavefronts, 1 to 8 units side by side, in parts and not, dealt or not, one KV
    head or two, 4, 8 and 16 columns: all occur among those that are run, for both kinds of
    calls."""
    have = run_by_tests(planner)
    for selected in (False, True):
        divided = [d[1:] for d in have if d[0] == "divided" and d[2] == selected]
        assert {(d[0], d[2], d[3]) for d in divided} == {
            (4, 1, 4), (4, 1, 8), (4, 2, 4), (4, 2, 8), (8, 1, 4), (8, 1, 8)}
        assert {d[4] for d in divided} == {0, 1, 2, 3}
        assert {d[5:] for d in divided} == {(False, False), (True, False), (True, True)}
        assert {d[5] for d in have if d[0] == "columns" and d[2] == selected} == {4, 8, 16}
