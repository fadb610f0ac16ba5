"""The way of a gradient of a lookup, without a device: the rule as the tests know it against the library's workspaces."""
import random

import pytest

import paper_2307_12059_amd as kgc
from tests.embed_plan import plan


def test_the_tests_rule_is_the_librarys():
    rng = random.Random(5)
    size = lambda hi: int(round(hi ** rng.random()))
    edges = [0, 1, 3500, 3501, 8192, 8193, 16384, 16385, 49152, 49153, 65536, 65537, 131072, 131073, 262144, 262145, 524415, 524416, 4194305]
    for _ in range(20000):
        n = rng.choice(edges) if rng.random() < 0.5 else size(5_000_000)
        N = rng.choice([1, 255, 256, 257, 511, 512, 2048, 245760, 245761, 262144, 262145]) if rng.random() < 0.5 else size(5_000_000)
        d = rng.choice([1, 3, 4, 64, 65, 128, 129, 256, 257, 512, 513, 960]) if rng.random() < 0.5 else size(960)
        assert kgc.kgc_lookup_grad_bytes(n, N, d) == plan(n, N, d).bytes, (n, N, d)


@pytest.mark.parametrize("n,N,d,form", [(3500, 9000, 8, "few"), (3501, 9000, 8, "once"), (8192, 2048, 8, "few"), (8192, 2049, 8, "once"), (8193, 4, 8, "table"),
                                        (16384, 511, 100, "once"), (16385, 511, 100, "sort"), (16385, 512, 100, "once"),
                                        (49152, 245760, 2, "once"), (49152, 245761, 2, "sort"), (48128, 262144, 2, "sort"),
                                        (47104, 262144, 2, "once"), (47104, 262145, 2, "sort"), (49153, 5000, 8, "sort")])
def test_borders_between_the_ways(n, N, d, form):
    assert plan(n, N, d).form == form
