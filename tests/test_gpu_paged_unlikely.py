"""Attention over pages: values that are not finite and that a row sees, at places whose probability is below fp32's smallest (e^-104), are in its result as the formula has them, wherever a share of the
keys ends."""
import math
import random

import pytest

import paged_reference as ref
from test_gpu_cache import Pages
from test_gpu_paged_attention import check, queries, trees

pytestmark = pytest.mark.gpu


def planted(c, have, page, bad, seed, each=3):
    rng = random.Random(seed)
    for s, n in enumerate(have):
        for place in rng.sample(range(n), min(each, n)):
            # (one value of one key head: the others' columns stay finite)
            c.v[ref.slot(c.table, page, c.k.shape[0], s, place)][rng.randrange(c.v.shape[2]), rng.randrange(c.v.shape[3])] = bad
    return c


@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("dim,page", [(64, 16), (128, 16), (128, 5)])
@pytest.mark.parametrize("kind", ["single", "many heads", "tree", "chunk", "long chunk"])
def test_values_of_unlikely_places(bad, dim, page, kind):
    heads, kv = (40, 2) if kind == "many heads" else (8, 2)
    have = [9000, 33, 2500, 700]
    new = {"single": [1] * 4, "many heads": [1] * 4, "tree": [40, 3, 17, 64], "chunk": [20, 5, 60, 1], "long chunk": [600, 33, 300, 1]}[kind]
    more = 200 if kind == "long chunk" else 0
    for seed in (1, 2):
        c = planted(Pages(seed, have, page, kv, dim, more=more), have, page, bad, seed)
        # (scores of some 60 either way: differences of more than 104 often, and none of 745, where 64 bits end)
        q = queries(seed, sum(new), heads, dim, 60.0)
        out, _ = check(c, q, new, have, dim, bits=trees(seed, new) if kind == "tree" else None)
        assert out.isnan().any() if math.isnan(bad) else out.isinf().any()
