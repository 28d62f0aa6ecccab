"""Whether a cache's keys and values share memory (csrc/cache_layout.h): the rule against every value of both.  Host only."""
import itertools
import random
import subprocess

import pytest

from paper_2601_17261_amd import build as B

PROGRAM = r"""
#include <cstdio>
#include "cache_layout.h"
using namespace agzo;
int main() {
    long long dim, between, at[2][6];
    while (scanf("%lld %lld", &dim, &between) == 2) {
        for (auto& t : at)
            for (int i = 0; i < 6; ++i) if (scanf("%lld", t + i) != 1) return 1;
        CacheLayout of[2];
        int fault = 0;
        for (int i = 0; i < 2; ++i) {
            const long long* t = at[i];
            const int64_t axes[3][2] = {{t[0], t[1]}, {t[2], t[3]}, {t[4], t[5]}};
            int64_t bad = 0;
            fault |= (int)cache_layout(dim, axes, of[i], bad) << (2 * i);
        }
        printf("%d %d\n", fault, fault ? -1 : (int)layouts_apart(of[0], of[1], between));
    }
}
"""


@pytest.fixture(scope="module")
def ask(tmp_path_factory):
    d = tmp_path_factory.mktemp("layout")
    src, exe = d / "layout.cpp", d / "layout"
    src.write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-Wall", "-I", B.CSRC, str(src), "-o", str(exe)], check=True)

    def run(cases):
        """cases: (dim, between, axes of k, axes of v), axes: ((stride, size) of page, row, head) -> [(fault, apart)]"""
        text = "\n".join(" ".join(map(str, (dim, between) + tuple(itertools.chain(*k)) + tuple(itertools.chain(*v)))) for dim, between, k, v in cases)
        out = subprocess.run([str(exe)], input=text, capture_output=True, text=True, check=True).stdout.split()
        return list(zip(map(int, out[::2]), map(int, out[1::2])))
    return run


def values(dim, axes, at=0):
    """of eight each, as strides are"""
    return [at // 8 + sum(i * s for i, s in zip(index, [a[0] // 8 for a in axes])) + j for index in itertools.product(*(range(a[1]) for a in axes)) for j in range(dim // 8)]


def test_rows_of_one_page_that_are_rows_of_the_next(ask):
    """64 values, rows 128 apart, pages of two rows 192 apart: values lie between the keys of a page, its second row where the next page's first key is"""
    axes = ((192, 4), (128, 2), (64, 1))
    assert len(set(values(64, axes)) & set(values(64, axes, 64))) * 8 == 192
    assert ask([(64, 64, axes, axes)]) == [(0, 0)]


def test_layouts_that_programs_have(ask):
    page, kv, dim, n = 16, 2, 64, 5
    heads_in_tokens = ((page * kv * dim, n), (kv * dim, page), (dim, kv))
    cases = [(dim, n * page * kv * dim, heads_in_tokens, heads_in_tokens),                                          # one behind the other
             (dim, page * kv * dim, *[((2 * page * kv * dim, n), (kv * dim, page), (dim, kv))] * 2),              # page by page
             (dim, page * kv * dim, *[((2 * page * kv * dim, n), (dim, page), (page * dim, kv))] * 2),            # ... with tokens inside heads
             (dim, kv * dim, *[((page * (2 * kv * dim + 16), n), (2 * kv * dim + 16, page), (dim, kv))] * 2),      # token by token, with room between
             (dim, dim, *[((2 * page * kv * dim, n), (2 * kv * dim, page), (2 * dim, kv))] * 2),                   # head by head
             (dim, dim, *[((2 * page * dim, n), (2 * dim, page), (dim, 1))] * 2),                                 # of one key head
             (dim, page * dim, *[((2 * page * kv * dim, n), (dim, page), (2 * page * dim, kv))] * 2),             # a head's tokens, keys then values
             (dim, dim, *[((0, 1), (2 * dim, page), (dim, 1))] * 2)]
    assert ask(cases) == [(0, 1)] * len(cases)
    assert ask([(d, 0, k, v) for d, _, k, v in cases]) == [(0, 0)] * len(cases)


def test_against_every_value(ask):
    """never apart where a value is of both; and apart wherever blocks of one lie in the other's gaps, which is how caches of both in one tensor are laid out"""
    rng, cases = random.Random(1), []
    for _ in range(6000):
        dim = rng.choice([8, 16, 24])
        sizes, strides, extent = [rng.randint(1, 4) for _ in range(3)], [0, 0, 0], dim
        for i in rng.sample(range(3), 3):
            strides[i] = extent + 8 * rng.choice([0, 0, 1, 2, 3, extent // 8, extent // 8 + 1])
            extent += (sizes[i] - 1) * strides[i]
        axes = tuple(zip(strides, sizes))
        cases.append((dim, 8 * rng.randint(0, extent // 8 + 2), axes, axes))
    kinds = set()
    for case, (fault, apart) in zip(cases, ask(cases)):
        dim, between, axes, _ = case
        assert fault == 0, case
        k = values(dim, axes)
        assert len(set(k)) == len(k)
        share = bool(set(k) & set(values(dim, axes, between)))
        assert not (apart and share), case
        kinds.add((share, apart))
    assert kinds == {(True, 0), (False, 1), (False, 0)}


def test_refused_layouts(ask):
    dim = 64
    good = ((256, 4), (128, 2), (64, 2))
    for axes, fault in ((good, 0), (((255, 4), (128, 2), (64, 2)), 1), (((256, 4), (128, 2), (56, 2)), 1), (((2 ** 40, 4), (128, 2), (64, 2)), 1), (((248, 4), (128, 2), (64, 2)), 2),
                        (((256, 4), (64, 2), (64, 2)), 2), (((2 ** 39, 2 ** 31), (128, 2), (64, 2)), 3), (((0, 1), (0, 1), (-7, 1)), 0), (((256, 0), (128, 2), (64, 2)), 0)):
        (got, _), = ask([(dim, 0, axes, good)])
        assert got == fault, axes
