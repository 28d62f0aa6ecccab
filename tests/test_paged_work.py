"""What attention over a cache in pages reckons its row tiles' work as (csrc/paged_work.h), up to the longest sequences and the most rows that the call takes: whole numbers of 32 bits.  Host only."""
import itertools
import random
import subprocess

import pytest

from paper_2601_17261_amd import build as B

MOST = 2 ** 31 - 1 - 1024       # keys of a sequence, rows of a key head
PROGRAM = r"""
#define __host__
#define __device__
#define __forceinline__ inline
#include <cstdio>
#include "paged_work.h"
int main() {
    int nq, nk, G, rows, tree, start;
    while (scanf("%d %d %d %d %d %d", &nq, &nk, &G, &rows, &tree, &start) == 6) {
        const agzo::PgWork w = agzo::pg_work(nq, nk, G, rows, tree != 0, start);
        const int last = w.tiles > 0 ? w.tiles - 1 : 0;
        printf("%d %d %d %d %d %lld\n", w.tiles, w.first, w.step, agzo::pg_of(w, 0), agzo::pg_of(w, last), (long long)agzo::pg_before(w, w.tiles));
    }
}
"""


@pytest.fixture(scope="module")
def ask(tmp_path_factory):
    d = tmp_path_factory.mktemp("work")
    src, exe = d / "work.cpp", d / "work"
    src.write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-Wall", "-fwrapv", "-I", B.CSRC, str(src), "-o", str(exe)], check=True)

    def run(cases):
        out = subprocess.run([str(exe)], input="\n".join(" ".join(map(str, c)) for c in cases), capture_output=True, text=True, check=True).stdout.split()
        return [tuple(map(int, out[i:i + 6])) for i in range(0, len(out), 6)]
    return run


def check(ask, cases):
    got = ask(cases)
    assert len(got) == len(cases)
    for case, (tiles, first, step, one, last, all_) in zip(cases, got):
        nq, nk, G, rows, tree, start = case
        assert tiles == -(-nq * G // rows), case
        assert start <= first < 2 ** 31 and step >= 0, case
        if tiles == 0:
            continue
        assert one == first and last == first + step * (tiles - 1) < 2 ** 31, case
        assert all_ == first * tiles + step * (tiles * (tiles - 1) // 2) < 2 ** 63, case
        # about the keys that a tile's rows see: a step is that of the queries that it goes on by, rounded
        assert step == 0 if tree else abs(step - rows / G) < 1, case
        for t in (0, tiles - 1):
            seen = nk if tree else max(nk - nq + min(((t + 1) * rows - 1) // G, nq - 1) + 1, 0)
            assert abs(first + step * t - start - seen) <= t + rows + max(nq - nk, 0), case


def test_ordinary_lengths(ask):
    rng, cases = random.Random(1), []
    for _ in range(5000):
        G = rng.choice([1, 2, 3, 4, 7, 8, 16, 31, 48, 100, 129, 1000])
        nq = rng.choice([0, 1, 2, rng.randint(0, 64), rng.randint(0, 5000)])
        cases.append((nq, rng.choice([0, nq, rng.randint(0, 300), nq + rng.randint(0, 200000)]), G, rng.choice([16, 128, 256]), rng.randint(0, 1), rng.choice([0, 64, 256, 448])))
    check(ask, cases)


def test_steps_are_rounded_up_where_they_fit(ask):
    for G, rows, step in ((1, 128, 128), (3, 128, 43), (7, 16, 3), (100, 128, 2), (300, 256, 1)):
        (_, first, got, *_), = ask([(1000, 5000, G, rows, 0, 256)])
        assert got == step and first == 4000 + step + 256


def test_the_longest_sequences_and_the_most_rows(ask):
    rng, cases = random.Random(2), []
    for G, rows, start in itertools.product([1, 2, 3, 5, 7, 15, 48, 100, 127, 128, 129, 255, 257, 1000, 65535], [16, 128, 256], [0, 64, 256, 448]):
        most = min(2 ** 24, MOST // G)
        for nq in {1, 2, 3, most, most - 1, rng.randint(1, most), rng.randint(1, min(most, 2000))}:
            for nk in (MOST, MOST - 1, MOST - nq, MOST - rng.randint(0, 2 ** 27), nq, 0):
                for tree in (0, 1):
                    cases.append((nq, max(nk, 0), G, rows, tree, start))
    check(ask, cases)
