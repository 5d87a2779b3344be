"""How attention's tiles are dealt out (csrc/wm_units.h), compiled for the host: shares cover all tiles in order, a tile's worker
is the one whose share has it, and numbers beyond 32 bits are whole."""
import os
import random
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PROGRAM = r"""
#include <cstdio>
#include <cinttypes>
#include "wm_units.h"
int main()
{
    char what;
    unsigned long long a, b, c;
    while (scanf(" %c %llu %llu %llu", &what, &a, &b, &c) == 4) {
        if (what == 's') printf("%llu\n", wm::share_of((uint32_t)a, b, c));
        if (what == 'w') printf("%u\n", wm::worker_of(a, b, c));
        if (what == 't') { const wm::TileAt t = wm::tile_at(a, (uint32_t)b); printf("%u %u\n", t.unit, t.j); }
        if (what == 'n') printf("%llu\n", wm::tiles_of((uint32_t)a, (uint32_t)b));
    }
}
"""


@pytest.fixture(scope="module")
def ask(tmp_path_factory):
    d = tmp_path_factory.mktemp("units")
    (d / "units.cpp").write_text(PROGRAM)
    subprocess.check_call(["g++", "-O1", "-std=c++17", "-Wall", "-I", os.path.join(ROOT, "paper_2607_10389_b200", "csrc"),
                           str(d / "units.cpp"), "-o", str(d / "units")])

    def run(lines):
        text = "\n".join(" ".join(str(x) for x in line) for line in lines)
        out = subprocess.run([str(d / "units")], input=text, capture_output=True, text=True, check=True).stdout.splitlines()
        assert len(out) == len(lines)
        return [[int(v) for v in x.split()] for x in out]
    return run


def test_a_tile_s_unit_at_every_size(ask):
    r = random.Random(1)
    cases = []
    for _ in range(4000):
        nt = min(1 << 23, int(2 ** r.uniform(0, 23)) + r.choice([0, 1]))
        unit = int(2 ** r.uniform(0, 31)) - 1
        cases.append((unit * nt + r.choice([0, nt - 1, r.randrange(nt)]), nt))
    cases += [(2 ** 32 - 1, 1 << 23), (2 ** 32, 1 << 23), (2 ** 32 + 5, 3), ((2 ** 31 - 1) * 2 ** 23, 1 << 23)]
    assert any(off >> 32 for off, _ in cases)
    assert ask([("t", off, nt, 0) for off, nt in cases]) == [[off // nt, off % nt] for off, nt in cases]


def test_a_count_of_tiles_at_every_size(ask):
    cases = [(1024, 1 << 23), (1024, (1 << 22) + 1), (512, 1 << 23), (1, 1), (16, 54)]
    assert ask([("n", u, nt, 0) for u, nt in cases]) == [[u * nt] for u, nt in cases]


@pytest.mark.parametrize("grid", [148, 160, 296, 320])
def test_shares_cover_all_tiles_and_know_their_workers(ask, grid):
    r = random.Random(grid)
    for total in [1, 2, grid - 1, grid, grid + 1, 4 * grid + 3, 2 ** 23 - 1, 2 ** 23, 2 ** 32 + 7, 2 ** 54 + 12345] + [int(2 ** r.uniform(0, 50)) for _ in range(20)]:
        workers = min(grid, total)
        at = [x[0] for x in ask([("s", w, total, workers) for w in range(grid + 1)])]
        assert at[0] == 0 and all(a < b for a, b in zip(at[:workers], at[1:workers + 1])) and all(a == total for a in at[workers:])
        tiles = sorted({t for a in at[:workers] for t in (a, a - 1) if 0 <= t < total} | {total - 1, total // 2})
        for t, (w,) in zip(tiles, ask([("w", t, total, workers) for t in tiles])):
            assert at[w] <= t < at[w + 1]
