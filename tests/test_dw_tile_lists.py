"""The lists of tiles that the gradients of the experts' weights are dealt out in, for experts of up to 2^30 rows: the arithmetic, compiled for the host."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
START = 96  # rows that a tile's start counts as

PROGRAM = r'''
#include <cstdio>
#include <vector>
#include "tile_lists.hpp"
// reads per, E and the experts' rows; prints the nine edges
int main() {
    int per, E;
    while (scanf("%d %d", &per, &E) == 2) {
        std::vector<int> used(E), first(E);
        int total = 0;
        for (int e = 0; e < E; ++e) {
            if (scanf("%d", &used[e]) != 1) return 1;
            first[e] = total, total += used[e] + moe::kDwStart;
        }
        for (int x = 0; x <= moe::kDwLists; ++x) printf("%d ", moe::dw_edge(x, E, per, total, first.data(), used.data()));
        printf("\n");
    }
}
'''


@pytest.fixture(scope="module")
def edges(tmp_path_factory):
    at = tmp_path_factory.mktemp("lists")
    (at / "edges.cpp").write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-Wall", "-Wextra", "-Werror", "-I",
                    os.path.join(ROOT, "paper_2605_00686_amd", "csrc"), str(at / "edges.cpp"), "-o", str(at / "edges")], check=True)

    def ask(per, used):
        out = subprocess.run([str(at / "edges")], input=f"{per} {len(used)} {' '.join(map(str, used))}", capture_output=True, text=True, check=True)
        return [int(v) for v in out.stdout.split()]
    return ask


MOST = 1 << 30
ROWS = [[0], [5], [2 ** 28 - 97], [2 ** 28 - 96], [2 ** 28], [2 ** 29 - 96], [2 ** 29], [2 ** 29 + 10 ** 6], [2 ** 29 + 2 ** 28], [MOST],
        [2 ** 29, 2 ** 29], [0, MOST, 0], [2 ** 29 + 7, 3, 0, 2 ** 28], [0] * 255 + [MOST], [MOST - 255] + [1] * 255, [0] * 256, [2 ** 22] * 256,
        [17 * i for i in range(200)]]


@pytest.mark.parametrize("used", ROWS, ids=lambda u: f"{len(u)}x{max(u)}")
def test_every_list_is_a_stretch_of_the_tiles(edges, used):
    for per in (1, 2, 32, 1001, (MOST - 1) // len(used)):
        got = edges(per, used)
        assert len(got) == 9 and got[0] == 0 and got[8] == per * len(used)
        assert all(a <= b for a, b in zip(got, got[1:])), got
        # the work in front of an edge is its share, to a tile
        weights = [u + START for u in used]
        before = [sum(weights[:e]) for e in range(len(used) + 1)]
        for x, at in enumerate(got):
            e, t = divmod(at, per)
            work = before[e] * per + (t * weights[e] if e < len(used) else 0)
            want = x * before[-1] * per
            assert 8 * work <= want < 8 * (work + (weights[e] if e < len(used) else 1)), (x, per)
