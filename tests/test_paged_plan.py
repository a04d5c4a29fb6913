"""Arithmetic of the paged cache that host and kernels share: division by a page size, and the cut of all tiles of a decode call into runs.
On the CPU: the header is plain C++, compiled here with the host compiler."""
import random
import subprocess

import pytest

from paper_2605_19726_amd import build

PROGRAM = r"""
#include <cstdio>
#include <cstring>
#include "paged_plan.hpp"
int main() {
  char what[16];
  long long a, b, c;
  while (std::scanf("%15s %lld %lld %lld", what, &a, &b, &c) == 4) {
    if (!std::strcmp(what, "div")) std::printf("%u\n", basa::fast_div((uint32_t)b).div((uint32_t)a));
    if (!std::strcmp(what, "run")) std::printf("%lld\n", (long long)basa::decode_run(a, (int)b));
    if (!std::strcmp(what, "tiles")) std::printf("%lld\n", (long long)basa::decode_tiles(a));
    if (!std::strcmp(what, "part")) std::printf("%d\n", basa::decode_part(a, b, c));
  }
}
"""


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    d = tmp_path_factory.mktemp("plan")
    (d / "p.cpp").write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-Wall", "-Werror", "-I", build.CSRC, str(d / "p.cpp"), "-o", str(d / "p")], check=True)

    def call(questions):
        text = "\n".join("%s %d %d %d" % tuple((list(q) + [0, 0])[:4]) for q in questions)
        return [int(x) for x in subprocess.run([str(d / "p")], input=text, check=True, capture_output=True, text=True).stdout.split()]
    return call


def test_division_by_a_page_size(plan):
    rng, asked = random.Random(1), []
    top = 2 ** 31 - 1
    for d in [1, 2, 3, 5, 7, 16, 20, 25, 64, 100, 127, 128, 255, 256, 641, 65535, 65536, 65537, 2 ** 30 - 1, 2 ** 30, 2 ** 30 + 1, top - 1, top]:
        near = [0, 1, d - 1, d, d + 1, 2 * d - 1, 2 * d, top - top % d - 1, top - top % d, top - 1, top]
        asked += [("div", n, d) for n in near + [rng.randrange(2 ** 31) for _ in range(40)] if 0 <= n <= top]
    assert plan(asked) == [n // d for _, n, d in asked]


def test_runs_cover_all_tiles_and_give_every_piece_a_place_of_its_own(plan):
    rng = random.Random(2)
    for _ in range(60):
        groups = rng.choice([1, 2, 5, 64, 768])
        lens = [int(2 ** rng.uniform(0, 14)) - 1 for _ in range(rng.randint(1, 40))]
        tiles = plan([("tiles", n) for n in lens])
        assert tiles == [max(1, -(-n // 32)) for n in lens]
        total = sum(tiles)
        run, = plan([("run", total, groups)])
        assert run % 4 == 0 and run * groups >= total and (run - 4) * groups < total
        first, places, questions = 0, set(), []
        for t in tiles:
            g0, g1 = first // run, (first + t - 1) // run
            if g0 != g1:
                questions += [("part", first, g, run) for g in range(g0, g1 + 1)]
            first += t
        got = plan(questions)
        assert len(set(got)) == len(got) and all(0 <= p < 2 * groups and p // 2 == q[2] for p, q in zip(got, questions))
