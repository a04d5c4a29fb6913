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
    if (!std::strcmp(what, "run")) std::printf("%lld\n", (long long)basa::decode_run(a));
    if (!std::strcmp(what, "steps")) std::printf("%lld\n", (long long)basa::decode_steps(a));
    if (!std::strcmp(what, "groups")) std::printf("%lld\n", (long long)basa::decode_groups(a));
    if (!std::strcmp(what, "first")) std::printf("%lld\n", (long long)basa::decode_first_group(a, b));
    if (!std::strcmp(what, "last")) std::printf("%lld\n", (long long)basa::decode_last_group(a, b, c));
    if (!std::strcmp(what, "piece")) {          // a: first place, b: steps, c: group, d: run
      long long d;
      if (std::scanf("%lld", &d) != 1) return 1;
      const basa::DecodePiece p = basa::decode_piece(a, b, c, d);
      std::printf("%lld %lld %lld\n", (long long)p.t0, (long long)p.t1, (long long)basa::decode_part(p, c));
    }
  }
}
"""


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    d = tmp_path_factory.mktemp("plan")
    (d / "p.cpp").write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-Wall", "-Werror", "-I", build.CSRC, str(d / "p.cpp"), "-o", str(d / "p")], check=True)

    def call(questions):
        text = "\n".join("%s %d %d %d" % tuple((list(q) + [0, 0])[:4]) + (" %d" % q[4] if len(q) > 4 else "") for q in questions)
        return [int(x) for x in subprocess.run([str(d / "p")], input=text, check=True, capture_output=True, text=True).stdout.split()]
    return call


def test_division_by_a_page_size(plan):
    rng, asked = random.Random(1), []
    top = 2 ** 31 - 1
    for d in [1, 2, 3, 5, 7, 16, 20, 25, 64, 100, 127, 128, 255, 256, 641, 65535, 65536, 65537, 2 ** 30 - 1, 2 ** 30, 2 ** 30 + 1, top - 1, top]:
        near = [0, 1, d - 1, d, d + 1, 2 * d - 1, 2 * d, top - top % d - 1, top - top % d, top - 1, top]
        asked += [("div", n, d) for n in near + [rng.randrange(2 ** 31) for _ in range(40)] if 0 <= n <= top]
    assert plan(asked) == [n // d for _, n, d in asked]


def test_runs_take_every_step_once_and_give_every_piece_a_place_of_its_own(plan):
    rng = random.Random(2)
    for case in range(80):
        n, most = rng.randint(1, 60), rng.choice([7, 12, 16, 20])
        lens = [int(2 ** rng.uniform(0, most)) - 1 for _ in range(n)]
        steps = plan([("steps", x) for x in lens])
        assert steps == [max(1, -(-x // 128)) for x in lens]
        total = sum(steps) + n                                   # a place in front of every sequence
        run, groups = plan([("run", total), ("groups", total)])
        assert run >= 1 and run * groups >= total                # the launch has a group for every run
        first, asked = 0, []
        for t in steps:
            asked += [("first", first, run), ("last", first, t, run)]
            first += t + 1
        ends, first, questions, of = plan(asked), 0, [], []
        for i, t in enumerate(steps):
            g0, g1 = ends[2 * i], ends[2 * i + 1]
            for g in range(max(g0 - 1, 0), min(g1 + 1, groups - 1) + 1):
                questions.append(("piece", first, t, g, run))
                of.append((i, g, g0 <= g <= g1))
            first += t + 1
        got = plan(questions)
        done, places = [0] * n, set()
        for (i, g, inside), t0, t1, place in zip(of, got[::3], got[1::3], got[2::3]):
            assert (t1 > t0) == inside                           # the groups between first and last, and no others, have steps of it
            if not inside:
                continue
            assert t0 == done[i]                                 # in order, without a gap
            done[i] = t1
            if (t0, t1) != (0, steps[i]):
                assert place not in places and place // 2 == g < groups
                places.add(place)
        assert done == steps


def test_a_launch_has_a_workgroup_for_every_run_of_several_units(plan):
    """Units of query heads share the places; the length of a run goes by places times units, the launch by the most there can be."""
    rng = random.Random(3)
    totals = [1, 2, 511, 512, 513, 12287, 12288, 12289, 16384, 16385, 10 ** 6, 10 ** 8] + [int(2 ** rng.uniform(0, 27)) for _ in range(200)]
    for units in (1, 2, 3, 4, 7):
        runs = plan([("run", t * units) for t in totals])
        groups = plan([("groups", t * units) for t in totals])
        for t, run, g in zip(totals, runs, groups):
            assert -(-t // run) <= -(-g // units), (t, units, run, g)
