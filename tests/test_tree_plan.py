"""Arithmetic of attention for several new tokens per sequence that host and kernels share: what a new token sees among 32, and the cut of all units of a call into runs; and what
the compiler made of these kernels.  On the CPU: the header is plain C++, compiled here with the host compiler."""
import os
import random
import re
import subprocess

import pytest

from paper_2605_19726_amd import build
from test_compiled_waits import _asm_files  # (builds what is not built)

PROGRAM = r"""
#include <cstdio>
#include <cstring>
#include "paged_plan.hpp"
int main() {
  char what[16];
  unsigned long long x, y;
  long long a, b, c, d, e;
  while (std::scanf("%15s", what) == 1) {
    if (!std::strcmp(what, "chain") && std::scanf("%lld %lld", &a, &b) == 2) std::printf("%u\n", basa::chain_bits(a, b));
    if (!std::strcmp(what, "tree") && std::scanf("%llu %llu %lld", &x, &y, &a) == 3) std::printf("%u\n", basa::tree_bits(x, y, a));
    if (!std::strcmp(what, "steps") && std::scanf("%lld %lld", &a, &b) == 2) std::printf("%d\n", basa::tree_steps(a, b));
    if (!std::strcmp(what, "units") && std::scanf("%lld %lld", &a, &b) == 2) std::printf("%d\n", basa::tree_units(a, b));
    if (!std::strcmp(what, "rows") && std::scanf("%lld %lld %lld", &a, &b, &c) == 3) {
      const basa::PackedRows r = basa::packed_rows(a, b, c);
      std::printf("%d %d\n", r.row0, r.n);
    }
    if (!std::strcmp(what, "lead") && std::scanf("%lld", &a) == 1) std::printf("%d\n", basa::tree_lead(a));
    if (!std::strcmp(what, "ends") && std::scanf("%lld %lld %lld %lld", &a, &b, &c, &d) == 4)
      std::printf("%d %d\n", basa::decode_first_group(a, c, d), basa::decode_last_group(a, b, c, d));
    if (!std::strcmp(what, "piece") && std::scanf("%lld %lld %lld %lld %lld", &a, &b, &c, &d, &e) == 5) {      // first place, steps, group, run, lead
      const basa::DecodePiece p = basa::decode_piece(a, b, c, d, e);
      std::printf("%d %d %d\n", p.t0, p.t1, basa::decode_part(p, c));
    }
  }
}
"""


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    d = tmp_path_factory.mktemp("tree_plan")
    (d / "p.cpp").write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-Wall", "-Werror", "-fsanitize=undefined", "-fno-sanitize-recover=all", "-I", build.CSRC, str(d / "p.cpp"), "-o", str(d / "p")], check=True)

    def call(questions):
        text = "\n".join(" ".join(str(x) for x in q) for q in questions)
        return [int(x) for x in subprocess.run([str(d / "p")], input=text, check=True, capture_output=True, text=True).stdout.split()]
    return call


def test_a_token_of_a_chain_sees_those_up_to_itself(plan):
    asked = [("chain", t, at) for t in (0, 1, 5, 30, 31, 32, 33, 63, 64, 200) for at in range(-70, 240, 3)]
    asked += [("chain", t, at) for t in (0, 2 ** 24) for at in (-2 ** 30, 2 ** 30)]
    assert plan(asked) == [sum(1 << i for i in range(32) if at + i <= t) for _, t, at in asked]


def test_words_of_a_mask_as_the_bits_of_a_step(plan):
    rng, asked, want = random.Random(1), [], []
    for _ in range(6):
        words = [rng.getrandbits(64) for _ in range(3)] + [0, 0]
        for at in list(range(-40, 192)) + [-2 ** 30]:
            low = max(at, 0) // 64
            asked.append(("tree", words[low], words[low + 1], at))
            # tokens before the new ones are seen by all
            want.append(sum(1 << i for i in range(32) if at + i < 0 or words[(at + i) // 64] >> ((at + i) % 64) & 1))
    assert plan(asked) == want


def test_rows_of_a_sequence_are_rows_of_the_batch(plan):
    """Whatever the offsets are, also where their difference is no 32-bit number: within [0, tokens], less than none where they do not ascend."""
    ends = [-2 ** 31, -2 ** 31 + 1, -1800, -1, 0, 1, 5, 1799, 1800, 1801, 2 ** 30, 2 ** 31 - 1]
    asked = [("rows", a, b, t) for a in ends for b in ends for t in (1, 6, 1800, 2 ** 30)]
    got = plan(asked)
    for (_, a, b, t), row0, n in zip(asked, got[::2], got[1::2]):
        first, end = (max(0, min(x, t)) for x in (a, b))
        assert (row0, n) == (first, end - first) and (n >= 0 or b < a)


@pytest.mark.parametrize("step", [16, 32])
def test_runs_take_every_step_of_every_unit_once(plan, step):
    rng = random.Random(step)
    lead = plan([("lead", step)])[0]
    assert lead >= 1
    for case in range(60):
        n, heads, tile, group = rng.randint(1, 30), rng.choice([1, 2, 5, 8, 9]), rng.choice([32, 64, 128, 256]), rng.choice([1, 4, 7])
        lens = [int(2 ** rng.uniform(0, rng.choice([7, 12, 16]))) - 1 for _ in range(n)]
        rows = [rng.choice([0, 1, 5, 33, 300]) * group for _ in range(n)]
        got = plan([q for x, r in zip(lens, rows) for q in (("steps", x, step), ("units", r, tile))])
        steps, units = got[::2], got[1::2]
        assert steps == [max(1, -(-x // step)) for x in lens] and units == [-(-r // tile) for r in rows]
        # one KV head after the other, in each the sequences, in each its units: (steps, first place)
        axis, at = [], 0
        for _ in range(heads):
            for s, u in zip(steps, units):
                for _ in range(u):
                    axis.append((s, at))
                    at += s + lead
        runs = rng.choice([8, 256, 512])
        run = max(-(-at // runs), 1)
        ends = plan([("ends", first, s, run, lead) for s, first in axis])
        asked, of = [], []
        for i, (s, first) in enumerate(axis):
            for g in range(max(ends[2 * i] - 1, 0), min(ends[2 * i + 1] + 1, runs - 1) + 1):
                asked.append(("piece", first, s, g, run, lead))
                of.append((i, g))
        got = plan(asked) if asked else []
        done, places = [0] * len(axis), set()
        for (i, g), t0, t1, place in zip(of, got[::3], got[1::3], got[2::3]):
            assert (t1 > t0) == (ends[2 * i] <= g <= ends[2 * i + 1])
            if t1 <= t0:
                continue
            assert t0 == done[i]
            done[i] = t1
            if (t0, t1) != (0, axis[i][0]):
                assert place == 2 * g + (g == ends[2 * i]) and place not in places       # where the join looks for it
                places.add(place)
        assert done == [s for s, _ in axis]


def test_no_kernel_spills():
    files = [f for f in _asm_files() if os.path.basename(f).startswith(("attn_tree-", "page_ops-"))]
    assert len(files) == 2, build.OBJ_DIR
    found, kernels = {}, 0
    for path in files:
        kernel = None
        for line in open(path):
            m = re.match(r"\s*\.amdhsa_(kernel|private_segment_fixed_size) (\S+)", line)
            if m and m.group(1) == "kernel":
                kernel = m.group(2)
                kernels += 1
            elif m and int(m.group(2)):
                found[kernel] = int(m.group(2))
    assert kernels > 20 and found == {}


def test_m0_is_an_operand_of_the_assembly_that_reads_it():
    """The compiler may keep a value in m0 across a statement that writes it unsaid: loads into the LDS take it as an operand, and no statement sets it."""
    found = 0
    for name in sorted(os.listdir(build.CSRC)):
        text = open(os.path.join(build.CSRC, name)).read()
        for m in re.finditer(r"\basm\b(?:\s+volatile)?\s*\((.*?)\);", text, re.S):
            assert not re.search(r"\bs_\w+\s+m0\b", m.group(1)), f"{name}: {m.group(0)}"
            if "load_lds" in m.group(1):
                found += 1
                assert '"{m0}"' in m.group(1), f"{name}: {m.group(0)}"
    assert found >= 2
    # what became of it: every such load has a write of m0 before it in its block, and no other load between the two
    (path,) = [f for f in _asm_files() if os.path.basename(f).startswith("attn_tree-")]
    loads, written = 0, False
    for line in open(path):
        if re.match(r"\.?\w+:", line):
            written = False
        elif re.match(r"\s*s_\w+ m0,", line):
            written = True
        elif "global_load_lds" in line:
            assert written, line
            loads, written = loads + 1, False
    assert loads > 100
