"""Whether two tensors share memory, as the entry points ask: the header is plain C++, compiled here with the host compiler, against the sets of bytes."""
import random
import subprocess

import pytest

from paper_2605_19726_amd import build

PROGRAM = r"""
#include <cstdio>
#include "row_sets.hpp"
int main() {
  unsigned long long v[16];
  for (;;) {
    for (auto& x : v) if (std::scanf("%llu", &x) != 1) return 0;
    basa::RowSet s[2];
    for (int i = 0; i < 2; ++i) {
      const unsigned long long* w = v + 8 * i;
      s[i] = basa::row_set(reinterpret_cast<const void*>((uintptr_t)w[0]), w[1], {w[2], w[3], w[4]}, {w[5], w[6], w[7]});
    }
    std::printf("%d %d %d\n", (int)basa::overlap(s[0], s[1]), (int)basa::is_nested(s[0]), (int)basa::is_nested(s[1]));
  }
}
"""


@pytest.fixture(scope="module")
def ask(tmp_path_factory):
    d = tmp_path_factory.mktemp("row_sets")
    (d / "p.cpp").write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-Wall", "-Werror", "-fsanitize=undefined", "-fno-sanitize-recover=all", "-I", build.CSRC, str(d / "p.cpp"), "-o", str(d / "p")], check=True)

    def call(pairs):
        text = "\n".join(" ".join(str(x) for at, width, n, stride in p for x in (at, width, *n, *stride)) for p in pairs)
        got = [int(x) for x in subprocess.run([str(d / "p")], input=text, check=True, capture_output=True, text=True).stdout.split()]
        return list(zip(got[::3], got[1::3], got[2::3]))
    return call


def members(at, width, n, stride):
    return {at + i * stride[0] + j * stride[1] + k * stride[2] + x for i in range(n[0]) for j in range(n[1]) for k in range(n[2]) for x in range(width)}


def test_against_sets_of_bytes(ask):
    rng = random.Random(3)
    pairs = []
    for _ in range(4000):
        pair = []
        for _ in range(2):
            n = [rng.choice([1, 1, 2, 3, 5]) for _ in range(3)]
            width = rng.randint(1, 6)
            inner = rng.randint(0, 8)
            axes = [inner, inner * n[2] + rng.randint(0, 6), 0]
            axes[2] = axes[1] * n[1] + rng.randint(0, 9)
            stride = axes[::-1] if rng.random() < 0.7 else [rng.randint(0, 30) for _ in range(3)]
            order = rng.sample(range(3), 3)
            pair.append((1000 + rng.randint(0, 60), width, [n[i] for i in order], [stride[i] for i in order]))
        pairs.append(pair)
    answers = ask(pairs)
    exact = 0
    for pair, (got, a, b) in zip(pairs, answers):
        want = bool(members(*pair[0]) & members(*pair[1]))
        if a or b:
            exact += 1
            assert got == want, pair
        else:
            assert got >= want, pair                        # neither is nested: never a shared byte missed
    assert exact > 3000 and 0.2 < sum(x[0] for x in answers) / len(answers) < 0.9


def test_slices_of_one_buffer(ask):
    T, h, d = 1000, 8, 256
    row = 3 * h * d
    q, k = (2 ** 40, d, [1, h, T], [0, d, row]), (2 ** 40 + h * d, d, [1, h, T], [0, d, row])           # of a projection
    even, odd = (2 ** 40, d, [1, h // 2, T], [0, 2 * d, row]), (2 ** 40 + d, d, [1, h // 2, T], [0, 2 * d, row])
    assert [x[0] for x in ask([(q, k), (q, q), (even, odd), (even, q), (k, odd)])] == [0, 1, 0, 1, 0]
    # K and V interleaved in pages; another tensor behind them, in a gap of theirs, and across its edge
    page = 2 * 16 * h * d
    kv = (2 ** 40, d, [500, h, 16], [page, d, h * d])
    v = (2 ** 40 + page // 2, d, [500, h, 16], [page, d, h * d])
    for at, want in ((2 ** 40 + 500 * page, 0), (2 ** 40 + 7 * page + page // 2, 0), (2 ** 40 + 7 * page + page // 2 - 1, 1), (2 ** 40 + 8 * page - 1, 1)):
        assert ask([(kv, (at, 2, [1, 1, 1], [0, 0, 0]))])[0][0] == want
    assert ask([(kv, v)])[0][0] == 0


def test_nothing_and_more_than_there_is(ask):
    some = (4096, 64, [3, 1, 1], [64, 0, 0])
    assert [x[0] for x in ask([(some, (0, 64, [1, 1, 1], [0, 0, 0])), (some, (4096, 0, [1, 1, 1], [0, 0, 0])), (some, (4096, 64, [0, 1, 1], [0, 0, 0])),
                               (some, (4096 + 191, 1, [2 ** 20, 2 ** 30, 1], [2 ** 50, 2 ** 60, 0])), (some, (4096 + 192, 1, [2 ** 31, 65535, 2 ** 20], [2 ** 62, 2 ** 62, 2 ** 61]))])] == [0, 0, 0, 1, 0]
