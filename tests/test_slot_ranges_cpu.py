"""Slots of offsets that are not in order: the rule that the feed-forward's plan applies, compiled for the host.  Its ranges
are disjoint and need no more tiles than the workspace holds."""
import os
import random
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("slots") / "slot_ranges_check")
    src = os.path.join(ROOT, "tests", "sanitize", "slot_ranges_check.cpp")
    subprocess.run(["g++", "-std=c++17", "-Wall", "-Werror", "-fsanitize=address,undefined", "-fno-sanitize-recover=all", "-I",
                    os.path.join(ROOT, "paper_2609_36959_b200", "csrc"), src, "-o", exe], check=True)
    return exe


def _cases():
    rng = random.Random(3)
    yield 4096, [(0, 4096)[i & 1] for i in range(65)], list(range(64))
    yield 65536, [0, 65536, 0, 65536, 0], [0, 1, 2, 3]
    yield 40, [0, 20, 10, 100000], [0, 1, 0]
    yield 100, [50, 100, 0, 80], [0, 1, 2]
    yield 100, [2**32 - 1, 0, 7, 2**31, 3], [0, 1, 2, 3]
    yield 0, [0, 5, 1], [0, 0]
    for _ in range(400):
        D, P = rng.randint(1, 40), rng.choice([1, 7, 300, 5000])
        offsets = [rng.randint(0, P + P // 4) for _ in range(D + 1)]
        if rng.random() < 0.5:                             # in order but for a few
            offsets.sort()
            for _ in range(rng.randint(0, 3)):
                offsets[rng.randint(0, D)] = rng.randint(0, P)
        yield P, offsets, [rng.randint(-1, 5) for _ in range(D)]


def test_ranges_are_disjoint_and_fit_the_tile_list(program):
    cases = list(_cases())
    text = "\n".join(" ".join(map(str, [P, len(e), *o, *e])) for P, o, e in cases)
    lines = subprocess.run([program], input=text, capture_output=True, text=True, check=True).stdout.splitlines()
    assert len(lines) == len(cases)
    for (P, offsets, experts), line in zip(cases, lines):
        got = [int(v) for v in line.split()]
        bound, slots = got[0], list(zip(got[1::3], got[2::3], got[3::3]))
        top = min(offsets[0], P)
        tiles, owner = 0, [None] * P
        for d, (first, rows, expert) in enumerate(slots):
            end = min(offsets[d + 1], P)
            want = max(0, end - top)                       # running maximum
            assert first == top and rows == (want if experts[d] >= 0 else 0), (offsets, d)
            assert expert == (experts[d] if rows else -1)
            for r in range(first, first + rows):
                assert owner[r] is None
                owner[r] = d
            tiles += (rows + 255) // 256
            top = max(top, end)
        assert tiles <= bound
