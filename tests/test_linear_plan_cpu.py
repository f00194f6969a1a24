"""linear's plan and workspace, compiled for the host: the parts of every product fit in the workspace, every split has blocks, and a call
of few tokens does not have to bring the workspace of many."""
import os
import random
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("plan") / "linear_plan_check")
    src = os.path.join(ROOT, "tests", "sanitize", "linear_plan_check.cpp")
    subprocess.run(["g++", "-O1", "-std=c++17", "-Wall", "-Werror", "-fsanitize=address,undefined", "-fno-sanitize-recover=all", "-I",
                    os.path.join(ROOT, "paper_2609_36959_b200", "csrc"), src, "-o", exe], check=True)

    def run(cases):
        text = "\n".join("%d %d %d" % c for c in cases)
        out = subprocess.run([exe], input=text, capture_output=True, text=True, check=True).stdout.splitlines()
        assert len(out) == len(cases)
        return [[int(v) for v in line.split()] for line in out]

    return run


def _cases():
    rng = random.Random(7)
    cases = [(1, 8, 8), (5, 65536, 8), (4096, 64, 64), (131072, 7168, 256), (300, 16384, 16384), (1 << 20, 8, 16), ((1 << 31) - (1 << 21), 8, 8),
             ((1 << 31) - (1 << 21), 65536, 65536), (1, 65536, 65536), (1, 7168, 2048), (257, 1000, 200)]
    for _ in range(3000):
        cases.append((int(2 ** rng.uniform(0, 20)), 8 * int(2 ** rng.uniform(0, 13)), 8 * int(2 ** rng.uniform(0, 13))))
    return cases


def test_parts_fit_in_the_workspace(plan):
    cases = _cases()
    for case, got in zip(cases, plan(cases)):
        size, bias, products = got[0], got[-1], [got[1 + 5 * i:6 + 5 * i] for i in range(4)]
        assert size % 256 == 0 and bias <= size
        for blocks, parts, n, splits, per in products:
            assert parts <= size, (case, products)
            assert n % 32 == 0 and 32 <= n <= 256 and 1 <= splits <= 32
            assert per * (splits - 1) < blocks <= per * splits


def test_the_librarys_sizes_are_these(plan):
    from paper_2609_36959_b200 import build
    build.build()
    import paper_2609_36959_b200.binding as cb
    cases = [c for c in _cases() if c[0] <= (1 << 31) - (1 << 21)][:400]
    for (T, K, N), got in zip(cases, plan(cases)):
        assert cb.linear_workspace_bytes(T, K, N) == got[0]


def test_few_tokens_need_no_workspace_of_many(plan):
    """One token's gradients are products of one block of k: their parts are those of one token's row.  65 tokens have two blocks."""
    for K, N in ((7168, 2048), (4096, 4096), (16384, 16384), (1000, 200)):
        one, two, some = (got[0] for got in plan([(1, K, N), (65, K, N), (257, K, N)]))
        row = 32 * max(K, N) * 4
        assert one <= row + 256
        assert two <= max(65 * row, 2 * K * N * 4) + 256
        assert some <= max(257 * row, 5 * K * N * 4) + 256
