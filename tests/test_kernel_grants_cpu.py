"""The record of the kernels' shared memory sizes, compiled for the host: concurrent first calls with different sizes."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_the_larger_size_stays_set(tmp_path):
    exe, src = str(tmp_path / "kernel_grants_check"), os.path.join(ROOT, "tests", "sanitize", "kernel_grants_check.cpp")
    subprocess.run(["g++", "-std=c++17", "-Wall", "-Werror", "-pthread", "-fsanitize=address,undefined", "-fno-sanitize-recover=all", "-I",
                    os.path.join(ROOT, "include"), "-I", os.path.join(ROOT, "paper_2609_36959_b200", "csrc"), src, "-o", exe], check=True)
    out = subprocess.run([exe], capture_output=True, text=True, check=True, timeout=60).stdout.split()
    attribute, again, lower, other, failed, retried, calls = map(int, out)
    assert attribute == 100000
    assert again == lower == other == retried == 0 and failed == -4
    assert calls == 2                                     # the other device, and the one that had failed
