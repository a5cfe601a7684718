"""The host-side arithmetic of the single layers' work split
(csrc/norm_plan.h), compiled by the host compiler and checked against its
definition in Python's unbounded integers."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_1703_02529_amd", "csrc")


def _compile(tmp, name, body):
    """A host program of the given C++ source; returns a function that runs it
    with one line of integers per query and gives its lines of integers."""
    src, exe = os.path.join(tmp, name + ".cpp"), os.path.join(tmp, name)
    with open(src, "w") as f:
        f.write(body)
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-fsanitize=undefined",
                    "-fno-sanitize-recover=undefined", "-I", CSRC, "-I",
                    os.path.join(ROOT, "include"), src, "-o", exe], check=True)

    def run(queries):
        text = "\n".join(" ".join(str(int(v)) for v in q) for q in queries) + "\n"
        out = subprocess.run([exe], input=text, capture_output=True, text=True, check=True).stdout
        return [[int(v) for v in line.split()] for line in out.splitlines()]
    return run


@pytest.fixture(scope="module")
def inside(tmp_path_factory):
    return _compile(str(tmp_path_factory.mktemp("inside")), "inside", r"""
#include "norm_plan.h"
#include <cstdio>
int main() {
  int hw, c, s, steps, p, pos, ve;
  while (scanf("%d %d %d %d %d %d %d", &hw, &c, &s, &steps, &p, &pos, &ve) == 7)
    printf("%d\n", nsc::values_inside(hw, c, s, steps, p, pos, ve));
}
""")


@pytest.mark.parametrize("hw,c,ve", [
    (5, 3, 8), (64, 45, 8), (37 * 41, 45, 4), (1, 1, 8), (4096 * 4096, 127, 8),
    (4096 * 4096, 129, 8), (4096 * 4096, 255, 8), (4095 * 4096 + 1, 1023, 4),
    (4096 * 4096 - 3, 509, 2), (4096 * 4096 - 1, 65535, 8)])
def test_values_of_a_vector_inside_an_image(inside, hw, c, ve):
    """Every vector that begins in the image holds min(ve, values left) of it,
    also where an image has more than 2^31 values."""
    import math
    s = ve // math.gcd(ve, c)
    steps = -(-hw // s)
    at = sorted({0, 1, 2, steps // 3, steps // 2, steps // 2 + 1, steps - 2, steps - 1} &
                set(range(steps)))
    where = [(p, v * ve) for p in at for v in {0, s * c // ve // 2, s * c // ve - 1}]
    got = inside([(hw, c, s, steps, p, pos, ve) for p, pos in where])
    for (p, pos), (n,) in zip(where, got):
        want = min(ve, hw * c - (p * s * c + pos))
        assert n == want or (want <= 0 and n <= 0), (p, pos)
