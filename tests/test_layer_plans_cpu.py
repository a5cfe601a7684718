"""The host-side arithmetic of the single layers' work split
(csrc/norm_plan.h, csrc/adapter_plan.h), compiled by the host compiler: checked
against its definition in Python's unbounded integers, and asked which kernels
calls reach."""
import math
import os
import random
import subprocess

import pytest

from layer_forms import ADAPTER_FORMS, norm_forms

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
    s = ve // math.gcd(ve, c)
    steps = -(-hw // s)
    at = sorted({0, 1, 2, steps // 3, steps // 2, steps // 2 + 1, steps - 2, steps - 1} &
                set(range(steps)))
    where = [(p, v * ve) for p in at for v in {0, s * c // ve // 2, s * c // ve - 1}]
    got = inside([(hw, c, s, steps, p, pos, ve) for p, pos in where])
    for (p, pos), (n,) in zip(where, got):
        want = min(ve, hw * c - (p * s * c + pos))
        assert n == want or (want <= 0 and n <= 0), (p, pos)


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def test_every_group_norm_kernel_is_run_by_a_form(tmp_path):
    """What 60,000 calls of all sizes reach (direction, bytes of an element, vector,
    one group or more of them, pixels of a step, vectors a thread, split or not),
    the forms of layer_forms.py reach as well."""
    run = _compile(str(tmp_path), "norm", r"""
#include "norm_plan.h"
#include <cstdio>
int main() {
  nsc_norm_desc d{};
  long long stride, align, n;
  int backward;
  while (scanf("%d %d %d %d %lld %lld %lld %d", &d.w, &d.c, &d.groups, &d.dtype, &stride, &align,
               &n, &backward) == 8) {
    d.h = 1;
    d.x_stride = d.y_stride = stride;
    const nsc::NormPlan p = nsc::plan_norm(d, (uintptr_t)align, n, backward);
    const bool one = p.ve == 1 || (p.s == 1 && p.ve * nsc::type_bytes(d.dtype) == 16 &&
                                   d.c / d.groups % p.ve == 0);
    printf("%d %d %d %d %d\n", p.ve, one, p.s > 1, p.v, p.parts > 1);
  }
}
""")

    def keys(calls):
        return {(q[7], min(q[3], 1), *k) for q, k in zip(calls, run(calls))}

    rng, calls = random.Random(7), []
    while len(calls) < 60000:
        c = rng.choice([_log_uniform(rng, 1, 1100), 8 * _log_uniform(rng, 1, 200),
                        4 * _log_uniform(rng, 1, 200), 2 * _log_uniform(rng, 1, 300), 16, 32, 64])
        g = rng.choice([g for g in range(1, c + 1) if c % g == 0 and c // g <= 1024])
        hw, n = _log_uniform(rng, 1, 90000), _log_uniform(rng, 1, 4000)
        dtype = rng.choice([0, 1])
        if n * hw * c < 4e9:
            calls.append((hw, c, g, dtype, hw * c + rng.choice([0, 0, 0, 8, 4, 2, 1]),
                          rng.choice([16, 16, 16, 8, 4, 4 - 2 * dtype]), n, rng.choice([0, 1])))
    forms = []
    for backward in (0, 1):
        for dtype, n, hw, c, groups, pad in norm_forms(backward):
            forms.append((hw, c, groups, {"f32": 0, "bf16": 1, "f16": 2}[dtype], hw * c + pad, 16,
                          n, backward))
    reached = keys(calls)
    assert len(reached) > 200
    assert not reached - keys(forms)


def test_every_adapter_kernel_is_run_by_a_form(tmp_path):
    """The same of the adapters' products (tiles, split or not, aligned or not), of
    the rank-wide rows' reductions and of the gradients' waves."""
    run = _compile(str(tmp_path), "adapter", r"""
#include "adapter_plan.h"
#include <cstdio>
int main() {
  nsc_adapter_desc d{};
  long long n;
  int backward;
  while (scanf("%d %d %d %d %d %lld %d", &d.k, &d.d, &d.rank, &d.n_adapters, &d.dtype, &n,
               &backward) == 7) {
    const nsc::AdapterLayout L = nsc::adapter_layout(d, n, backward);
    printf("%d %d %d %d %d %d %d\n", L.g.tn, L.g.tm, L.g.parts > 1, L.list, L.t_parts > 1,
           backward && L.u_parts > 1,
           backward ? nsc::grad_row_waves((int64_t)d.k + d.d, d.n_adapters, n,
                                          nsc::type_bytes(d.dtype)) : 0);
  }
}
""")

    def keys(calls):
        out = set()
        for q, k in zip(calls, run([q[:7] for q in calls])):
            kind = (q[6], min(q[4], 1))
            out.add(("product", *kind, q[7], *k[:3]))
            if q[6]:
                out |= {("gradient", *kind, k[6]), ("its parts", *kind, *k[4:6])}
            else:
                out.add(("rank-wide rows", *kind, *k[2:5]))
        return out

    rng, calls = random.Random(9), []
    for _ in range(60000):
        calls.append((_log_uniform(rng, 1, 10000), _log_uniform(rng, 1, 10000), 8,
                      _log_uniform(rng, 1, 300), rng.choice([0, 1]), _log_uniform(rng, 1, 20000),
                      rng.choice([0, 1]), rng.choice([0, 1])))
    asked = []
    for n, k, d, rank, m, t, pad in ADAPTER_FORMS:
        full = 4 if t == "f32" else 8
        for backward in (0, 1):
            aligned = k % full == 0 and pad % full == 0 and (not backward or d % full == 0)
            asked.append((k, d, rank, m, int(t != "f32"), n, backward, int(aligned)))
    reached = keys(calls)
    assert len(reached) > 40
    assert not reached - keys(asked)
