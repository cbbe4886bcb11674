"""How the steps around the attention are spread over the chip (csrc/row_plan.h), on the CPU: the header itself, compiled for the host.  Every row
is taken once, by threads that there are."""
import collections
import os
import random
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "paper_2602_12675_amd", "csrc", "row_plan.h")
NORMS, PARTS, MODS = ["none", "head", "token"], {"before": 1, "after": 2, "both": 3}, ["batch", "token", "shared"]

# what row_plan.h takes from common.h
COMMON = """#pragma once
#include <stddef.h>
#include <stdint.h>
#include "sla2.h"
#define __host__
#define __device__
namespace sla2 { constexpr int kWave = 64; }
"""
MAIN = """#include <stdio.h>
#include "row_plan.h"
using namespace sla2;
int main() {      // per line: kind backward, then B H N d norm bf16 tensors | B N C part mods x_n h_n mod_n
  int kind, backward;
  while (scanf("%d %d", &kind, &backward) == 2) {
    if (kind == 0) {
      RopeArgs a{};
      int bf16;
      if (scanf("%d %d %d %d %d %d %d", &a.B, &a.H, &a.N, &a.d, &a.norm, &bf16, &a.tensors) != 7) return 1;
      a.bf16 = bf16;
      plan_rope(&a, backward);
      const size_t floats = rope_partial_floats(a);
      if (backward && a.norm) plan_rope_direct(&a);
      printf("%d %d %d %d %d %d %d %d %d %zu\\n", a.team.lanes, a.team.waves, a.team.vec, a.teams, a.walkers, a.direct, a.groups, a.heads, a.cached, floats);
    } else {
      NormArgs a{};
      int part;
      if (scanf("%d %d %d %d %d %lld %lld %lld", &a.B, &a.N, &a.C, &part, &a.mods, &a.x_n, &a.h_n, &a.mod_n) != 8) return 1;
      const void* there = &a;
      if (part & kAfter) a.y = there;
      if (part & kBefore) (backward ? a.dh : *(const void**)&a.h) = there;
      plan_norm(&a, backward);
      if (backward) plan_norm_direct(&a);
      printf("%d %d %d %d %d %d 1 0 0 0\\n", a.team.lanes, a.team.waves, a.team.vec, a.teams, a.walkers, a.direct);
    }
  }
}
"""
Plan = collections.namedtuple("Plan", "lanes waves vec teams walkers direct groups heads cached floats")


@pytest.fixture(scope="module")
def plans(tmp_path_factory):
    """plans(list of lines) -> list of Plan"""
    if shutil.which("g++") is None:
        pytest.skip("no C++ compiler")
    folder = tmp_path_factory.mktemp("plan")
    shutil.copy(HEADER, folder / "row_plan.h")
    (folder / "common.h").write_text(COMMON)
    (folder / "main.cpp").write_text(MAIN)
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), "-o", "plan", "main.cpp"], cwd=folder, check=True)

    def ask(lines):
        got = subprocess.run([str(folder / "plan")], input="\n".join(" ".join(map(str, x)) for x in lines) + "\n", capture_output=True, text=True,
                             check=True, timeout=60).stdout.splitlines()
        assert len(got) == len(lines)
        return [Plan(*map(int, x.split())) for x in got]
    return ask


def rope(B, H, N, d, norm="token", bf16=True, tensors=2, backward=False):
    return 0, int(backward), B, H, N, d, NORMS.index(norm), int(bf16), tensors


def norm(B, N, C, part="both", mods="batch", backward=False, stride=None):
    return 1, int(backward), B, N, C, PARTS[part], MODS.index(mods), stride or C, stride or C, C if mods == "token" else 0


def steps(plan, N):
    """Rows that a team takes one after the other."""
    return -(-N // (plan.teams * plan.walkers))


def check(p, N, chunks, per_part, most_vec, most_threads):
    threads = p.lanes * p.waves
    assert p.lanes in (8, 16, 32, 64) and (p.lanes == 64 or p.waves == 1) and 1 <= p.vec <= most_vec
    assert threads * p.vec >= chunks and p.teams >= 1 and p.walkers >= 1
    assert -(-p.teams * threads // 64) * 64 <= most_threads
    assert (steps(p, N) - 1) * p.teams * p.walkers < N                       # no step without a row
    assert (p.walkers - 1) * p.teams < N                                     # no workgroup without a row
    assert per_part * p.walkers <= max(per_part, 1024)                       # as many workgroups as are resident, or one for each sequence
    if p.direct:
        assert per_part == 1 and p.walkers == 1 and p.teams >= N


def test_every_row_once(plans):
    rng = random.Random(0)
    size = lambda hi: int(round(2 ** rng.uniform(0, hi)))                     # noqa: E731
    asked, wanted = [], []
    for _ in range(4000):
        backward, N = rng.random() < 0.5, size(17)
        if rng.random() < 0.5:
            d, H, nm = rng.choice([64, 128]), rng.randint(1, 140), rng.choice(NORMS)
            H = min(H, 8192 // d) if nm == "token" else H
            B = min(size(10), 65535 // H)
            backward = backward and nm != "none"
            asked.append(rope(B, H, N, d, nm, rng.random() < 0.5, 2, backward))
            wanted.append((N, None, B, backward, H, d))
        else:
            C, B = 8 * rng.randint(1, 1024), size(16) - 1 or 1
            asked.append(norm(B, N, C, rng.choice(list(PARTS)), rng.choice(MODS), backward, rng.choice([None, C + 8, (1 << 26) + 8, (1 << 33) + 8])))
            wanted.append((N, C // 8, B, backward, 0, 0))
    for line, p, (N, chunks, B, backward, H, d) in zip(asked, plans(asked), wanted):
        try:
            if H:
                assert p.groups * p.heads >= H and (p.groups - 1) * p.heads < H and p.heads * d <= 8192
                chunks = p.heads * d // 8
            check(p, N, chunks, B * p.groups, 1 if backward else 3, 1024 if backward else 512)
        except AssertionError as e:
            raise AssertionError((line, p)) from e


def test_results_that_stay_in_the_memory_side_cache(plans):
    """Those of a call that come to 256 MB or less: of q and k, or of q alone."""
    for bf16, esz in ((True, 2), (False, 4)):
        for B, H, d in ((1, 12, 128), (2, 20, 64)):
            fits = (256 << 20) // (B * H * d * esz)                          # tokens of one tensor
            for tensors in (1, 2):
                n = fits // tensors
                got = plans([rope(B, H, n, d, "token", bf16, tensors), rope(B, H, n + 1, d, "token", bf16, tensors),
                             rope(B, H, n, d, "token", bf16, tensors, backward=True)])
                assert [p.cached for p in got] == [1, 0, 0], (bf16, B, H, d, tensors)


def test_sizes_of_the_gpu_tests_go_round_the_loop(plans):
    """Of tests/test_gpu_row_loop.py: at least two steps both ways, and for each kernel one size with three and a last one that is not full."""
    from test_gpu_row_loop import FORMS, NORM, ROPE, WAYS
    for backward in (False, True):
        for nm, _, dtype in WAYS:
            sizes = [s for s in ROPE if nm != "token" or s[1] * s[3] <= 8192]
            got = plans([rope(*s[:4], nm, dtype == "bf16", 2, backward and nm != "none") for s in sizes])
            assert all(steps(p, s[2]) >= 2 for p, s in zip(got, sizes)), (nm, backward, [(s, steps(p, s[2]), p) for p, s in zip(got, sizes)])
            ragged = [p for p, s in zip(got, sizes) if steps(p, s[2]) >= 3 and s[2] % (p.teams * p.walkers)]
            assert {p.waves > 1 for p in ragged} == {True, False}
            assert {p.walkers > 1 for p in got} == {True, False}
        for _, _, _, _, mods, part in FORMS:
            got = plans([norm(*s, part, mods, backward) for s in NORM])
            assert all(steps(p, s[1]) >= 2 for p, s in zip(got, NORM)), (part, mods, backward, [(s, steps(p, s[1]), p) for p, s in zip(got, NORM)])
            ragged = [p for p, s in zip(got, NORM) if steps(p, s[1]) >= 3 and s[1] % (p.teams * p.walkers)]
            assert {p.waves > 1 for p in ragged} >= ({True, False} if backward else {False})
            assert {p.walkers > 1 for p in got} == {True, False}
