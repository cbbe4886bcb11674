"""How the attention over the cache is spread over workgroups (csrc/cache_line.h), on the CPU: the header itself, compiled for the host, and the two
kernels' walks over it.  Every block of every sequence is taken once, every result is written once, and every part that is joined was written in
the same call, by a workgroup that has blocks of that sequence: whatever the table has room for, and whatever the lengths are at the time of the call."""
import os
import random
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "paper_2602_12675_amd", "csrc", "cache_line.h")

# what cache_line.h takes from common.h
COMMON = """#pragma once
#include <stddef.h>
#define __host__
#define __device__
#define __forceinline__ inline
"""
MAIN = """#include <algorithm>
#include <stdio.h>
#include <vector>
#include "cache_line.h"
using namespace sla2;

static int bad(const char* what, int B, long long room, long long heads, const std::vector<int>& len, int at) {
  printf("%s: %d sequences in tables of %lld tokens, %lld heads, at %d, lengths", what, B, room, heads, at);
  for (int n : len) printf(" %d", n);
  printf("\\n");
  return 1;
}

// The walks of cache_attention_kernel and cache_join_kernel over the sequences, for one key head
static int call(long long room, long long heads, const std::vector<int>& len) {
  const int B = (int)len.size(), most = most_parts(B, room, heads);
  std::vector<long long> first(B);
  std::vector<int> nb(B), results(B, 0);
  std::vector<std::vector<int>> taken(B);
  long long all = 0;
  for (int b = 0; b < B; b++) {
    nb[b] = (int)((std::min<long long>(std::max(len[b], 0), room) + kDecodeBlock - 1) / kDecodeBlock);
    taken[b].assign(nb[b], 0);
    first[b] = all + kOverhead;
    all = first[b] + nb[b];
  }
  if (!most) return room > 1024 ? bad("a workgroup a sequence", B, room, heads, len, 0) : 0;
  const int parts = parts_of(most, all);
  if (parts < 1 || parts > most) return bad("parts", B, room, heads, len, parts);
  std::vector<int> slot(2 * (size_t)most, -1);                 // the sequence whose part is there: the workspace has these slots
  for (int p = 0; p < parts; p++) {
    const long long x = stretch_begin(all, parts, p), y = stretch_begin(all, parts, p + 1);
    if (x >= y || (p == 0 && x != 0) || (p + 1 == parts && y != all)) return bad("stretch", B, room, heads, len, p);
    for (int b = 0; b < B; b++) {
      const long long at = first[b] - kOverhead;
      const BlockRange r = blocks_in(x, y, first[b], nb[b]);
      if (r.lo >= r.hi && !(nb[b] == 0 && at >= x && at < y)) continue;
      for (int i = r.lo; i < r.hi; i++) taken[b][i]++;
      if (r.lo > 0 || r.hi < nb[b]) {
        int& s = slot[part_slot(p, r.lo == 0)];
        if (s >= 0) return bad("slot written twice", B, room, heads, len, p);
        s = b;
      } else {
        results[b]++;
      }
    }
  }
  for (int b = 0; b < B; b++) {
    for (int n : taken[b])
      if (n != 1) return bad("block", B, room, heads, len, b);
    if (nb[b]) {
      const int p0 = part_at(all, parts, first[b]), p1 = part_at(all, parts, first[b] + nb[b] - 1);
      if (p0 != p1) {
        for (int p = p0; p <= p1; p++)
          if (p < 0 || p >= parts || slot[part_slot(p, p == p0)] != b) return bad("part that nobody wrote", B, room, heads, len, b);
        results[b]++;
      }
    }
    if (results[b] != 1) return bad("result", B, room, heads, len, b);
  }
  return 0;
}

int main() {      // per line: room, heads, step, from, to: one sequence of each of these lengths; or 0, room, heads, B, lengths
  long long room, heads;
  while (scanf("%lld", &room) == 1) {
    if (room) {
      int step, from, to;
      if (scanf("%lld %d %d %d", &heads, &step, &from, &to) != 4) return 2;
      for (int n = from; n <= to; n += step)
        if (call(room, heads, {n})) return 1;
    } else {
      int B;
      if (scanf("%lld %lld %d", &room, &heads, &B) != 3) return 2;
      std::vector<int> len(B);
      for (int& n : len)
        if (scanf("%d", &n) != 1) return 2;
      if (call(room, heads, len)) return 1;
    }
  }
  printf("done\\n");
}
"""


@pytest.fixture(scope="module")
def replay(tmp_path_factory):
    if shutil.which("g++") is None:
        pytest.skip("no C++ compiler")
    folder = tmp_path_factory.mktemp("line")
    shutil.copy(HEADER, folder / "cache_line.h")
    (folder / "common.h").write_text(COMMON)
    (folder / "main.cpp").write_text(MAIN)
    subprocess.run(["g++", "-std=c++17", "-O2", "-Wall", "-Werror", "-o", "line", "main.cpp"], cwd=folder, check=True)

    def ask(lines):
        got = subprocess.run([str(folder / "line")], input="\n".join(" ".join(map(str, x)) for x in lines) + "\n", capture_output=True, text=True, timeout=120)
        assert got.returncode == 0 and got.stdout == "done\n", got.stdout[:2000]
    return ask


@pytest.mark.parametrize("heads", [1, 4, 8, 12, 40, 300, 512, 4000])
def test_one_sequence_of_every_length(replay, heads):
    """Tables from a little more than 1,024 tokens to 131,072."""
    replay([(room, heads, 1 if room <= 8192 else 16, 0, room) for room in (1040, 2048, 8192, 32768, 75648, 131072)])


def test_sequences_that_are_short_for_their_table(replay):
    """A stream's first tokens: what is reserved is far longer than what is there."""
    replay([(0, room, heads, B) + (n,) * B for room in (2048, 8192, 16384, 32768, 131072) for heads in (1, 4, 8, 12, 40)
            for B in (1, 2, 3, 4, 5, 8, 64, 80) for n in (0, 1, 32, 33, 100, 500, 1500, 1792)])


@pytest.mark.parametrize("seed", range(4))
def test_random_lengths(replay, seed):
    rng = random.Random(seed)
    lines = []
    for _ in range(3000):
        room, B = 16 * rng.randint(65, 8192), rng.randint(1, 80)
        most = rng.choice([40, 300, 2000, room, room + 500])
        lines.append((0, room, rng.choice([1, 2, 3, 4, 8, 12, 16, 40, 97, 600]), B) + tuple(
            rng.choice([0, 1, 32, 33, rng.randint(-3, most), rng.randint(0, most), room]) for _ in range(B)))
    replay(lines)
