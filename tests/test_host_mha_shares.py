"""How the gradient of attention shares out the steps of its items (csrc/mha_shares.h), compiled for the host: every
step of every shared item belongs to exactly one CTA, at sizes that no GPU run reaches too."""

import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

PROGRAM = r"""
#include <stdio.h>
#include <stdlib.h>
#include <algorithm>
#include <vector>
#include "mha_shares.h"

struct Alike {
  int64_t per;
  int64_t operator()(int slot) const { return (slot + 1) * per; }
};
struct Uneven {
  const std::vector<int64_t>* sums;
  int64_t operator()(int slot) const { return (*sums)[slot]; }
};

// The walk of every CTA, with the items' steps of its own, in 128 bits.
template <class Upto>
int check(const Upto& upto, const std::vector<int64_t>& steps, int heads, int full, int ctas) {
  const int slots = (int)steps.size();
  acid::StepShares<Upto> sh(upto, heads, slots, full, ctas, 4);
  typedef __int128 big;
  big total = 0, before = 0;
  for (int i = 0; i < slots; ++i) total += steps[i];
  for (int i = 0; i < full % slots; ++i) before += steps[i];
  const big base = big(full / slots) * total + before, end = big(heads) * total;
  if (sh.shares < 1 || sh.shares > ctas) return 1;
  if (sh.bound(0) != base || sh.bound(sh.shares) != end) return 2;
  big next = base;  // the first step that no share has taken
  for (int c = 0; c < sh.shares; ++c) {
    const big from = sh.bound(c), to = sh.bound(c + 1);
    if (from != next || to < from) return 3;
    int item;
    int64_t first;
    sh.begin(c, item, first);
    if (item < full || item >= heads * (int64_t)slots) return 4;
    big at = big(item / slots) * total;
    for (int i = 0; i < item % slots; ++i) at += steps[i];
    if (first != at) return 5;
    if (from < to && c > 0 && !(at <= from && from < at + steps[item % slots])) return 6;
    for (; at < to && item < heads * (int64_t)slots; at += steps[item++ % slots])
      next += std::max(big(0), std::min(to, at + steps[item % slots]) - std::max(from, at));
  }
  return next == end ? 0 : 7;
}

int main(int argc, char** argv) {
  // alike: rows of the stationary side, streamed rows, heads, query heads to a key head, CTAs
  const int64_t rows = atoll(argv[1]), streamed = atoll(argv[2]);
  const int heads = atoi(argv[3]), group = atoi(argv[4]), ctas = atoi(argv[5]);
  const int slots = (int)((rows + 127) / 128);
  const int64_t items = (int64_t)slots * heads;
  const int full = (int)(items < ctas ? 0 : items / ctas * ctas);
  if (full == items) return 0;  // nothing is shared out
  if (argc < 7) {
    const int64_t per = (streamed + 127) / 128 * group;
    return check(Alike{per}, std::vector<int64_t>(slots, per), heads, full, ctas);
  }
  // uneven steps, some of them none
  std::vector<int64_t> steps(slots), sums(slots);
  uint64_t x = atoll(argv[6]);
  int64_t sum = 0;
  for (int i = 0; i < slots; ++i) {
    x = x * 6364136223846793005ull + 1442695040888963407ull;
    steps[i] = (x >> 33) % 3 == 0 ? 0 : (int64_t)((x >> 33) % ((streamed + 127) / 128 + 1)) * group;
    sums[i] = sum += steps[i];
  }
  return check(Uneven{&sums}, steps, heads, 0, ctas);
}
"""


@pytest.fixture(scope="module")
def walk(tmp_path_factory):
    d = tmp_path_factory.mktemp("shares")
    src, exe = d / "shares.cpp", d / "shares"
    src.write_text(PROGRAM)
    subprocess.run(["g++", "-O2", "-std=c++17", "-I", os.path.join(ROOT, "paper_2607_12358_gb300", "csrc"), str(src), "-o",
                    str(exe)], check=True)

    def call(*args):
        return subprocess.run([str(exe), *map(str, args)], timeout=300).returncode

    return call


@pytest.mark.parametrize("ctas", [148, 152])
@pytest.mark.parametrize("rows, streamed, heads, group", [
    (400, 1500, 3, 1), (1100, 1100, 36, 1), (1, 2000, 1, 1), (600, 1500, 2, 4), (19 * 128, 4096, 8, 1),
    # a head's steps at, over and far past 2^31
    (1 << 20, 1 << 20, 1, 32), (1500000, 1500000, 1, 16), (1 << 21, 1 << 21, 1, 16), (524288, 524288, 1, 128),
    (5932800, 5932800, 1, 1), (6000000, 6000000, 12, 1), (1 << 24, 1 << 24, 3, 2)])
def test_alike_items(walk, rows, streamed, heads, group, ctas):
    assert walk(rows, streamed, heads, group, ctas) == 0


@pytest.mark.parametrize("seed", range(6))
@pytest.mark.parametrize("rows, streamed, heads, group", [
    (400, 1500, 3, 1), (600, 900, 6, 2), (151 * 128, 4096, 1, 1), (1000, 100, 4, 4), (151 * 128, 1 << 30, 1, 16)])
def test_uneven_items(walk, rows, streamed, heads, group, seed):
    assert walk(rows, streamed, heads, group, 152, seed) == 0
