"""Which kernel a call over shared entries takes (groups.h, compiled for the CPU), and shapes that take the
kernels of large row tiles: 64 rows (bf16, fp32) or 128 rows (bf16) a workgroup, their states joined by a launch of
its own.  The plan goes by the work, so the shapes here have packed arrays of more rows than the entries
in use, as where the arrays hold the entries of every layer."""
import functools
import os
import random
import subprocess
import tempfile

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SOURCE = r"""
#include <stdio.h>
#include "groups.h"
using namespace gkv;
int main() {
  int bf, G, per, d, B, S;
  long entries;
  while (scanf("%d %d %d %d %d %d %ld", &bf, &G, &per, &d, &B, &S, &entries) == 7) {
    const SharedPlan p = shared_plan(SharedDims{bf, G, G * per, d, per, B, S, 0}, entries);
    printf("%s %d\n", p.few ? "few" : "many", p.waves);
  }
  return 0;
}
"""


@functools.lru_cache(maxsize=None)
def _program():
    folder = tempfile.mkdtemp()
    src, exe = os.path.join(folder, "plan.cpp"), os.path.join(folder, "plan")
    with open(src, "w") as f:
        f.write(SOURCE)
    subprocess.run(["g++", "-O1", "-std=c++17", "-Wall", "-Werror", "-I", os.path.join(ROOT, "paper_2608_07001_amd", "csrc"), src, "-o", exe],
                   check=True)
    return exe


@functools.lru_cache(maxsize=None)
def kernel(dtype, d, G, H, n_seq, n_group, rows):
    """("few" or "many", waves of a workgroup) for packed arrays of so many rows."""
    text = f"{int(dtype == 'bf16')} {G} {H // G} {d} {n_seq} {n_group} {rows}"
    kind, waves = subprocess.run([_program()], input=text, capture_output=True, text=True, check=True).stdout.split()
    return kind, int(waves)


PAD = 10300                     # rows of the arrays for each (group, KV head), beside those in use
KINDS = [("bf16", 64, 4), ("bf16", 128, 4), ("bf16", 64, 8), ("bf16", 128, 8), ("f32", 64, 4), ("f32", 128, 4)]      # type, d, waves


def _counts(r, n, hi):
    return [r.randint(0, hi) for _ in range(n)]


def one_group(kind):
    """(G, H, groups): rows that fill no tile, one and several, of KV heads with 1, 3 and more query heads."""
    return {("bf16", 4): [(1, 1, [17]), (2, 6, [21]), (1, 16, [4])], ("bf16", 8): [(1, 1, [65]), (2, 14, [20]), (1, 4, [64])],
            ("f32", 4): [(1, 1, [33]), (2, 6, [21]), (1, 4, [32])]}[kind[0], kind[2]]


def several_groups(kind):
    """(G, H, groups, counts): groups of no sequence and of one among larger ones; no entries, one, part of a tile."""
    groups = [70, 0, 31, 1, 160] if kind[2] == 8 else [20, 0, 31, 1, 60, 9] if kind[0] == "bf16" else [40, 0, 31, 1, 60, 9]
    counts = _counts(random.Random(len(groups)), 2 * len(groups), 300)
    counts[:4], counts[5], counts[-1] = [700, 0, 5, 1], 128, 129
    return 2, 4, groups, counts


def deep(kind):
    """(G, H, groups, counts): as many row tiles as leave each a chunk of several key tiles."""
    r = random.Random(kind[2])
    S = 40 if kind[2] == 8 else 60
    lo, hi = {("bf16", 4): (5, 20), ("bf16", 8): (25, 60), ("f32", 4): (10, 40)}[kind[0], kind[2]]
    return 1, 3, [r.randint(lo, hi) for _ in range(S)], [r.randint(500, 1000) for _ in range(S)]


def many_units(kind):
    """(G, H, groups, counts): more (group, KV head) than a wave looks at in one round, a long one first, between and last."""
    r = random.Random(kind[1] + kind[2])
    S, G, hi = {("bf16", 4): (40, 2, 25), ("bf16", 8): (24, 3, 100), ("f32", 4): (33, 2, 50)}[kind[0], kind[2]]
    groups = [r.choice([0, r.randint(1, hi), hi, hi]) for _ in range(S)]
    groups[0], groups[-1] = hi, hi // 2
    counts = _counts(r, S * G, 400)
    counts[0], counts[S * G // 2], counts[-1] = 5000, 2600, 3001
    return G, 2 * G, groups, counts


def descending(kind):
    """(G, H, groups) of which a test gives all sequences to every second group, up to 64 units and more."""
    B = {("bf16", 4): 300, ("bf16", 8): 600, ("f32", 4): 400}[kind[0], kind[2]]
    return [(3, 12, [B] + [0] * (n - 1)) for n in (21, 25)]


def shapes(kind):
    """Every (G, H, groups) above."""
    return one_group(kind) + descending(kind) + [f(kind)[:3] for f in (several_groups, deep, many_units)]


def rows_of(G, groups, counts):
    """Rows of the packed arrays that the tests of a shape have."""
    return sum(counts) + 3 + PAD * G * len(groups)
