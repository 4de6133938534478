"""Attention over quantised pages with eight waves a workgroup: which calls take it, and that their chunks run at once
(the kernels' arithmetic, compiled for the CPU)."""
import os
import random
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SOURCE = r"""
#include <stdio.h>
#include <algorithm>
#include <vector>
#include "pages.h"
using namespace gkv;
// a line: n_seq, KV heads, query heads of each, d, table width in pages of 16, then a length a sequence
int main() {
  int n, G, per, d, width;
  while (scanf("%d %d %d %d %d", &n, &G, &per, &d, &width) == 5) {
    std::vector<int> len(n);
    for (auto& x : len) if (scanf("%d", &x) != 1) return 1;
    PageDims p{1, G, G * per, d, per, n, 4, width, 1000, 0};
    const int R = n * G;
    long long chunks = 0;
    const bool eight = eight_waves(p);
    if (eight) {                                       // as launch_quant_paged and find_chunk have it: pairs of 32 tokens' tiles
      const int room = (int)std::min<int64_t>(chunk_room(p, 0, 64), PA_CUS - R / 2);
      const float join = join_cost(per, d) / 2;
      uint64_t total = 0;
      for (int x : len) total += (uint64_t)tiles_of<64>(x, 0) * G;
      auto count = [&](int size) {
        long long c = 0;
        for (int x : len) c += (long long)chunks_of(tiles_of<64>(x, 0), size, join) * G;
        return c;
      };
      int size = chunk_tiles(total, room);
      size = one_round(total, R, size, n > 64 ? R + room : count(size));
      chunks = count(size);
      if (room < 1 || size < PA_MIN) chunks = -1;
    }
    printf("%d %lld\n", eight, chunks);
  }
  return 0;
}
"""


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    folder = tmp_path_factory.mktemp("plan")
    (folder / "p.cpp").write_text(SOURCE)
    subprocess.run(["g++", "-O1", "-std=c++17", "-Wall", "-Werror", "-I", os.path.join(ROOT, "paper_2608_07001_amd", "csrc"),
                    str(folder / "p.cpp"), "-o", str(folder / "p")], check=True)

    def run(cases):
        text = "\n".join(" ".join(map(str, [len(lens), G, per, d, width] + lens)) for G, per, d, width, lens in cases)
        out = subprocess.run([str(folder / "p")], input=text, capture_output=True, text=True, check=True).stdout.split("\n")[:-1]
        assert len(out) == len(cases)
        return [tuple(int(x) for x in line.split()) for line in out]
    return run


def _case(r, n, G, per, d, top):
    lens = [top] * n if r.random() < 0.4 else [r.randint(0, top) for _ in range(n)]
    return G, per, d, max(1, -(-top // 16) * r.choice([1, 1, 8])), lens


def test_chunks_of_eight_waves_run_at_once(plan):
    r = random.Random(3)
    cases = [(8, 4, 128, 2048, [32768] * 7), (8, 4, 128, 2048, [32768] * 3), (1, 8, 128, 512, [8192] * 53), (1, 4, 128, 512, [8192] * 33)]
    for _ in range(9000):
        G = r.choice([1, 1, 2, 3, 8])
        n = r.randint(1, max(1, 255 // G))
        cases.append(_case(r, n, G, r.choice([1, 3, 4, 5, 8, 16, 20]), r.choice([64, 128]), int(2 ** r.uniform(4, 17))))
    out = plan(cases)
    taken = [(c, line) for c, line in zip(cases, out) if line[0]]
    assert all(line[0] for line in out[:4]) and len(taken) > 1000
    for c, (_, chunks) in taken:
        assert 0 < chunks <= 256, (c, chunks)
    assert sum(line[1] > 200 for _, line in taken) > 100                  # and they fill the chip


def test_batches_beyond_what_eight_waves_serve_take_four(plan):
    # 9 to 31 sequences of the 8 KV heads that a table lets grow long: 16 of 1 to 8192 tokens 34 us with four waves, 50 with eight
    for n in (9, 12, 16, 20, 24, 31):
        for per in (1, 4, 8):
            for d in (64, 128):
                assert plan([(8, per, d, 512, [8192] * n), (8, per, d, 64, [1024] * n)]) == [(0, 0)] * 2
    assert [x[0] for x in plan([(8, 8, 128, 48, [768] * 24), (8, 8, 128, 512, [8192] * 8), (8, 4, 128, 512, [8192] * 8), (8, 4, 128, 8, [100])])] == [1, 1, 1, 0]
