"""The rules by which the 8-bit paged attention cuts its work (csrc/pieces.hpp), compiled for the host as the kernels have them: no more pieces than the workspace and the grid are planned for, every
piece somebody's, quotients by a reciprocal exact."""
import os
import random
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_1911_02150_amd", "libmqa_decode.so")
CXX = os.environ.get("CXX", "g++")
pytestmark = [pytest.mark.skipif(not os.path.exists(LIB), reason="library not built (run __graft_entry__.build())"),
              pytest.mark.skipif(shutil.which(CXX) is None, reason="no compiler for the host")]

PROGRAM = r"""
#include "pieces.hpp"
#include <cstdio>
#include <vector>
using namespace mqa;

int quotients() {                    // wrong ones
  int wrong = 0;
  for (int per = 4; per <= (1 << 20); per += per < 4096 ? 4 : per / 1024 * 4) {
    const PiecesOf pieces = PiecesOf::cut(per);
    for (int tiles = 0; tiles < (1 << 19) + 1; tiles += tiles < 3000 ? 1 : 61) wrong += pieces(tiles) != pieces_of(tiles, per);
    for (long long x = per; x < (1 << 19) + 1; x += per)
      for (int d = -1; d <= 1; ++d) wrong += pieces((int)x + d) != pieces_of((int)x + d, per);
  }
  return wrong;
}

int main() {
  std::printf("%d\n", quotients());
  int b, heads, blocks;
  while (std::scanf("%d %d %d", &b, &heads, &blocks) == 3) {
    std::vector<int> tiles(b);
    int sum = 0, longest = 0;
    for (int& t : tiles) {
      if (std::scanf("%d", &t) != 1) return 1;
      sum += t;
      longest = t > longest ? t : longest;
    }
    const int total = sum * heads;
    PiecesOf pieces;
    int all;
    auto cut = [&](int into) {
      pieces = PiecesOf::cut(into);
      all = 0;
      for (int t : tiles) all += pieces(t);
      return all;
    };
    if (b > 1024) {
      std::printf("%d 1\n", cut(listed_share(blocks, longest, total)) * heads);
      continue;
    }
    scaled_cut(b, heads, blocks, longest, total, cut);
    const int per = pieces.per;
    unsigned long long whole = 0;
    std::vector<unsigned long long> before(b);
    for (int i = 0; i < b; ++i) {
      before[i] = whole;
      whole += (unsigned long long)pieces(tiles[i]) << (16 * quarter_of(tiles[i], pieces(tiles[i]), per));
    }
    std::vector<int> taken(all, 0);
    bool once = true;
    for (int i = 0; i < b; ++i) {
      const int n = pieces(tiles[i]), first = (int)((before[i] + quarters_before(whole)) >> (16 * quarter_of(tiles[i], n, per)) & 0xffff);
      for (int x = first; x < first + n; ++x) once = once && x < all && taken[x]++ == 0;
    }
    std::printf("%d %d\n", all * heads, once ? 1 : 0);
  }
}
"""

UNITS = 256


def block_rows(groups, R, tiles, wide):
    little = groups * tiles * R * (4 if wide > 128 else 2) <= 3 << 16 and groups * (-(-R // 16)) <= (3 if wide <= 64 else 2) * UNITS
    return 16 if R <= 16 or little else 32


LENGTHS = [lambda r, t: t, lambda r, t: r.randint(0, t), lambda r, t: r.choice([0, 1, t, r.randint(0, t)]), lambda r, t: r.choice([t, 1]), lambda r, t: min(t, int(t * r.random() ** 6))]


def test_the_cut_that_the_kernels_make(tmp_path):
    import paper_1911_02150_amd as m
    source, program = tmp_path / "cut.cpp", tmp_path / "cut"
    source.write_text(PROGRAM)
    subprocess.run([CXX, "-O2", "-std=c++17", "-D__host__=", "-D__device__=", "-I", os.path.join(ROOT, "paper_1911_02150_amd", "csrc"), str(source), "-o", str(program)], check=True)
    r, cases, lines = random.Random(5), [], []
    while len(cases) < 6000:
        b = r.choice([1, 2, r.randint(1, 64), r.randint(1, 300), r.randint(1, 80), r.randint(1, 1100)])
        h_kv, R = r.choice([1, 1, 2, 4, 8, r.randint(1, 70)]), r.choice([1, 4, 8, 16, 32, 64, r.randint(1, 600), r.randint(1, 1024)])
        tiles, k = r.choice([r.randint(1, 40), r.randint(13, 300), r.randint(1, 2000), r.randint(1, 1 << 19)]), r.choice([32, 64, 128, 256])
        room = m.mqa_paged_scaled_decode_workspace_bytes(b, 1, R * h_kv, h_kv, 32, tiles, k, k, m.MQA_INT8)
        if not room:                         # (whole groups, or too large a call)
            continue
        lengths = r.choice(LENGTHS)
        cases.append((b, h_kv, R, tiles, k, room))
        lines.append(" ".join(map(str, [b, h_kv, -(-R // block_rows(b * h_kv, R, tiles, k)), *(lengths(r, tiles) for _ in range(b))])))
    out = subprocess.run([str(program)], input="\n".join(lines), capture_output=True, text=True, check=True).stdout.split("\n")
    assert out[0] == "0" and len(out) == len(cases) + 2      # (the last line's end)
    for (b, h_kv, R, tiles, k, room), got in zip(cases, out[1:]):
        n, once = map(int, got.split())
        assert once, (b, h_kv, R, tiles, k)
        assert n * R * (k + 2) * 4 + b * h_kv * 8 <= room, (b, h_kv, R, tiles, k, n)
        assert n <= b * h_kv + 768 and (b <= 1024 or n // h_kv <= b + 768)      # the grid; the list
