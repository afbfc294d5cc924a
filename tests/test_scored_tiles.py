"""csrc/scored_tiles.h, the arithmetic by which attention of prompts with formed scores numbers its tiles, compiled for the host: every tile of every sequence has
a workgroup, in batches of fewer tokens than sequences too."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

NUMBERING = r"""
#include <cstdio>
#include <random>
#include <vector>
#include "scored_tiles.h"
using namespace eco;
// every (sequence, tile) once, found as the kernel finds it
static bool covered(const std::vector<int>& S, int G, int rows) {
  const int B = (int)S.size();
  std::vector<int> cu(B + 1, 0);
  for (int b = 0; b < B; ++b) cu[b + 1] = cu[b] + S[b];
  std::vector<std::vector<int>> seen(B);
  for (int b = 0; b < B; ++b) seen[b].assign(((int64_t)S[b] * G + rows - 1) / rows, 0);
  if (prefill_scored_first_tile(rows, G, 0, 0) != 0) return false;
  for (int b = 1; b < B; ++b)
    if (prefill_scored_first_tile(rows, G, cu[b], b) < prefill_scored_first_tile(rows, G, cu[b - 1], b - 1)) return false;
  const int64_t units = prefill_scored_tiles(rows, B, cu[B], G);
  for (int64_t unit = 0; unit < units; ++unit) {
    int b = 0;
    while (b + 1 < B && prefill_scored_first_tile(rows, G, cu[b + 1], b + 1) <= unit) ++b;
    const int64_t tile = unit - prefill_scored_first_tile(rows, G, cu[b], b);
    if (S[b] > 0 && tile * rows < (int64_t)S[b] * G) ++seen[b][tile];
  }
  for (int b = 0; b < B; ++b)
    for (int n : seen[b])
      if (n != 1) return std::printf("%d sequences, %d tokens, %d heads, tiles of %d: a tile of sequence %d has %d workgroups\n", B, cu[B], G, rows, b, n), false;
  return true;
}
int main() {
  bool ok = covered({0, 1}, 8, 128) && covered({0, 0, 5, 0, 0, 0, 1}, 8, 128) && covered({1}, 1, 128) && covered({0, 0, 0, 300}, 16, 256);
  std::vector<int> few(72, 0);
  few[60] = 1, few[71] = 4;
  ok = ok && covered(few, 4, 128);
  std::mt19937 r(1);
  for (int n = 0; ok && n < 4000; ++n) {
    std::vector<int> S(1 + r() % 140);
    const int none = r() % 101, longest = 1 + r() % (n % 3 ? 3 : 400);
    for (int& s : S) s = (int)(r() % 100) < none ? 0 : 1 + r() % longest;
    for (int rows : {128, 256}) ok = ok && covered(S, 1 + r() % 16, rows);
  }
  if (ok) std::printf("ok\n");
}
"""


def test_every_tile_has_a_workgroup(tmp_path):
    src, exe = tmp_path / "tiles.cpp", tmp_path / "tiles"
    src.write_text(NUMBERING)
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-I", os.path.join(ROOT, "paper_2504_18154_amd", "csrc"), str(src), "-o", str(exe)], check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=60)
    assert r.returncode == 0 and r.stdout == "ok\n", r.stdout
