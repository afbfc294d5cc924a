"""csrc/scored_tiles.h, the arithmetic by which attention of prompts with formed scores numbers its tiles and finds the blocks of their keys, compiled for the host: every tile
of every sequence has a workgroup, in batches of fewer tokens than sequences too, and no entry of the block table is read but those of blocks with a key that a row sees."""
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


BLOCKS = r"""
#include <algorithm>
#include <cstdio>
#include <random>
#include <utility>
#include <vector>
#include "scored_tiles.h"
using namespace eco;
typedef std::vector<std::pair<int, int>> Ranges;
// What the kernel reads and keeps of a tile whose rows have these ranges (no keys: 2^31 - 1, 0).
static bool right(const Ranges& given) {
  // (a row without keys stands in for the one in front of it, among its wavefront's 32, that has some, or the first one behind it)
  Ranges rows = given;
  for (size_t w = 0; w < rows.size(); w += 32) {
    const size_t end = std::min(w + 32, rows.size());
    for (size_t i = w + 1; i < end; ++i)
      if (rows[i].second == 0) rows[i] = rows[i - 1];
    for (size_t i = end - 1; i > w; --i)
      if (rows[i - 1].second == 0) rows[i - 1] = rows[i];
  }
  bool gaps = false;
  int lo = 0x7fffffff, hi = 0;
  for (size_t i = 0; i < rows.size(); ++i) {
    if (i + 1 < rows.size()) gaps |= ranges_apart(rows[i].first, rows[i].second, rows[i + 1].first, rows[i + 1].second);
    lo = std::min(lo, rows[i].first), hi = std::max(hi, rows[i].second);
  }
  if (hi == 0) return true;
  std::vector<char> sees(hi + 64, 0);
  for (const auto& r : given)
    for (int k = r.first; k < r.second; ++k) sees[k] = 1;
  for (int j = lo / 64; j <= (hi - 1) / 64; ++j) {
    uint64_t seen = 0;
    if (gaps)
      for (const auto& r : rows) seen |= keys_seen(r.first, r.second, j * 64);
    for (int i = 0; i < 4; ++i) {
      const int blk = 4 * j + i, at = entry_of_block(blk, lo >> 4, (hi - 1) >> 4, gaps, seen);
      if (at < 0 || std::find(sees.begin() + 16 * at, sees.begin() + 16 * at + 16, 1) == sees.begin() + 16 * at + 16) return std::printf("entry %d holds no key that is seen (block %d)\n", at, blk), false;
      const uint32_t slots = (uint32_t)(gaps ? seen >> (16 * i) : keys_seen(lo, hi, 16 * blk)) & 0xffffu;
      for (int s = 0; s < 16; ++s) {
        if ((slots >> s & 1) != (uint32_t)sees[16 * blk + s]) return std::printf("key %d is %s\n", 16 * blk + s, slots >> s & 1 ? "kept" : "cleared"), false;
        if (sees[16 * blk + s] && at != blk) return std::printf("block %d is read in place of %d\n", at, blk), false;
      }
    }
  }
  return true;
}
int main() {
  const std::pair<int, int> none = {0x7fffffff, 0};
  bool ok = right({{0, 16}, {1000, 1016}}) && right({{1000, 1016}, none, {0, 5}, {9, 30}}) && right({none, {3, 4}}) && right({{0, 5}, {5, 9}, {9, 500}});
  std::mt19937 r(2);
  for (int n = 0; ok && n < 20000; ++n) {
    Ranges rows(1 + r() % 256);
    const int kind = r() % 4, most = 1 + r() % 2000, window = 1 + r() % 300, p0 = r() % 500;
    for (size_t i = 0; i < rows.size(); ++i) {
      int a = r() % most, b = a + r() % (kind == 1 ? most : 20);
      if (kind == 2) b = p0 + (int)i + 1, a = std::max(0, b - window);                     // a window
      if (kind == 3) b = p0 + (int)i + 1, a = (b - 1) / window * window;                   // documents
      rows[i] = a < b && r() % 50 != 0 ? std::make_pair(a, b) : kind < 2 || r() % 3 == 0 ? none : std::make_pair(a, b);
      if (kind < 2 && i > 0 && r() % 4) rows[i] = rows[i - 1];                             // heads of one token
    }
    ok = right(rows);
  }
  // (windows and documents alone touch)
  for (int i = 0; i < 600; ++i) ok = ok && !ranges_apart(std::max(0, i - 30), i + 1, std::max(0, i - 29), i + 2) && !ranges_apart(i / 41 * 41, i + 1, (i + 1) / 41 * 41, i + 2);
  if (ok) std::printf("ok\n");
}
"""


def test_blocks_without_a_key_that_is_seen_are_not_named(tmp_path):
    src, exe = tmp_path / "blocks.cpp", tmp_path / "blocks"
    src.write_text(BLOCKS)
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-I", os.path.join(ROOT, "paper_2504_18154_amd", "csrc"), str(src), "-o", str(exe)], check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=60)
    assert r.returncode == 0 and r.stdout == "ok\n", r.stdout
