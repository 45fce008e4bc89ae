"""How the work of attention with shared prefixes is divided (no GPU): requests
and groups in one list, by the library's own division compiled for the host."""
import os
import subprocess

import numpy as np
import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2608_06557_amd", "csrc")

# Every range of a list of (length, rows' tokens; below 0 of a group, whose rows
# see all of it).  Exit 0 if each row tile is run over once from its first to its
# last token, and what is told of it is where its parts are: one range has it
# whole, or the range before the one that tells has its beginning and the next
# ones, up to the last that is told, the rest.
WALK = r"""
#include <cstdio>
#include <cstdlib>
#include <map>
#include <tuple>
#include <vector>
#include "attention_work.h"
using namespace cascade;
typedef std::tuple<int, int, int> Key;  // item, head, tile
struct Part { int w, from, to; };
#define CHECK(x) do { if (!(x)) { printf("%s at line %d\n", #x, __LINE__); return 1; } } while (0)

int main(int argc, char **argv) {
  std::vector<int> v;
  for (int i = 1; i < argc; ++i) v.push_back(atoi(argv[i]));
  const int n = v[0], heads = v[1], grid = v[2];
  const Cuts a = {v[3], v[4], v[5], v[6], v[7]};
  const int *count = &v[8], *len = count + n;
  std::vector<char> room(list_bytes(n));
  const List list(room.data(), n);
  long long total = 0;
  for (int i = 0; i < n; ++i) {
    list.before[i] = total;
    list.ids[i] = i, list.len[i] = len[i], list.count[i] = count[i];
    total += MixedSegments(len[i], count[i], a.tile_tokens).total() * heads;
  }
  list.before[n] = total;
  const int groups = ranges(a, total, grid), uncut = uncut_keys(a, total, groups);
  std::map<Key, std::vector<Part>> parts;
  std::map<Key, int> whole;
  std::map<Key, std::pair<int, int>> told;
  for (int w = 0; w < groups; ++w) {
    auto begin = [&](int k) { return locate<MixedSegments>(a, heads, list, n, uncut, cut(total, k, groups)); };
    Place at = begin(w);
    const Place end = begin(w + 1);
    if (at.key > 0) {
      const Split s = first_cut<MixedSegments>(a, list, at, begin(w ? w - 1 : 0), total, groups);
      if (s.last >= w) {
        CHECK(told.count(Key(at.item, at.head, at.tile)) == 0);
        told[Key(at.item, at.head, at.tile)] = {w, s.last};
      }
    }
    while (at.item < n) {
      const MixedSegments seg(list.len[at.item], list.count[at.item], a.tile_tokens);
      CHECK(at.tile < seg.tiles() && at.head < heads);
      const int length = (int)seg.length(at.tile);
      const bool last = end.item == at.item && end.head == at.head && end.tile == at.tile;
      const int stop = last ? end.key : length;
      if (last && stop == at.key) break;
      CHECK(at.key <= stop && stop <= length);
      const Key key(at.item, at.head, at.tile);
      if (at.key == 0 && stop == length) ++whole[key];
      else parts[key].push_back(Part{w, at.key, stop});
      if (last) break;
      at.key = 0;
      if (++at.tile == seg.tiles()) {
        at.tile = 0;
        if (++at.head == heads) at.head = 0, ++at.item;
      }
    }
  }
  for (int i = 0; i < n; ++i) {
    const MixedSegments seg(list.len[i], list.count[i], a.tile_tokens);
    const int rows = abs(list.count[i]);
    CHECK(seg.tiles() == (rows + a.tile_tokens - 1) / a.tile_tokens);
    for (int t = 0; t < seg.tiles(); ++t) {
      long long sees = list.len[i];
      if (list.count[i] > 0) sees += least((t + 1) * a.tile_tokens, rows) - rows;
      CHECK(seg.length(t) == (sees < 0 ? 0 : sees));
      for (int h = 0; h < heads; ++h) {
        const Key key(i, h, t);
        const auto &p = parts[key];
        CHECK(whole[key] == (p.empty() ? 1 : 0));
        CHECK(told.count(key) == (p.empty() ? 0u : 1u));
        if (p.empty()) continue;
        CHECK(p.size() >= 2 && told[key].first == p[1].w && told[key].second == p.back().w);
        CHECK(p.front().from == 0 && p.back().to == seg.length(t));
        for (size_t j = 1; j < p.size(); ++j) CHECK(p[j].from == p[j - 1].to && p[j].w == p[j - 1].w + 1);
        for (const Part &x : p) CHECK(x.from < x.to && x.from % a.cut_keys == 0);
      }
    }
  }
  return 0;
}
"""

# tile rows, least, most uncut tokens, step, least of a range, workgroups
RULES = {"tiles": (256, 128, 2048, 64, 128, 256), "half-tiles": (128, 128, 2048, 64, 128, 512),
         "tiles256": (128, 128, 2048, 32, 128, 256), "few": (16, 512, 512, 32, 256, 1024),
         "few-short": (32, 1024, 1024, 32, 256, 512)}


@pytest.fixture(scope="module")
def walk(tmp_path_factory):
    d = tmp_path_factory.mktemp("work")
    (d / "walk.cpp").write_text(WALK)
    exe = str(d / "walk")
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-I", CSRC, str(d / "walk.cpp"), "-o", exe], check=True)

    def run(rule, counts, lengths, heads=1, group=1):
        rows, *cuts, grid = RULES[rule]
        args = [len(counts), heads, grid, max(rows // group, 1), *cuts, *counts, *lengths]
        out = subprocess.run([exe, *map(str, args)], capture_output=True, text=True)
        assert out.returncode == 0, (rule, heads, group, out.stdout, list(counts)[:8], list(lengths)[:8])

    return run


@pytest.mark.parametrize("rule", list(RULES))
def test_every_row_tile_is_told_once(walk, rule):
    rng = np.random.default_rng(1)
    for i in range(60):
        n = int(rng.integers(1, 40))
        counts = rng.integers(1, 700 if "tiles" in rule else 9, n)
        lengths = counts + np.exp(rng.uniform(0, 9 if i % 2 else 4, n)).astype(int)
        counts = np.where(rng.random(n) < 0.4, -counts, counts)
        walk(rule, counts, lengths, int(rng.integers(1, 9)), int(rng.choice([1, 3, 8])))
    walk(rule, [1, -1], [1, 16])
    walk(rule, [-128, *[1] * 128], [8192, *range(1, 129)], 8, 8)
    walk(rule, [-5000], [16])
    walk(rule, [-5, 3], [1 << 30, 1 << 29])
    walk(rule, [2000, -40, 1], [100, 160, 0], 2, 4)  # rows that see nothing beside a group's
