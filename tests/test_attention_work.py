"""How attention's work is divided (no GPU): the library's own division,
compiled for the host, walked as the kernels walk it."""
import os
import subprocess

import numpy as np
import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2608_06557_amd", "csrc")

# Every range of a batch, segment by segment.  Exit 0 if each row tile is run
# over once from its first to its last token, and is either written whole by
# one range or has all of its parts joined.
WALK = r"""
#include <cstdio>
#include <cstdlib>
#include <map>
#include <tuple>
#include <vector>
#include "attention_work.h"
using namespace cascade;
typedef std::tuple<int, int, int> Key;  // request, head, tile
struct Part { int w, from, to; };
#define CHECK(x) do { if (!(x)) { printf("%s at line %d\n", #x, __LINE__); return 1; } } while (0)

int main(int argc, char **argv) {
  std::vector<int> v;
  for (int i = 1; i < argc; ++i) v.push_back(atoi(argv[i]));
  const int n = v[0], heads = v[1], block = v[2], grid = v[3];
  const Cuts a = {v[4], v[5], v[6], v[7], v[8]};
  const int *count = &v[9], *len = count + n;
  long long table = 0;
  std::vector<char> room(list_bytes(n));
  const List list(room.data(), n);
  long long total = 0;
  int items = 0;
  for (int i = 0; i < n; ++i) {
    table += (len[i] + block - 1) / block * block;
    if (!count[i]) continue;
    list.before[items] = total;
    list.ids[items] = i, list.len[items] = len[i], list.count[items] = count[i];
    total += Segments(len[i], count[i], a.tile_tokens).total() * heads;
    ++items;
  }
  list.before[items] = total;
  const bool joins = table > a.least_keys;  // what the host decides a launch by
  const int groups = ranges(a, total, grid), uncut = uncut_keys(a, total, groups);
  std::map<Key, std::vector<Part>> parts;
  std::map<Key, int> whole;
  std::map<Key, std::pair<int, int>> joined;  // first and last range of a cut
  for (int w = 0; w < groups && items; ++w) {
    auto begin = [&](int k) { return locate(a, heads, list, items, uncut, cut(total, k, groups)); };
    Place at = begin(w);
    const Place end = begin(w + 1);
    const Split s = first_cut(a, list, at, begin(w ? w - 1 : 0), total, groups);
    if (s.request >= 0) {
      CHECK(joined.count(Key(s.request, s.head, s.tile)) == 0);
      joined[Key(s.request, s.head, s.tile)] = {w - 1, s.last};
    }
    while (at.item < items) {
      const Segments seg(list.len[at.item], list.count[at.item], a.tile_tokens);
      CHECK(at.tile < seg.tiles() && at.head < heads);
      const int length = (int)seg.length(at.tile);
      const bool last = end.item == at.item && end.head == at.head && end.tile == at.tile;
      const int stop = last ? end.key : length;
      if (last && stop == at.key) break;
      CHECK(at.key <= stop && stop <= length);
      const Key key(list.ids[at.item], at.head, at.tile);
      // the look-ups of few rows (8 waves, 32 tokens each, two steps ahead) and of
      // row tiles (a sub-block to a wave, two stages ahead), made where there are tokens
      const int blocks = (list.len[at.item] + block - 1) / block;
      if (at.key < stop) {
        const SubBlocks subs(__builtin_ctz(block), stop);
        for (int k = at.key; k <= stop + 3 * 256; k += 16) {
          CHECK(subs.entry(k >> 4) >= 0 && subs.entry(k >> 4) < blocks);
          CHECK(subs.within(k >> 4) >= 0 && subs.within(k >> 4) < block / 16);
        }
        CHECK(subs.entry((stop - 1) >> 4) == (stop - 1) / block);
      } else {
        CHECK(stop == 0 && SubBlocks(__builtin_ctz(block), stop).entry(0) < 0);  // not to be looked up
      }
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
  for (int i = 0; i < items; ++i) {
    const Segments seg(list.len[i], list.count[i], a.tile_tokens);
    CHECK(list.before[i] + heads * seg.total() == list.before[i + 1]);
    long long sum = 0;
    for (int t = 0; t < seg.tiles(); ++t) {
      CHECK(seg.start(t) == sum);
      // the tile's last row is its token min((t + 1) per, count) - 1
      long long sees = (long long)list.len[i] - list.count[i] + least((t + 1) * a.tile_tokens, list.count[i]);
      if (sees < 0) sees = 0;
      CHECK(seg.length(t) == sees && sees <= table);
      sum += sees + kFixedKeys;
      for (int h = 0; h < heads; ++h) {
        const Key key(list.ids[i], h, t);
        const auto &p = parts[key];
        CHECK(whole[key] == (p.empty() ? 1 : 0));
        CHECK(joined.count(key) == (p.empty() ? 0u : 1u));
        if (p.empty()) continue;
        CHECK(joins);
        CHECK(p.size() >= 2 && joined[key].first == p.front().w && joined[key].second == p.back().w);
        CHECK(p.front().from == 0 && p.back().to == seg.length(t));
        for (size_t j = 1; j < p.size(); ++j) CHECK(p[j].from == p[j - 1].to && p[j].w == p[j - 1].w + 1);
        for (const Part &x : p) CHECK(x.from < x.to && x.from % a.cut_keys == 0);
      }
    }
  }
  return 0;
}
"""

# row tiles of dims up to 128 and of 256, and few rows of long and short tables:
# tile rows, least, most uncut tokens, step, least of a range, workgroups
RULES = {"tiles": (256, 1024, 2048, 64, 256, 256), "tiles256": (128, 512, 2048, 32, 256, 256),
         "few": (16, 512, 512, 32, 256, 1024), "few-short": (64, 1024, 1024, 32, 256, 1024)}


@pytest.fixture(scope="module")
def walk(tmp_path_factory):
    d = tmp_path_factory.mktemp("work")
    (d / "walk.cpp").write_text(WALK)
    exe = str(d / "walk")
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-I", CSRC, str(d / "walk.cpp"), "-o", exe], check=True)

    def run(rule, counts, lengths, heads=1, group=1, block=16):
        rows, *cuts, grid = RULES[rule]
        args = [len(counts), heads, block, grid, max(rows // group, 1), *cuts, *counts, *lengths]
        out = subprocess.run([exe, *map(str, args)], capture_output=True, text=True)
        assert out.returncode == 0, (rule, heads, group, out.stdout, list(counts)[:8], list(lengths)[:8])

    return run


@pytest.mark.parametrize("rule", list(RULES))
def test_every_row_tile_is_written_once(walk, rule):
    rng = np.random.default_rng(1)
    for i in range(60):
        n = int(rng.integers(1, 40))
        counts = rng.integers(0, 700 if "tiles" in rule else 9, n)
        lengths = counts + np.exp(rng.uniform(0, 9 if i % 2 else 4, n)).astype(int)
        walk(rule, counts, lengths, int(rng.integers(1, 9)), int(rng.choice([1, 3, 8])))
    walk(rule, [1], [1])
    walk(rule, [1], [1 << 30])
    walk(rule, [8192], [131072], 8, 8)


@pytest.mark.parametrize("rule", list(RULES))
def test_more_new_tokens_than_cached_ones(walk, rule):
    """Rows that see nothing have no length, and no segment is longer than the
    table, so that what is cut is joined."""
    for count, length in ((2000, 100), (2000, 0), (9000, 1), (700, 699), (256, 0), (5000, 1100), (5000, 3000)):
        for heads in (1, 8):
            for group in (1, 4):
                walk(rule, [count], [length], heads, group)
                walk(rule, [3, count, 1], [0, length, 40], heads, group, 32)


@pytest.mark.parametrize("rule", list(RULES))
def test_nothing_is_looked_up_where_nothing_is_seen(walk, rule):
    """Batches of requests without cached tokens, the first one among them,
    with and without a table."""
    for block in (16, 128):
        walk(rule, [1], [0], 8, 8, block)
        walk(rule, [64], [0], 2, 1, block)
        walk(rule, [5, 1, 2], [0, 0, 0], 2, 4, block)
        walk(rule, [5, 1, 70], [0, 17, 30], 2, 4, block)
