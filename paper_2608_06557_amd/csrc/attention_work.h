// attention_work.h -- how attention's work is divided among workgroups: whole
// numbers only, the same on the GPU and, for checks, on the host.  Internal to
// the library.
#pragma once

#ifdef __HIPCC__
#include <hip/hip_runtime.h>
#define CASCADE_WORK_FN __host__ __device__ __forceinline__
#else
#define CASCADE_WORK_FN inline
#endif

namespace cascade {

// What a segment costs besides its tokens (its queries, first loads and
// output), in tokens.  128 decode rows over caches up to 8192 tokens: 56 us,
// without it 65; 128 to 512 are alike.  A 32 Ki token prefill in chunks: 1.87
// ms, without it 1.98.
constexpr int kFixedKeys = 256;

// Where a kernel's segments may be cut.
struct Cuts {
  int tile_tokens;  // tokens of one row tile
  // segments up to twice a workgroup's share are not cut, within these bounds
  int least_keys, atomic_keys;
  int cut_keys;     // cuts are at multiples of this power of two, the tokens of a step
  int range_keys;   // least tokens of one workgroup, at least two steps
};

// A cut segment: request, KV head, row tile, last workgroup with a part of it.
struct Split {
  int request, head, tile, last;
};

template <typename T>
CASCADE_WORK_FN T least(T a, T b) { return b < a ? b : a; }
template <typename T>
CASCADE_WORK_FN T most(T a, T b) { return a < b ? b : a; }

// The segments of one request and KV head: row tiles, each as long as its last
// row sees tokens.  With more new tokens than cached ones the first rows see
// none, so no segment is longer than the cache.
struct Segments {
  long long shown;  // cached tokens that every row sees; below 0 the first -shown rows see none
  int count, per;
  CASCADE_WORK_FN Segments(int len, int count, int tile_tokens)
      : shown((long long)len - count), count(count), per(tile_tokens) {}
  CASCADE_WORK_FN int tiles() const { return (count + per - 1) / per; }
  // tokens that row tile t runs over
  CASCADE_WORK_FN long long length(int t) const {
    return most(shown + least((long long)(t + 1) * per, (long long)count), 0ll);
  }
  // the costs of the tiles before t
  CASCADE_WORK_FN long long start(int t) const {
    return t * (shown + kFixedKeys) + (long long)per * ((long long)t * (t + 1) / 2) + (shown < 0 ? unseen(t) : 0);
  }
  CASCADE_WORK_FN long long total() const {
    const int t = tiles() - 1;
    return start(t) + length(t) + kFixedKeys;
  }

 private:
  // by how much the tiles before t that see nothing bring the sum of shown + (t + 1) per below 0
  CASCADE_WORK_FN long long unseen(int t) const {
    const long long z = least((int)-shown / per, t);
    return -z * shown - per * (z * (z + 1) / 2);
  }
};

// The same, or with a negative count those of rows that all see every token.
struct MixedSegments {
  Segments causal;
  bool even;
  long long len;
  CASCADE_WORK_FN MixedSegments(int len, int count, int tile_tokens)
      : causal(len, count < 0 ? -count : count, tile_tokens), even(count < 0), len(len) {}
  CASCADE_WORK_FN int tiles() const { return causal.tiles(); }
  CASCADE_WORK_FN long long length(int t) const { return even ? len : causal.length(t); }
  CASCADE_WORK_FN long long start(int t) const { return even ? t * (len + kFixedKeys) : causal.start(t); }
  CASCADE_WORK_FN long long total() const { return even ? start(tiles()) : causal.total(); }
};

// floor(a / b) of whole numbers 0 <= a < 2^52, 0 < b: by doubles, whose
// quotient is off by one at most
CASCADE_WORK_FN long long quotient(long long a, long long b) {
  long long q = (long long)((double)a / (double)b);
  const long long r = a - q * b;
  return r < 0 ? q - 1 : r >= b ? q + 1 : q;
}

struct Place {
  int item, head, tile, key;
};

// The list of requests with rows of a kernel's kind, in LDS.
struct List {
  long long *before;  // cost before each, and of all
  int *ids, *len, *count;
  CASCADE_WORK_FN List(char *lds, int n)
      : before(reinterpret_cast<long long *>(lds)), ids(reinterpret_cast<int *>(before + n + 1)), len(ids + n),
        count(len + n) {}
};
#ifdef __HIPCC__
__host__ __device__
#endif
constexpr int list_bytes(int n) { return (20 * n + 8 + 15) & ~15; }

// Where the range of cost `c` begins: a segment and a token of it.
template <typename S = Segments>
CASCADE_WORK_FN Place locate(const Cuts &a, int kv_heads, const List &list, int n, int atomic_keys, long long c) {
  Place p = {n, 0, 0, 0};
  if (n == 0 || c >= list.before[n]) return p;
  int lo = 0, hi = n;  // before[lo] <= c < before[hi]
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (list.before[mid] <= c) lo = mid; else hi = mid;
  }
  p.item = lo;
  const S s(list.len[lo], list.count[lo], a.tile_tokens);
  const long long per_head = s.total();
  long long left = c - list.before[lo];
  p.head = (int)quotient(left, per_head);
  left -= p.head * per_head;
  const int tiles = s.tiles();
  int t0 = 0, t1 = tiles;  // start(t0) <= left < start(t1)
  while (t1 - t0 > 1) {
    const int mid = (t0 + t1) >> 1;
    if (s.start(mid) <= left) t0 = mid; else t1 = mid;
  }
  p.tile = t0;
  left -= s.start(t0);
  const long long length = s.length(t0);
  if (length > atomic_keys) {
    p.key = (int)most(left - kFixedKeys, 0ll) & -a.cut_keys;
  } else if (2 * left >= length + kFixedKeys) {  // not cut: the nearer end
    p.tile = t0 + 1;
    if (p.tile == tiles) {
      p.tile = 0;
      if (++p.head == kv_heads) {
        p.head = 0;
        ++p.item;
      }
    }
  }
  return p;
}

// Where range w of `groups` begins: total w / groups, rounded down in two steps
// whose products stay small.
CASCADE_WORK_FN long long cut(long long total, int w, int groups) {
  const long long whole = quotient(total, groups);
  return whole * w + (unsigned)((unsigned)(total - whole * groups) * (unsigned)w) / (unsigned)groups;
}

// How many of `grid` workgroups take a range of work of cost `total`.
CASCADE_WORK_FN int ranges(const Cuts &a, long long total, int grid) {
  const int cap = (int)least((long long)grid, quotient(total, a.range_keys));
  return cap >= 8 ? cap & ~7 : most(cap, 1);
}
// The longest segment that they leave whole.
CASCADE_WORK_FN int uncut_keys(const Cuts &a, long long total, int groups) {
  const long long share = least(quotient(total, groups), (long long)a.atomic_keys);
  return least(most(2 * (int)share, a.least_keys), a.atomic_keys);
}

// The segment that range w, which begins at `at`, is the first to cut, the
// range before beginning at `prev`; request -1 if there is none.
template <typename S = Segments>
CASCADE_WORK_FN Split first_cut(const Cuts &a, const List &list, const Place &at, const Place &prev, long long total,
                                int groups) {
  const bool inside = at.key > 0 && !(prev.key > 0 && prev.item == at.item && prev.head == at.head &&
                                      prev.tile == at.tile);
  if (!inside) return Split{-1, 0, 0, 0};
  const S seg(list.len[at.item], list.count[at.item], a.tile_tokens);
  const long long stop = list.before[at.item] + at.head * seg.total() + seg.start(at.tile) +
                         seg.length(at.tile) + kFixedKeys;
  // the last range that begins before `stop`
  int end = least((int)quotient(stop, most(quotient(total, groups), 1ll)) + 1, groups - 1);
  while (cut(total, end, groups) >= stop) --end;
  return Split{list.ids[at.item], at.head, at.tile, end};
}

// The sub-blocks (16 tokens) of a request's tokens before `end`, which is above
// 0: a segment that sees nothing has none, and its request may have no blocks.
struct SubBlocks {
  int shift, last;  // log2 of sub-blocks a block, last sub-block
  CASCADE_WORK_FN SubBlocks(int block_shift, int end) : shift(block_shift - 4), last((end - 1) >> 4) {}
  // table entry of sub-block `sub`, or of the last one, and its place in the block
  CASCADE_WORK_FN int entry(int sub) const { return least(sub, last) >> shift; }
  CASCADE_WORK_FN int within(int sub) const { return least(sub, last) & ((1 << shift) - 1); }
};

}  // namespace cascade
