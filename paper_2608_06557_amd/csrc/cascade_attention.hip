// cascade_attention.hip -- attention of a ragged batch's new tokens over the
// 8-bit paged KV cache, on gfx950.
//
// For each request, KV head and tile of query rows (a row is one new token
// and one query head of the group that shares the KV head)
//   S^T = K Q^T,  P = exp2(S - m),  O^T = V^T P^T
// 32 cached tokens at a time with a running m, sum and O in registers (one
// pass, 32 bits).  Transposed, a lane owns one query row (lane % 16) and 4
// tokens of each 16 (lane / 16): its scores leave the first product exactly
// where the second wants its weights, so P never moves between lanes, and m is
// a scalar per lane.  K and V codes come straight from the cache in operand
// order, 16 bytes a lane, and are widened by the scaled FP8 conversion, which
// applies the block's power-of-two scale exactly.
//
// m follows the row's maximum only when a score exceeds it by 2^8: most tiles
// then rescale nothing and need no exchange between lanes; sums stay below
// 2^8 times a row's length.
//
// Work is the list of (request, head, row tile) segments, each as long as
// its last row sees tokens, cut into equal ranges of tokens, one per
// workgroup.  Every workgroup derives the list from the batch's lengths by
// itself (a scan), so ragged batches need neither a host plan nor another launch.  A
// segment that one workgroup covers is written at once; parts of a cut one go
// to the workspace and a second launch joins them.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <cmath>

#include "cascade.h"
#include "device_util.h"
#include "kv_format.h"

namespace cascade {
namespace {

typedef float f2 __attribute__((ext_vector_type(2)));
typedef float f4 __attribute__((ext_vector_type(4)));
typedef unsigned u2 __attribute__((ext_vector_type(2)));
typedef unsigned u4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf8 __attribute__((ext_vector_type(8)));
typedef _Float16 h2 __attribute__((ext_vector_type(2)));
typedef _Float16 h8 __attribute__((ext_vector_type(8)));

constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;
constexpr float kLowest = -3.402823466e+38f;
constexpr float kSlack = 8.f;  // a row's m lags its maximum by at most this (log2)

template <int kType> struct El;
template <> struct El<CASCADE_BF16> {
  typedef bf2 v2;
  typedef bf8 v8;
  static __device__ __forceinline__ unsigned widen_lo(unsigned w, float s) {
    return __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, s, false));
  }
  static __device__ __forceinline__ unsigned widen_hi(unsigned w, float s) {
    return __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, s, true));
  }
  static __device__ __forceinline__ f4 mfma(v8 a, v8 b, f4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
  }
};
template <> struct El<CASCADE_F16> {
  typedef h2 v2;
  typedef h8 v8;
  static __device__ __forceinline__ unsigned widen_lo(unsigned w, float s) {
    return __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, s, false));
  }
  static __device__ __forceinline__ unsigned widen_hi(unsigned w, float s) {
    return __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, s, true));
  }
  static __device__ __forceinline__ f4 mfma(v8 a, v8 b, f4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
  }
};

template <int kType>
__device__ __forceinline__ typename El<kType>::v8 widen8(unsigned lo, unsigned hi, float s0, float s1) {
  const u4 w = {El<kType>::widen_lo(lo, s0), El<kType>::widen_hi(lo, s0), El<kType>::widen_lo(hi, s1),
                El<kType>::widen_hi(hi, s1)};
  return __builtin_bit_cast(typename El<kType>::v8, w);
}
template <int kType>
__device__ __forceinline__ unsigned narrow2(float a, float b) {
  const f2 f = {a, b};
  return __builtin_bit_cast(unsigned, __builtin_convertvector(f, typename El<kType>::v2));
}

struct Rows {
  char *data;
  int64_t token_stride, head_stride;  // bytes
};

// A cut segment: request, KV head, row tile, last workgroup with a part of it.
struct Split {
  int request, head, tile, last;
};

struct Attention {
  KvView kv;
  cascade_kv_batch_t batch;
  const int32_t *row_offsets, *slots;
  Rows q, out;
  int q_heads, group;      // query heads, and those of one KV head
  float scale;             // of q.k, or of the capped score; in log2 units, >= 0
  float cap_in;            // softcap: exp2 argument per q.k
  unsigned keep, flip;     // q's bits: none where the scale was 0, turned signs where it was negative
  float *lse;              // [n_tokens][q_heads] or NULL
  float *logs;             // [sub-block][window][q_heads]: log2 of a sub-block's weight, or NULL
  int window;
  int64_t min_rows, max_rows;  // requests with min_rows < rows <= max_rows are taken
  int tile_tokens;         // tokens of one row tile
  int atomic_keys;         // segments up to this long are not cut
  int cut_keys;            // cuts are at multiples of this power of two, the tokens of a step
  int range_keys;          // least tokens of one workgroup, at least two steps
  Split *splits;           // [gridDim]
  float *parts;            // [gridDim][2][rows][kDim]
  float *part_sums;        // [gridDim][2][rows][2]: m and sum
  int32_t *status;
};

// ---------------------------------------------------------------- the work

struct Segments {  // of one request and KV head
  long long before;  // cached tokens that every row sees
  int count, per;
  __device__ __forceinline__ Segments(const KvRequest &r, int tile_tokens)
      : before(r.len > r.count ? r.len - r.count : 0), count(r.count), per(tile_tokens) {}
  __device__ __forceinline__ int tiles() const { return (count + per - 1) / per; }
  // tokens that row tile t runs over
  __device__ __forceinline__ long long length(int t) const {
    return before + min((long long)(t + 1) * per, (long long)count);
  }
  // the same summed over the tiles before t
  __device__ __forceinline__ long long start(int t) const {
    return t * before + (long long)per * ((long long)t * (t + 1) / 2);
  }
  __device__ __forceinline__ long long total() const {
    const int t = tiles() - 1;
    return start(t) + length(t);
  }
};

struct Place {
  int item, head, tile, key;
};

// Where the range of cost `c` begins: a segment and a token of it.
__device__ __forceinline__ Place locate(const Attention &a, const long long *before, const int *ids,
                                        int n, long long c) {
  Place p = {n, 0, 0, 0};
  if (n == 0 || c >= before[n]) return p;
  int lo = 0, hi = n;  // before[lo] <= c < before[hi]
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (before[mid] <= c) lo = mid; else hi = mid;
  }
  p.item = lo;
  const Segments s(kv_request(a.batch, a.row_offsets, a.kv.block_shift, ids[lo]), a.tile_tokens);
  long long left = c - before[lo];
  const long long per_head = s.total();
  p.head = (int)(left / per_head);
  left -= p.head * per_head;
  int t0 = 0, t1 = s.tiles();  // start(t0) <= left < start(t1)
  while (t1 - t0 > 1) {
    const int mid = (t0 + t1) >> 1;
    if (s.start(mid) <= left) t0 = mid; else t1 = mid;
  }
  p.tile = t0;
  left -= s.start(t0);
  const long long length = s.length(t0);
  if (length > a.atomic_keys) {
    p.key = (int)left & -a.cut_keys;
  } else if (2 * left >= length) {  // not cut: the nearer end
    p.tile = t0 + 1;
    if (p.tile == s.tiles()) {
      p.tile = 0;
      if (++p.head == a.kv.kv_heads) {
        p.head = 0;
        ++p.item;
      }
    }
  }
  return p;
}

__device__ __forceinline__ Place uniform(const Place &p, int lane) {
  return {__builtin_amdgcn_readlane(p.item, lane), __builtin_amdgcn_readlane(p.head, lane),
          __builtin_amdgcn_readlane(p.tile, lane), __builtin_amdgcn_readlane(p.key, lane)};
}

// ------------------------------------------------------------- one wave

// What a wave keeps of 16 * kTiles query rows.
template <int kType, int kDim, int kTiles, bool kCap>
struct Rowset {
  typedef typename El<kType>::v8 v8;
  v8 q[kTiles][kDim / 32];
  f4 o[kTiles][kDim / 16];
  float m[kTiles], sum[kTiles];
  int limit[kTiles];    // last cached token that the lane's row sees
  float *log_at[kTiles];  // the row's place in the log sums of sub-block 0, NULL for none

  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int t = 0; t < kTiles; ++t) {
      m[t] = kLowest;
      sum[t] = 0.f;
#pragma unroll
      for (int d = 0; d < kDim / 16; ++d) o[t][d] = f4{0.f, 0.f, 0.f, 0.f};
    }
  }

  // kB sub-blocks of 16 tokens from `key` on.  `k(b, d)` gives the operand of
  // sub-block b and dims step d, `v(b, d)` that of sub-blocks 2 b and 2 b + 1
  // and dims 16 d, with 0 for tokens past the cache's end, which may be
  // anything.  `masked`: some row does not see all of the tokens.  `after_k`
  // is called once K's operands have been taken.
  template <int kB, typename KOp, typename VOp, typename AfterK>
  __device__ __forceinline__ void step(const Attention &a, KOp k, VOp v, AfterK after_k, int key, int len,
                                       bool masked, bool logs, int64_t log_row) {
    const int lane = lane_id(), g = lane >> 4;
    f4 s[kTiles][kB];
#pragma unroll
    for (int b = 0; b < kB; ++b) {
#pragma unroll
      for (int t = 0; t < kTiles; ++t) s[t][b] = f4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int d = 0; d < kDim / 32; ++d) {
        const v8 x = k(b, d);
#pragma unroll
        for (int t = 0; t < kTiles; ++t) s[t][b] = El<kType>::mfma(x, q[t][d], s[t][b]);
      }
    }
    after_k();
    if (kCap) {
#pragma unroll
      for (int t = 0; t < kTiles; ++t)
#pragma unroll
        for (int b = 0; b < kB; ++b)
#pragma unroll
          for (int i = 0; i < 4; ++i)  // tanh(x) = 1 - 2 / (exp(2 x) + 1)
            s[t][b][i] = 1.f - 2.f * __builtin_amdgcn_rcpf(__builtin_amdgcn_exp2f(s[t][b][i] * a.cap_in) + 1.f);
    }
    if (masked) {
#pragma unroll
      for (int t = 0; t < kTiles; ++t) {
        const int seen = limit[t] - key - 4 * g;
#pragma unroll
        for (int b = 0; b < kB; ++b)
#pragma unroll
          for (int i = 0; i < 4; ++i) s[t][b][i] = 16 * b + i <= seen ? s[t][b][i] : -__builtin_inff();
      }
    }
    v8 p[kTiles][kB / 2];
#pragma unroll
    for (int t = 0; t < kTiles; ++t) {
      float top = s[t][0][0];
#pragma unroll
      for (int i = 1; i < 4 * kB; ++i) top = fmaxf(top, s[t][i >> 2][i & 3]);
      top *= a.scale;
      if (__any(top > m[t] + kSlack)) {
        top = fmaxf(top, __shfl_xor(top, 16));
        top = fmaxf(top, __shfl_xor(top, 32));
        const float now = fmaxf(m[t], top), f = __builtin_amdgcn_exp2f(m[t] - now);
        m[t] = now;
        sum[t] *= f;
#pragma unroll
        for (int d = 0; d < kDim / 16; ++d) o[t][d] *= f;
      }
      float part[kB];
#pragma unroll
      for (int b = 0; b < kB; ++b) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
          s[t][b][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[t][b][i], a.scale, -m[t]));
        part[b] = (s[t][b][0] + s[t][b][1]) + (s[t][b][2] + s[t][b][3]);
        sum[t] += part[b];
      }
#pragma unroll
      for (int b = 0; b < kB; b += 2) {
        const u4 w = {narrow2<kType>(s[t][b][0], s[t][b][1]), narrow2<kType>(s[t][b][2], s[t][b][3]),
                      narrow2<kType>(s[t][b + 1][0], s[t][b + 1][1]),
                      narrow2<kType>(s[t][b + 1][2], s[t][b + 1][3])};
        p[t][b / 2] = __builtin_bit_cast(v8, w);
      }
      if (logs) {
#pragma unroll
        for (int b = 0; b < kB; ++b) {
          float x = part[b];
          x += __shfl_xor(x, 16);
          x += __shfl_xor(x, 32);
          if (g == 0 && log_at[t] && key + 16 * b < len)
            log_at[t][(int64_t)((key >> 4) + b) * log_row] = __builtin_amdgcn_logf(x) + m[t];
        }
      }
    }
#pragma unroll
    for (int b = 0; b < kB / 2; ++b) {
#pragma unroll
      for (int d = 0; d < kDim / 16; ++d) {
        const v8 x = v(b, d);
#pragma unroll
        for (int t = 0; t < kTiles; ++t) o[t][d] = El<kType>::mfma(x, p[t][b], o[t][d]);
      }
    }
  }
};

// Where a request's head lies in the cache.
template <int kDim>
struct Cache {
  const char *base;    // the head's codes in slot 0
  int64_t kv_stride, slot_stride, scales;  // `scales`: from the codes to the head's scale
  const int32_t *slots;
  int num_slots, shift, last;  // log2 of sub-blocks a block, last sub-block
  int32_t *status;
  __device__ __forceinline__ Cache(const Attention &a, const KvRequest &r, int head)
      : base(a.kv.base + ((int64_t)head << a.kv.block_shift) * kDim), kv_stride(a.kv.kv_stride),
        slot_stride(a.kv.slot_stride),
        scales(((int64_t)(a.kv.kv_heads - head) << a.kv.block_shift) * kDim + 4 * head),
        slots(a.slots + r.row), num_slots(a.kv.num_slots), shift(a.kv.block_shift - 4),
        last((r.len - 1) >> 4), status(a.status) {}
  // the slot of sub-block `sub`, or of the last one
  __device__ __forceinline__ int slot(int sub) const { return uniform_load(slots + (min(sub, last) >> shift)); }
  // the head's codes in a slot; a slot outside the pool is reported and read as slot 0
  __device__ __forceinline__ const char *block(int slot) const {
    if ((unsigned)slot >= (unsigned)num_slots) {
      kv_report(status);
      slot = 0;
    }
    return base + slot * slot_stride;
  }
  __device__ __forceinline__ const char *codes(const char *block, int sub) const {
    return block + (min(sub, last) & ((1 << shift) - 1)) * 16 * kDim;
  }
  __device__ __forceinline__ float k_scale(const char *block) const {
    return uniform_load(reinterpret_cast<const float *>(block + scales));
  }
  __device__ __forceinline__ float v_scale(const char *block) const {
    return uniform_load(reinterpret_cast<const float *>(block + scales + kv_stride));
  }
};
// Byte of a lane's 16 codes within 1024: of K its token is lane % 16 and its
// dims those of lane / 16, V lies in lane order.
__device__ __forceinline__ int k_place() { return (lane_id() & 15) * 64 + (lane_id() >> 4) * 16; }
__device__ __forceinline__ int v_place() { return lane_id() * 16; }

// Of 4 tokens `at` .. at + 4, the bytes of those before `len`.
__device__ __forceinline__ unsigned live_bytes(int at, int len) {
  const int n = len - at;
  return n >= 4 ? ~0u : n <= 0 ? 0u : (1u << 8 * n) - 1;
}

// 32 cached tokens of one head in registers: two sub-blocks.
template <int kDim>
struct Codes {
  u4 k[2][kDim / 64], v[2][kDim / 64];
  float ks[2], vs[2];
  __device__ __forceinline__ void fetch_k(const Cache<kDim> &c, const int (&slot)[2], int key) {
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      const char *block = c.block(slot[b]), *at = c.codes(block, (key >> 4) + b);
#pragma unroll
      for (int i = 0; i < kDim / 64; ++i) k[b][i] = *reinterpret_cast<const u4 *>(at + 1024 * i + k_place());
      ks[b] = c.k_scale(block);
    }
  }
  __device__ __forceinline__ void fetch_v(const Cache<kDim> &c, const int (&slot)[2], int key) {
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      const char *block = c.block(slot[b]), *at = c.codes(block, (key >> 4) + b) + c.kv_stride;
#pragma unroll
      for (int i = 0; i < kDim / 64; ++i) v[b][i] = *reinterpret_cast<const u4 *>(at + 1024 * i + v_place());
      vs[b] = c.v_scale(block);
    }
  }
};

// ------------------------------------------------------------- the kernel

// kKeyWaves waves share a row tile's tokens and combine in LDS; the
// kWaves / kKeyWaves groups of them each have rows of their own.
// Bytes of the list of requests at the head of a workgroup's LDS.
__host__ __device__ constexpr int list_bytes(int n) { return (12 * n + 8 + 15) & ~15; }
// Tokens that a row tile's waves share at a time.
__host__ __device__ constexpr int stage_tokens(int dim) { return dim == 256 ? 32 : 64; }
constexpr int waves_per_simd(int dim, int tiles, int key_waves) {
  if (key_waves == 1) return dim == 256 ? 1 : 2;
  const int held = dim * tiles;  // of q, o and codes in registers
  return held <= 64 ? 5 : tiles == 1 && held <= 128 ? 4 : held <= 128 ? 3 : held <= 256 ? 2 : 1;
}
template <int kType, int kDim, int kTiles, int kKeyWaves, bool kCap>
__global__ __launch_bounds__(kBlock, waves_per_simd(kDim, kTiles, kKeyWaves)) void attention_kernel(Attention a) {
  constexpr int kRows = 16 * kTiles * (kWaves / kKeyWaves);
  constexpr int kPart = kDim < 128 ? kDim : 128;  // dims that one combination takes
  constexpr int kPitch = kPart + 4;
  typedef typename El<kType>::v8 v8;
  extern __shared__ __align__(16) char lds[];
  __shared__ unsigned long long scan[2 * kWaves];
  long long *before = reinterpret_cast<long long *>(lds);
  int *ids = reinterpret_cast<int *>(before + a.batch.n + 1);
  float *mix = reinterpret_cast<float *>(lds + list_bytes(a.batch.n));
  const int lane = lane_id(), g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(wave_id());
  const int kv_heads = a.kv.kv_heads;

  // the list of requests with rows of this kernel's kind, and the cost before each
  int n = 0;
  long long total = 0;
  for (int i0 = 0; i0 < a.batch.n; i0 += kBlock) {
    const int i = i0 + threadIdx.x;
    unsigned long long v[2] = {0, 0}, all[2];
    if (i < a.batch.n) {
      const KvRequest r = kv_request(a.batch, a.row_offsets, a.kv.block_shift, i);
      if (!r.ok) {
        kv_report(a.status);
      } else {
        const int64_t rows = (int64_t)r.count * a.group;
        if (rows > a.min_rows && rows <= a.max_rows)
          v[0] = Segments(r, a.tile_tokens).total() * kv_heads;
      }
    }
    const unsigned long long cost = v[0];
    v[1] = cost > 0;
    block_exclusive_scan<2, unsigned long long>(v, all, scan);
    if (cost) {
      before[n + v[1]] = total + v[0];
      ids[n + v[1]] = i;
    }
    n += (int)all[1];
    total += all[0];
  }
  if (threadIdx.x == 0) before[n] = total;
  __syncthreads();

  // this workgroup's range: neighbours in cost on one XCD (workgroups go to
  // the 8 XCDs in turn), where heads and row tiles of a request share its L2
  const int cap = (int)min((long long)gridDim.x, total / a.range_keys);
  const int groups = cap >= 8 ? cap & ~7 : max(cap, 1);
  const int block = blockIdx.x;
  if (block >= groups || n == 0) {
    if (threadIdx.x == 0) a.splits[block] = Split{-1, 0, 0, 0};
    return;
  }
  const int w = groups >= 8 ? (block & 7) * (groups >> 3) + (block >> 3) : block;
  // lanes 0, 1, 2: this range's begin, its end, the one before's begin
  const int which = lane == 1 ? w + 1 : lane == 2 ? max(w - 1, 0) : w;
  const Place found = locate(a, before, ids, n, total * which / groups);
  Place at = uniform(found, 0);
  const Place end = uniform(found, 1), prev = uniform(found, 2);

  if (threadIdx.x == 0) {
    Split s = {-1, 0, 0, 0};
    const bool inside = at.key > 0 && !(prev.key > 0 && prev.item == at.item && prev.head == at.head &&
                                        prev.tile == at.tile);
    if (inside) {
      const int id = ids[at.item];
      const Segments seg(kv_request(a.batch, a.row_offsets, a.kv.block_shift, id), a.tile_tokens);
      const long long stop = before[at.item] + at.head * seg.total() + seg.start(at.tile) + seg.length(at.tile);
      s = {id, at.head, at.tile, (int)((stop * groups + total - 1) / total) - 1};
    }
    a.splits[w] = s;
  }

  Rowset<kType, kDim, kTiles, kCap> r;
  const int row0 = kKeyWaves == kWaves ? 0 : wave / kKeyWaves * 16 * kTiles;
  const int key_wave = wave % kKeyWaves;
  while (at.item < n) {
    const int id = __builtin_amdgcn_readfirstlane(ids[at.item]);
    const KvRequest req = kv_request<true>(a.batch, a.row_offsets, a.kv.block_shift, id);
    const Segments seg(req, a.tile_tokens);
    const int length = (int)seg.length(at.tile);
    const bool last = end.item == at.item && end.head == at.head && end.tile == at.tile;
    const int stop = last ? end.key : length;
    if (last && stop == at.key) break;

    // rows: lane n of row set t has row row0 + 16 t + n of the tile
    const int tile_rows = a.tile_tokens * a.group, shown = req.len - req.count;
    bool valid[kTiles];
    int token[kTiles], head[kTiles];
    const int64_t log_row = (int64_t)a.window * a.q_heads;
    bool logs = false;
#pragma unroll
    for (int t = 0; t < kTiles; ++t) {
      const int row = row0 + 16 * t + (lane & 15);
      token[t] = at.tile * a.tile_tokens + row / a.group;
      head[t] = at.head * a.group + row % a.group;
      valid[t] = row < tile_rows && token[t] < req.count;
      r.limit[t] = valid[t] ? shown + token[t] : -1;
      const char *q = a.q.data + (int64_t)(req.first + (valid[t] ? token[t] : 0)) * a.q.token_stride +
                      (valid[t] ? head[t] : 0) * a.q.head_stride + 32 * g;
#pragma unroll
      for (int d = 0; d < kDim / 32; ++d) {
        u4 x = *reinterpret_cast<const u4 *>(q + 128 * (d >> 1) + 16 * (d & 1));
        if (!valid[t]) x = u4{0, 0, 0, 0};
        x = (x & a.keep) ^ a.flip;
        r.q[t][d] = __builtin_bit_cast(typename El<kType>::v8, x);
      }
      r.log_at[t] = nullptr;
      const int back = req.count - 1 - token[t];
      if (a.logs && valid[t] && back < a.window)
        r.log_at[t] = a.logs + ((int64_t)req.row << (a.kv.block_shift - 4)) * log_row +
                      (int64_t)back * a.q_heads + head[t];
      logs |= r.log_at[t] != nullptr;
    }
    logs = __any(logs);
    r.clear();

    // the wave's rows begin at token first_token and end at last_token
    const int first_token = at.tile * a.tile_tokens + row0 / a.group;
    const int last_token =
        min(at.tile * a.tile_tokens + (min(row0 + 16 * kTiles, tile_rows) - 1) / a.group, req.count - 1);
    const int key_end =
        row0 >= tile_rows || first_token >= req.count ? 0 : min(min(stop, req.len), shown + last_token + 1);
    const int clear_end = shown + first_token + 1;  // every row sees the tokens before it
    const Cache<kDim> cache(a, req, at.head);
    if (kKeyWaves > 1) {
      // each wave takes every kKeyWaves-th 32 tokens, straight into registers:
      // the next K codes leave when these have been taken, V codes likewise,
      // and the slots are known a step ahead of them
      constexpr int kStride = 32 * kKeyWaves;
      int key = at.key + 32 * key_wave;
      if (key < key_end) {
        Codes<kDim> c;
        int slot[2];
        auto look = [&](int key) {
          slot[0] = cache.slot(key >> 4);
          slot[1] = cache.slot((key >> 4) + 1);
        };
        look(key);
        c.fetch_k(cache, slot, key);
        c.fetch_v(cache, slot, key);
        look(key + kStride);
        while (true) {
          const int next = key + kStride;
          if (key + 32 > req.len) {
            const unsigned live[2] = {live_bytes(key + 4 * g, req.len), live_bytes(key + 16 + 4 * g, req.len)};
#pragma unroll
            for (int i = 0; i < kDim / 64; ++i)
#pragma unroll
              for (int b = 0; b < 2; ++b) c.v[b][i] &= live[b];
          }
          r.template step<2>(
              a,
              [&](int b, int d) {
                const u4 w = c.k[b][d >> 1];
                return widen8<kType>(w[2 * (d & 1)], w[2 * (d & 1) + 1], c.ks[b], c.ks[b]);
              },
              [&](int, int d) {
                return widen8<kType>(c.v[0][d >> 2][d & 3], c.v[1][d >> 2][d & 3], c.vs[0], c.vs[1]);
              },
              [&] { if (next < key_end) c.fetch_k(cache, slot, next); }, key, req.len, key + 32 > clear_end,
              logs, log_row);
          if (next >= key_end) break;
          c.fetch_v(cache, slot, next);
          look(next + kStride);
          key = next;
        }
      }
    } else {
      // the waves share the tokens through LDS, kStage of them at a time,
      // widened once and in operand order; the next stage's codes cross in
      // registers meanwhile.  Pieces of 1 KiB of codes: sub-block, K or V, 64
      // dims; a wave carries kOwn, all of one sub-block and side or both.
      constexpr int kSubs = stage_tokens(kDim) / 16, kStage = 16 * kSubs;
      constexpr int kSlices = kDim / 64, kOwn = kSubs * 2 * kSlices / kWaves;
      constexpr int kBytes = kStage * kDim * 4;  // of a stage: K's operands, then V's
      char *stage = lds + list_bytes(a.batch.n);
      const int block_end = min(stop, min(req.len, shown + min((at.tile + 1) * a.tile_tokens, req.count)));
      const int sub = wave * kOwn / (2 * kSlices);
      u4 own[kOwn];
      float ks, vs;
      int live_key;
      auto fetch = [&](int key) {
        const char *block = cache.block(cache.slot((key >> 4) + sub));
        const char *from = cache.codes(block, (key >> 4) + sub);
        ks = cache.k_scale(block);
        vs = cache.v_scale(block);
        live_key = key + 16 * sub;
#pragma unroll
        for (int i = 0; i < kOwn; ++i) {
          const int p = (wave * kOwn + i) % (2 * kSlices), side = p / kSlices;
          own[i] = *reinterpret_cast<const u4 *>(from + side * cache.kv_stride + p % kSlices * 1024 +
                                                 (side ? v_place() : k_place()));
        }
      };
      // K: operand [sub-block][dims step][lane]; V: [pair of sub-blocks][16 dims][lane],
      // the pair's halves side by side
      auto put = [&](char *to) {
        const unsigned live = live_bytes(live_key + 4 * g, req.len);
#pragma unroll
        for (int i = 0; i < kOwn; ++i) {
          const int p = (wave * kOwn + i) % (2 * kSlices), side = p / kSlices, c = p % kSlices;
          if (side == 0) {
            char *at = to + ((sub * kSlices + c) * 2 * 64 + lane) * 16;
#pragma unroll
            for (int h = 0; h < 2; ++h)
              *reinterpret_cast<v8 *>(at + h * 1024) = widen8<kType>(own[i][2 * h], own[i][2 * h + 1], ks, ks);
          } else {
            char *at = to + kBytes / 2 + (((sub >> 1) * 4 * kSlices + 4 * c) * 64 + lane) * 16 + (sub & 1) * 8;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const unsigned w = own[i][j] & live;
              *reinterpret_cast<u2 *>(at + j * 1024) = u2{El<kType>::widen_lo(w, vs), El<kType>::widen_hi(w, vs)};
            }
          }
        }
      };
      auto compute = [&](const char *from, int key) {
        if (key >= key_end) return;
        r.template step<kSubs>(
            a,
            [&](int b, int d) {
              return *reinterpret_cast<const v8 *>(from + ((b * 2 * kSlices + d) * 64 + lane) * 16);
            },
            [&](int b, int d) {
              return *reinterpret_cast<const v8 *>(from + kBytes / 2 + ((b * 4 * kSlices + d) * 64 + lane) * 16);
            },
            [] {}, key, req.len, key + kStage > clear_end, logs, log_row);
      };
      if (at.key < block_end) {
        fetch(at.key);
        put(stage);
        __syncthreads();
        int buffer = 0;
        for (int key = at.key;;) {
          const int next = key + kStage;
          if (next < block_end) fetch(next);
          compute(stage + buffer * kBytes, key);
          if (next >= block_end) break;
          key = next;
          buffer ^= 1;
          put(stage + buffer * kBytes);
          __syncthreads();
        }
      }
      __syncthreads();
    }

#pragma unroll
    for (int t = 0; t < kTiles; ++t) {
      r.sum[t] += __shfl_xor(r.sum[t], 16);
      r.sum[t] += __shfl_xor(r.sum[t], 32);
    }
    const bool whole = at.key == 0 && stop == length;
    const int64_t part = ((int64_t)w * 2 + (at.key > 0 ? 0 : 1)) * kRows;
    if (kKeyWaves == 1) {
#pragma unroll
      for (int t = 0; t < kTiles; ++t) {
        const int row = row0 + 16 * t + (lane & 15);
        if (!valid[t]) continue;
        if (whole) {
          const float f = r.sum[t] > 0.f ? 1.f / r.sum[t] : r.sum[t] == 0.f ? 0.f : r.sum[t];
          char *out = a.out.data + (int64_t)(req.first + token[t]) * a.out.token_stride +
                      head[t] * a.out.head_stride;
#pragma unroll
          for (int d = 0; d < kDim / 16; ++d) {
            const u2 x = {narrow2<kType>(r.o[t][d][0] * f, r.o[t][d][1] * f),
                          narrow2<kType>(r.o[t][d][2] * f, r.o[t][d][3] * f)};
            *reinterpret_cast<u2 *>(out + 2 * (16 * d + 4 * g)) = x;
          }
          if (a.lse && g == 0)
            a.lse[(int64_t)(req.first + token[t]) * a.q_heads + head[t]] =
                (r.m[t] + __builtin_amdgcn_logf(r.sum[t])) * kLn2;
        } else {
          float *o = a.parts + (part + row) * kDim + 4 * g;
#pragma unroll
          for (int d = 0; d < kDim / 16; ++d) *reinterpret_cast<f4 *>(o + 16 * d) = r.o[t][d];
          if (g == 0) *reinterpret_cast<f2 *>(a.part_sums + 2 * (part + row)) = f2{r.m[t], r.sum[t]};
        }
      }
    } else {
      // the waves' m, sum and O of one row set at a time
      float *ms = mix, *os = mix + 2 * kWaves * 16;
#pragma unroll
      for (int t = 0; t < kTiles; ++t) {
        if (g == 0) {
          ms[(wave * 16 + lane) * 2] = r.m[t];
          ms[(wave * 16 + lane) * 2 + 1] = r.sum[t];
        }
        __syncthreads();
        float top = kLowest;
#pragma unroll
        for (int k = 0; k < kWaves; ++k) top = fmaxf(top, ms[(k * 16 + (lane & 15)) * 2]);
        const float f = __builtin_amdgcn_exp2f(r.m[t] - top);
#pragma unroll
        for (int d0 = 0; d0 < kDim; d0 += kPart) {
#pragma unroll
          for (int d = d0 / 16; d < (d0 + kPart) / 16; ++d)
            *reinterpret_cast<f4 *>(os + (wave * 16 + (lane & 15)) * kPitch + 16 * d - d0 + 4 * g) = r.o[t][d] * f;
          __syncthreads();
          for (int j = threadIdx.x; j < 16 * kPart / 4; j += kBlock) {
            const int n16 = j / (kPart / 4), d = j % (kPart / 4) * 4;
            f4 o = {0.f, 0.f, 0.f, 0.f};
            float m = kLowest, sum = 0.f;
#pragma unroll
            for (int k = 0; k < kWaves; ++k) {
              o += *reinterpret_cast<const f4 *>(os + (k * 16 + n16) * kPitch + d);
              m = fmaxf(m, ms[(k * 16 + n16) * 2]);
            }
#pragma unroll
            for (int k = 0; k < kWaves; ++k)
              sum += ms[(k * 16 + n16) * 2 + 1] * __builtin_amdgcn_exp2f(ms[(k * 16 + n16) * 2] - m);
            const int row = 16 * t + n16, tok = at.tile * a.tile_tokens + row / a.group;
            if (row >= tile_rows || tok >= req.count) continue;
            if (whole) {
              const int h = at.head * a.group + row % a.group;
              const float inv = sum > 0.f ? 1.f / sum : sum == 0.f ? 0.f : sum;
              const u2 x = {narrow2<kType>(o[0] * inv, o[1] * inv), narrow2<kType>(o[2] * inv, o[3] * inv)};
              *reinterpret_cast<u2 *>(a.out.data + (int64_t)(req.first + tok) * a.out.token_stride +
                                      h * a.out.head_stride + 2 * (d0 + d)) = x;
              if (a.lse && d0 + d == 0)
                a.lse[(int64_t)(req.first + tok) * a.q_heads + h] = (m + __builtin_amdgcn_logf(sum)) * kLn2;
            } else {
              *reinterpret_cast<f4 *>(a.parts + (part + row) * kDim + d0 + d) = o;
              if (d0 + d == 0) *reinterpret_cast<f2 *>(a.part_sums + 2 * (part + row)) = f2{m, sum};
            }
          }
          __syncthreads();
        }
      }
    }

    if (last) break;
    at.key = 0;
    if (++at.tile == seg.tiles()) {
      at.tile = 0;
      if (++at.head == kv_heads) {
        at.head = 0;
        ++at.item;
      }
    }
  }
}

// Joins the parts of cut segments: one wave per row.
template <int kType, int kDim>
__global__ __launch_bounds__(kBlock) void join_kernel(Attention a, int rows) {
  constexpr int kLanes = kDim / 4, kParts = 64 / kLanes;
  const Split s = a.splits[blockIdx.x];
  if (s.request < 0) return;
  const int row = __builtin_amdgcn_readfirstlane((int)blockIdx.y * kWaves + wave_id()), lane = lane_id();
  const KvRequest req = kv_request(a.batch, a.row_offsets, a.kv.block_shift, s.request);
  const int token = s.tile * a.tile_tokens + row / a.group;
  if (row >= a.tile_tokens * a.group || token >= req.count) return;
  const int head = s.head * a.group + row % a.group;
  // part 0 ends the range of the workgroup before the cut, the others begin theirs
  const int w = blockIdx.x, parts = s.last - w + 2;
  auto place = [&](int p) { return ((int64_t)(w - 1 + p) * 2 + (p == 0)) * rows + row; };
  float top = kLowest;
  for (int p = lane; p < parts; p += 64) top = fmaxf(top, a.part_sums[2 * place(p)]);
#pragma unroll
  for (int d = 32; d; d >>= 1) top = fmaxf(top, __shfl_xor(top, d));
  float sum = 0.f;
  for (int p = lane; p < parts; p += 64) {
    const f2 ms = *reinterpret_cast<const f2 *>(a.part_sums + 2 * place(p));
    sum += ms[1] * __builtin_amdgcn_exp2f(ms[0] - top);
  }
#pragma unroll
  for (int d = 32; d; d >>= 1) sum += __shfl_xor(sum, d);
  f4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
  for (int p = lane / kLanes; p < parts; p += kParts) {
    const float f = __builtin_amdgcn_exp2f(a.part_sums[2 * place(p)] - top);
    o += *reinterpret_cast<const f4 *>(a.parts + place(p) * kDim + 4 * (lane % kLanes)) * f;
  }
#pragma unroll
  for (int d = 32; d >= kLanes; d >>= 1)
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] += __shfl_xor(o[i], d);
  if (lane < kLanes) {
    const float f = sum > 0.f ? 1.f / sum : sum == 0.f ? 0.f : sum;
    const u2 x = {narrow2<kType>(o[0] * f, o[1] * f), narrow2<kType>(o[2] * f, o[3] * f)};
    *reinterpret_cast<u2 *>(a.out.data + (int64_t)(req.first + token) * a.out.token_stride +
                            head * a.out.head_stride + 8 * lane) = x;
  }
  if (a.lse && lane == 0)
    a.lse[(int64_t)(req.first + token) * a.q_heads + head] = (top + __builtin_amdgcn_logf(sum)) * kLn2;
}

// Adds to each table entry the weight that its request's last tokens gave it:
// one wave per entry, its sub-blocks' log sums against the rows' totals.
constexpr int kEntries = 4 * kWaves;  // entries of one workgroup
__global__ __launch_bounds__(kBlock) void weight_kernel(Attention a, float *block_weight) {
  __shared__ unsigned sums[kWaves];
  const int e0 = blockIdx.x * kEntries, lane = lane_id(), subs = a.kv.block_shift - 4;
  unsigned ended[1] = {0};
  for (int i = threadIdx.x; i < a.batch.n; i += kBlock) ended[0] += a.row_offsets[i + 1] <= e0;
  block_sum<1, unsigned>(ended, sums);
  int i = __builtin_amdgcn_readfirstlane((int)ended[0]);
  for (int e = e0 + wave_id(); e < min(e0 + kEntries, a.batch.n_entries); e += kWaves) {
    while (i < a.batch.n && a.row_offsets[i + 1] <= e) ++i;
    if (i >= a.batch.n) return;
    const KvRequest r = kv_request(a.batch, a.row_offsets, a.kv.block_shift, i);
    if (!r.ok || e < r.row || (int64_t)(e - r.row) << (subs + 4) >= r.len || r.count == 0) continue;
    const int rows = min(a.window, r.count) * a.q_heads;
    float sum = 0.f;
    for (int s = 0; s < 1 << subs; ++s) {
      const int first = (((e - r.row) << subs) + s) << 4;  // the sub-block's first token
      const float *log = a.logs + (((int64_t)e << subs) + s) * a.window * a.q_heads;
      for (int j = lane; j < rows; j += 64) {
        const int back = j / a.q_heads;
        if (first > r.len - 1 - back) continue;  // not seen
        const float lse = a.lse[(int64_t)(r.first + r.count - 1 - back) * a.q_heads + j % a.q_heads];
        sum += __builtin_amdgcn_exp2f(log[j] - lse * kLog2e);
      }
    }
#pragma unroll
    for (int d = 32; d; d >>= 1) sum += __shfl_xor(sum, d);
    if (lane == 0) block_weight[e] += sum;
  }
}

// ------------------------------------------------------------------- host

constexpr int kGroups = 1024;      // workgroups of the kernel that splits tokens over waves
constexpr int kTileGroups = 512;   // of the kernel that splits rows over waves
constexpr int kTileRows = 128;     // its row tile
constexpr int most_rows(int dim) { return dim == 256 ? 32 : 64; }  // of a request in the former

struct Workspace {
  size_t splits, tile_splits, parts, tile_parts, sums, tile_sums, lse, logs, total;
};

size_t aligned(size_t n) { return (n + 255) & ~(size_t)255; }

Workspace layout(const cascade_kv_format_t *f, const cascade_kv_batch_t *b, int q_heads, int window) {
  Workspace w;
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t here = at;
    at += aligned(bytes);
    return here;
  };
  w.splits = take(sizeof(Split) * kGroups);
  w.tile_splits = take(sizeof(Split) * kTileGroups);
  w.parts = take(sizeof(float) * kGroups * 2 * most_rows(f->head_dim) * f->head_dim);
  w.tile_parts = take(sizeof(float) * kTileGroups * 2 * kTileRows * f->head_dim);
  w.sums = take(sizeof(float) * kGroups * 2 * most_rows(f->head_dim) * 2);
  w.tile_sums = take(sizeof(float) * kTileGroups * 2 * kTileRows * 2);
  w.lse = take(window ? sizeof(float) * b->n_tokens * q_heads : 0);
  w.logs = take(window ? sizeof(float) * b->n_entries * (f->block_tokens / 16) * window * q_heads : 0);
  w.total = at;
  return w;
}

bool heads_ok(const cascade_kv_format_t *f, int q_heads) {
  return q_heads >= 1 && q_heads % f->kv_heads == 0 && q_heads / f->kv_heads <= 128;
}

template <int kType, int kDim, int kTiles, int kKeyWaves>
void start(const Attention &a, int grid, bool cap, hipStream_t stream) {
  // combination of the waves, or two stages of operands
  const size_t mix = kKeyWaves > 1 ? sizeof(float) * kWaves * 16 * (2 + (kDim < 128 ? kDim : 128) + 4)
                                   : 2 * stage_tokens(kDim) * 4 * kDim;
  auto kernel = cap ? attention_kernel<kType, kDim, kTiles, kKeyWaves, true>
                    : attention_kernel<kType, kDim, kTiles, kKeyWaves, false>;
  hipLaunchKernelGGL(kernel, dim3(grid), dim3(kBlock), list_bytes(a.batch.n) + mix, stream, a);
}

template <int kType, int kDim>
int run(Attention a, char *ws, const Workspace &w, bool cap, float *block_weight, hipStream_t s) {
  const int64_t most = (int64_t)a.batch.max_new * a.group;  // rows of a request and KV head
  const int64_t keys = ((int64_t)a.batch.n_entries << a.kv.block_shift) * a.kv.kv_heads;
  // few rows: 4 waves share a tile's tokens.  More: row tiles of 128,
  // and requests of up to 32 rows beside them in the first kernel
  const bool tiled = most > most_rows(kDim);
  const int small = most <= 16 ? 16 : most <= 32 || tiled ? 32 : 64;
  a.min_rows = 0;
  a.max_rows = small;
  a.tile_tokens = small / a.group > 0 ? small / a.group : 1;
  a.atomic_keys = 0;
  a.cut_keys = 32;
  a.range_keys = 256;
  a.splits = reinterpret_cast<Split *>(ws + w.splits);
  a.parts = reinterpret_cast<float *>(ws + w.parts);
  a.part_sums = reinterpret_cast<float *>(ws + w.sums);
  int64_t grid = keys / a.range_keys;
  grid = grid < 8 ? 8 : grid > kGroups ? kGroups : grid;
  if (small == 16)
    start<kType, kDim, 1, 4>(a, (int)grid, cap, s);
  else if (small == 32)
    start<kType, kDim, 2, 4>(a, (int)grid, cap, s);
  else if constexpr (kDim < 256)
    start<kType, kDim, 4, 4>(a, (int)grid, cap, s);
  hipLaunchKernelGGL((join_kernel<kType, kDim>), dim3((int)grid, small / kWaves), dim3(kBlock), 0, s, a,
                     small);
  if (tiled) {
    a.min_rows = small;
    a.max_rows = INT64_MAX;
    a.tile_tokens = kTileRows / a.group;
    a.atomic_keys = 2048;
    a.cut_keys = stage_tokens(kDim);
    a.range_keys = 256;
    a.splits = reinterpret_cast<Split *>(ws + w.tile_splits);
    a.parts = reinterpret_cast<float *>(ws + w.tile_parts);
    a.part_sums = reinterpret_cast<float *>(ws + w.tile_sums);
    start<kType, kDim, 2, 1>(a, kTileGroups, cap, s);
    hipLaunchKernelGGL((join_kernel<kType, kDim>), dim3(kTileGroups, kTileRows / kWaves), dim3(kBlock), 0,
                       s, a, kTileRows);
  }
  if (block_weight)
    hipLaunchKernelGGL(weight_kernel, dim3((a.batch.n_entries + kEntries - 1) / kEntries), dim3(kBlock), 0,
                       s, a, block_weight);
  return hipGetLastError() == hipSuccess ? CASCADE_OK : CASCADE_EHIP;
}

template <int kType>
int run(const Attention &a, char *ws, const Workspace &w, bool cap, float *block_weight, hipStream_t s) {
  switch (a.kv.head_dim) {
    case 64: return run<kType, 64>(a, ws, w, cap, block_weight, s);
    case 128: return run<kType, 128>(a, ws, w, cap, block_weight, s);
    default: return run<kType, 256>(a, ws, w, cap, block_weight, s);
  }
}

}  // namespace
}  // namespace cascade

using namespace cascade;

extern "C" size_t cascade_attention_workspace_bytes(const cascade_kv_format_t *format,
                                                    const cascade_kv_batch_t *batch, int32_t q_heads,
                                                    int32_t weight_window) {
  if (!kv_format_ok(format) || !batch || batch->n_tokens < 0 || batch->n_entries < 0 ||
      !heads_ok(format, q_heads) || weight_window < 0 || weight_window > 64)
    return 0;
  return layout(format, batch, q_heads, weight_window).total;
}

extern "C" int cascade_attention(const cascade_kv_pool_t *pool, int32_t layer,
                                 const cascade_kv_format_t *format, const cascade_kv_batch_t *batch,
                                 const cascade_block_table_t *table, const cascade_attention_t *args,
                                 void *workspace, size_t workspace_bytes, int32_t *status_dev,
                                 void *stream) {
  if (!kv_pool_ok(pool, layer, format) || !kv_batch_ok(batch, table) || !args) return CASCADE_EINVAL;
  if ((args->dtype != CASCADE_BF16 && args->dtype != CASCADE_F16) || !heads_ok(format, args->q_heads) ||
      !std::isfinite(args->scale) || !std::isfinite(args->softcap) || args->softcap < 0)
    return CASCADE_EINVAL;
  if (args->block_weight ? args->weight_window < 1 || args->weight_window > 64 : args->weight_window != 0)
    return CASCADE_EINVAL;
  if (!workspace || ((uintptr_t)workspace & 255)) return CASCADE_EINVAL;
  const Workspace w = layout(format, batch, args->q_heads, args->weight_window);
  if (workspace_bytes < w.total) return CASCADE_ENOSPC;
  if (batch->n == 0 || batch->n_tokens == 0 || batch->max_new == 0) return CASCADE_OK;
  if (!kv_rows_ok(&args->q) || !kv_rows_ok(&args->out)) return CASCADE_EINVAL;
  Attention a = {};
  a.kv = kv_view(pool, layer, format);
  a.batch = *batch;
  a.row_offsets = table->row_offsets;
  a.slots = table->slots;
  a.q = Rows{static_cast<char *>(args->q.data), 2 * args->q.token_stride, 2 * args->q.head_stride};
  a.out = Rows{static_cast<char *>(args->out.data), 2 * args->out.token_stride, 2 * args->out.head_stride};
  a.q_heads = args->q_heads;
  a.group = args->q_heads / format->kv_heads;
  const bool cap = args->softcap > 0;
  // softmax(-s q.k) is softmax(s (-q).k): the largest score is then that of
  // the largest product
  const float scale = std::fabs(args->scale);
  a.flip = args->scale < 0 ? 0x80008000u : 0u;
  a.keep = scale > 0 ? ~0u : 0u;
  a.scale = (cap ? args->softcap : scale > 0 ? scale : 1.f) * kLog2e;
  a.cap_in = cap ? 2 * kLog2e * scale / args->softcap : 0.f;
  char *ws = static_cast<char *>(workspace);
  a.window = args->weight_window;
  a.lse = args->lse ? args->lse : a.window ? reinterpret_cast<float *>(ws + w.lse) : nullptr;
  a.logs = a.window && batch->n_entries ? reinterpret_cast<float *>(ws + w.logs) : nullptr;
  a.status = status_dev;
  const auto s = static_cast<hipStream_t>(stream);
  float *weight = a.logs ? args->block_weight : nullptr;
  return args->dtype == CASCADE_BF16 ? run<CASCADE_BF16>(a, ws, w, cap, weight, s)
                                     : run<CASCADE_F16>(a, ws, w, cap, weight, s);
}
