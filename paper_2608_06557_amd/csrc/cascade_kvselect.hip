// cascade_kvselect.hip -- bounds of the keys of each block of the 8-bit paged
// KV cache, and the blocks whose bounds promise a token's largest scores, on
// gfx950.
//
// With u_d and l_d the largest and least of a block's keys in dim d, a key's
// score is at most sum_d max(q_d u_d, q_d l_d) = sum_d q+_d u_d + q-_d l_d,
// q+ = max(q, 0), q- = min(q, 0): a product of 2 head_dim numbers for a block's
// block_tokens keys.  Bounds are whole numbers (an E4M3 code is at most 448:
// ceil(u / 4), floor(l / 4) fit 8 bits with their block's scale), queries are
// rounded to whole numbers up to 127 of a power of two, and the sums, below
// 2^23, are exact in the 8-bit matrix instructions.  Scores are exact too
// (whole numbers times powers of two), so a selection does not depend on the
// order of sums.
//
// bounds: one wave reads a block and head's codes in operand order, 16 dims of
// a token in a lane, and halves the dims it answers for at each exchange.  4.5 us
// for 128 single tokens and 8.5 us for 512 blocks of 8 heads x 128 dims, inputs in
// HBM: the launch and three dependent loads (offsets, slot, codes).
// score: a wave holds the queries of 16 rows (tokens and heads of a group) as the
// first operand and takes 16 blocks at a time as the second, so a lane has one
// block's scores of 4 rows, and the largest over a group's heads is taken in
// registers.  Nothing but a block's bounds, 2 head_dim bytes a head,
// and its scale is read, so 128 single tokens over 84 thousand blocks are bound
// by HBM: 48 us, 209 MB fetched (the bounds are 173; the 1 KB of a block begin inside a
// line), 4.3 TB/s.  With many rows of one request the bounds come from LDS for four
// waves' row sets: 128 sets of each of 8 KV heads over 2001 blocks 23 us, by the vector
// instructions of scaling and of the heads' largest, and by their latency.
// select: a row's candidates stay in registers, of a workgroup or of one wave; a
// histogram of their range in LDS leaves few in the part where the least score that
// stays is (else a radix selection over the scores' bits finds it), and ballots write
// the blocks in order.  1024 rows of 660 blocks 9.0 us, 4096 rows of 2000 17 us (a wave
// to a row), of 4000 35 us (a workgroup).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "cascade.h"
#include "device_util.h"
#include "kv_format.h"

namespace cascade {
namespace {

typedef int i4 __attribute__((ext_vector_type(4)));
typedef unsigned u4 __attribute__((ext_vector_type(4)));
typedef _Float16 h2 __attribute__((ext_vector_type(2)));

constexpr int kMinExponent = -100;  // of a row of whole queries

// From a chunk's begin to its head's bounds.
__device__ __forceinline__ int64_t bounds_at(const KvView &kv, int head) {
  const int64_t codes = (int64_t)kv.kv_heads * kv.head_dim << kv.block_shift;
  return codes + (4 * kv.kv_heads + 15) / 16 * 16 + (int64_t)head * kv.head_dim;
}
__device__ __forceinline__ int64_t scale_at(const KvView &kv, int head) {
  return ((int64_t)kv.kv_heads * kv.head_dim << kv.block_shift) + 4 * head;
}

// ------------------------------------------------------------------ bounds

struct Bounds {
  KvView kv;
  cascade_kv_batch_t batch;
  const int32_t *row_offsets, *slots;
  int whole;  // all of the requests' blocks, not only those of new tokens
  int units;  // table entries, or new tokens
  int group;  // of them a workgroup
  int32_t *status;
};

__device__ __forceinline__ h2 larger(h2 a, h2 b) { return __builtin_elementwise_max(a, b); }
__device__ __forceinline__ h2 smaller(h2 a, h2 b) { return __builtin_elementwise_min(a, b); }
__device__ __forceinline__ h2 other_lane(h2 x, int mask) {
  return __builtin_bit_cast(h2, __shfl_xor(__builtin_bit_cast(int, x), mask));
}
// ceil or floor of a quarter, as a byte
__device__ __forceinline__ unsigned quarter_up(_Float16 x) {
  return (unsigned)(int)__builtin_ceilf((float)x * 0.25f) & 255u;
}
__device__ __forceinline__ unsigned quarter_down(_Float16 x) {
  return (unsigned)(int)__builtin_floorf((float)x * 0.25f) & 255u;
}

// One wave: the bounds of the first `tokens` tokens of a block.
template <int kDim>
__device__ __forceinline__ void bound_block(const Bounds &a, int slot, int head, int tokens) {
  const int lane = lane_id();
  char *const chunk = const_cast<char *>(a.kv.base) + slot * a.kv.slot_stride;
  const char *const codes = chunk + ((int64_t)head * kDim << a.kv.block_shift);
  h2 top[kDim / 64][8], low[kDim / 64][8];
  const _Float16 inf = (_Float16)__builtin_inff();
#pragma unroll
  for (int c = 0; c < kDim / 64; ++c)
#pragma unroll
    for (int i = 0; i < 8; ++i) top[c][i] = h2{-inf, -inf}, low[c][i] = h2{inf, inf};
  // 4 KB of codes are on their way at once; past the end the last
  // sub-block's are read again
  constexpr int kAtOnce = 256 / kDim;
  const int last = (tokens - 1) & ~15;
  for (int t0 = 0; t0 < tokens; t0 += 16 * kAtOnce) {
    u4 w[kAtOnce][kDim / 64];
#pragma unroll
    for (int j = 0; j < kAtOnce; ++j)
#pragma unroll
      for (int c = 0; c < kDim / 64; ++c)
        w[j][c] = *reinterpret_cast<const u4 *>(codes + min(t0 + 16 * j, last) * kDim + 1024 * c + 16 * lane);
#pragma unroll
    for (int j = 0; j < kAtOnce; ++j) {
      if (t0 + 16 * j > last) break;
      if (t0 + 16 * j + lane / 4 >= tokens) continue;  // may be anything
#pragma unroll
      for (int c = 0; c < kDim / 64; ++c)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const h2 x = __builtin_bit_cast(h2, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w[j][c][i], 1.f, false));
          const h2 y = __builtin_bit_cast(h2, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w[j][c][i], 1.f, true));
          top[c][2 * i] = larger(top[c][2 * i], x), low[c][2 * i] = smaller(low[c][2 * i], x);
          top[c][2 * i + 1] = larger(top[c][2 * i + 1], y), low[c][2 * i + 1] = smaller(low[c][2 * i + 1], y);
        }
    }
  }
  // lanes 4 t + p hold dims 16 p .. of token t: at each exchange a lane keeps half
  const int64_t at = bounds_at(a.kv, head);
#pragma unroll
  for (int c = 0; c < kDim / 64; ++c) {
    int first = 0;  // of the dims pairs that are left
    auto halve = [&](auto left) {
      constexpr int kKeep = decltype(left)::value, kMask = 8 * kKeep;
      const bool upper = lane & kMask;
#pragma unroll
      for (int i = 0; i < kKeep; ++i) {
        const h2 mine = upper ? top[c][kKeep + i] : top[c][i], give = upper ? top[c][i] : top[c][kKeep + i];
        top[c][i] = larger(mine, other_lane(give, kMask));
        const h2 mine_low = upper ? low[c][kKeep + i] : low[c][i], give_low = upper ? low[c][i] : low[c][kKeep + i];
        low[c][i] = smaller(mine_low, other_lane(give_low, kMask));
      }
      first += upper ? kKeep : 0;
    };
    halve(std::integral_constant<int, 4>());
    halve(std::integral_constant<int, 2>());
    halve(std::integral_constant<int, 1>());
    const h2 u = larger(top[c][0], other_lane(top[c][0], 4)), l = smaller(low[c][0], other_lane(low[c][0], 4));
    if (!(lane & 4)) {
      char *const to = chunk + at + 64 * c + 16 * (lane & 3) + 2 * first;
      *reinterpret_cast<uint16_t *>(to) = (uint16_t)(quarter_up(u[0]) | quarter_up(u[1]) << 8);
      *reinterpret_cast<uint16_t *>(to + a.kv.kv_stride) = (uint16_t)(quarter_down(l[0]) | quarter_down(l[1]) << 8);
    }
  }
}

// A unit is a table entry, or a new token; a token stands for its block if it
// is the first new one there.
template <int kDim>
__global__ __launch_bounds__(kBlock) void bounds_kernel(Bounds a) {
  if (blockIdx.x == gridDim.x - 1) {
    if (blockIdx.y == 0) check_requests(a.batch, a.row_offsets, a.kv.block_shift, a.status);
    return;
  }
  __shared__ int owners[kWaves];
  const int u0 = blockIdx.x * a.group, u1 = u0 + min(a.group, a.units - u0);
  int i = owner_of(a.whole ? a.row_offsets : a.batch.token_offsets, a.batch.n, u0, owners);
  const int bt = 1 << a.kv.block_shift;
  for (int u = u0; i < a.batch.n && u < u1; ++i) {
    const KvRequest r = kv_request(a.batch, a.row_offsets, a.kv.block_shift, i);
    if (!r.ok) continue;
    const int first = a.whole ? r.row : r.first;
    const int end = a.whole ? r.row + ((r.len + bt - 1) >> a.kv.block_shift) : r.first + r.count;
    for (u = max(u, first); u < min(u1, end); ++u) {
      int block = u - r.row;
      if (!a.whole) {
        const int token = r.len - r.count + (u - r.first);  // below 0: more new tokens than cached
        if (token < 0 || ((token & (bt - 1)) && u != r.first)) continue;
        block = token >> a.kv.block_shift;
      }
      const int slot = a.slots[r.row + block];
      if ((unsigned)slot >= (unsigned)a.kv.num_slots) {
        kv_report(a.status);
        continue;
      }
      const int tokens = min(bt, r.len - (block << a.kv.block_shift));
      for (int head = blockIdx.y * kWaves + wave_id(); head < a.kv.kv_heads; head += gridDim.y * kWaves)
        bound_block<kDim>(a, slot, head, tokens);
    }
  }
}

// ------------------------------------------------------------------- score

struct QRows {
  const char *data;
  int64_t token_stride, head_stride;  // bytes
};

struct Select {
  KvView kv;
  cascade_kv_batch_t batch;
  const int32_t *row_offsets, *slots;
  QRows q;
  int group;   // query heads of a KV head
  int padded;  // the same as a power of two up to 16, or a multiple of 16
  int shift;   // log2 of a token's rows in a set
  int keep, sink, recent;
  int span;    // table entries of a workgroup
  int spans, sets;  // how many, and sets of rows of a workgroup
  int first, run;   // the new tokens of each request that are scored and selected, and how many at most
  int most, pitch;  // by tokens: blocks of a request, and those in whole lines of 16; else any and 0
  float *scores;  // [token][KV head][pitch], or request by request [token of the run][KV head][block], in lines of 16
  int *limit;       // the first request behind which offsets fall: from there on none is scored
  int scored;       // whether any is
  int32_t *selected;
  int32_t *status;
};

__device__ __forceinline__ int blocks_of(const KvRequest &r, int block_shift) {
  return (int)(((long long)r.len + (1 << block_shift) - 1) >> block_shift);
}
// A row's scores, and how many there is room for; `token` is one of the run.  By tokens a row's
// place is its number.  By requests, where request i's begin: 16 (floor(row / 16) + i) lines' places for each
// token and head, which leaves room for its blocks rounded up, as the next request's row is at
// least as many entries further.
__device__ __forceinline__ int score_pitch(const Select &a, const KvRequest &r) {
  return a.pitch ? a.pitch : (blocks_of(r, a.kv.block_shift) + 15) & ~15;
}
__device__ __forceinline__ float *scores_of(const Select &a, const KvRequest &r, int i, int token, int head) {
  const int64_t first = a.pitch ? (int64_t)r.first * a.kv.kv_heads * a.pitch
                                : ((int64_t)(r.row & ~15) + 16 * i) * a.run * a.kv.kv_heads;
  return a.scores + first + ((int64_t)token * a.kv.kv_heads + head) * score_pitch(a, r);
}

typedef uint16_t us2 __attribute__((ext_vector_type(2)));

template <int kType>
__device__ __forceinline__ void widen2(unsigned w, float &a, float &b) {
  if constexpr (kType == CASCADE_BF16) {
    a = __uint_as_float(w << 16), b = __uint_as_float(w & 0xffff0000u);
  } else {
    const h2 x = __builtin_bit_cast(h2, w);
    a = (float)x[0], b = (float)x[1];
  }
}

// A row of queries (16 of them, a row to lane % 16): its dims 16 (lane / 16) .. of each 64.
template <int kType, int kDim>
struct Query {
  static constexpr unsigned kInf = kType == CASCADE_BF16 ? 0x7f80 : 0x7c00;
  u4 w[kDim / 64][2];
  __device__ __forceinline__ void load(const Select &a, const KvRequest &r, int head, int token, int of_group,
                                       bool valid) {
    const char *from = a.q.data + (int64_t)(r.first + (valid ? token : 0)) * a.q.token_stride +
                       (int64_t)(head * a.group + (valid ? of_group : 0)) * a.q.head_stride + 32 * (lane_id() >> 4);
#pragma unroll
    for (int s = 0; s < kDim / 64; ++s)
#pragma unroll
      for (int v = 0; v < 2; ++v) {
        w[s][v] = *reinterpret_cast<const u4 *>(from + 128 * s + 16 * v);
        w[s][v] = valid ? w[s][v] : u4{0, 0, 0, 0};
      }
  }
  // The exponent of its whole numbers; elements that are not finite become 0.
  __device__ __forceinline__ int exponent(bool &bad) {
    auto magnitude = [&] {  // 16-bit magnitudes are in the order of their values
      us2 most = {0, 0};
#pragma unroll
      for (int s = 0; s < kDim / 64; ++s)
#pragma unroll
        for (int i = 0; i < 8; ++i)
          most = __builtin_elementwise_max(most, __builtin_bit_cast(us2, w[s][i >> 2][i & 3] & 0x7fff7fffu));
      return most[0] > most[1] ? most[0] : most[1];
    };
    unsigned most = magnitude();
    if (__builtin_expect(__any(most >= kInf), false)) {
      bad |= most >= kInf;
#pragma unroll
      for (int s = 0; s < kDim / 64; ++s)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          unsigned x = w[s][i >> 2][i & 3];
          x = (x & 0x7fffu) >= kInf ? x & 0xffff0000u : x;
          x = (x >> 16 & 0x7fffu) >= kInf ? x & 0xffffu : x;
          w[s][i >> 2][i & 3] = x;
        }
      most = magnitude();
    }
    float x, none;
    widen2<kType>(most, x, none);
    x = fmaxf(x, __shfl_xor(x, 16));
    x = fmaxf(x, __shfl_xor(x, 32));
    // the least with x <= 127 * 2^exponent; 127 is 1.984375 * 2^6
    const unsigned b = __float_as_uint(x);
    return max((int)(b >> 23) - 127 - 6 + ((b & 0x7fffffu) > 0x7e0000u ? 1 : 0), kMinExponent);
  }
};

// 16 rows in whole numbers, in operand order.
template <int kDim>
struct Operand {
  i4 plus[kDim / 64], minus[kDim / 64];
  template <int kType>
  __device__ __forceinline__ void round(const Query<kType, kDim> &q, int exponent) {
    const float inverse = __uint_as_float((unsigned)(127 - exponent) << 23);
    // 1.5 * 2^23 and a whole number up to 127 have that number in the last byte
    // of their sum, rounded to nearest even
    constexpr float kMagic = 12582912.f;
#pragma unroll
    for (int s = 0; s < kDim / 64; ++s)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float x[4];
        widen2<kType>(q.w[s][i >> 1][2 * (i & 1)], x[0], x[1]);
        widen2<kType>(q.w[s][i >> 1][2 * (i & 1) + 1], x[2], x[3]);
        unsigned n[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) n[j] = __float_as_uint(__builtin_fmaf(x[j], inverse, kMagic));
        const unsigned low = __builtin_amdgcn_perm(n[1], n[0], 0x0c0c0400u);
        const unsigned high = __builtin_amdgcn_perm(n[3], n[2], 0x04000c0cu);
        const unsigned all = low | high, negative = (all >> 7 & 0x01010101u) * 255u;
        plus[s][i] = (int)(all & ~negative);
        minus[s][i] = (int)(all & negative);
      }
  }
};

// The bounds of 16 blocks and a head as the second operand, from where they lie:
// lane % 16 is the block, lane / 16 its dims 16 (lane / 16) of each 64.  (Lines that
// a load takes whole, and an exchange in LDS, are 2 % faster to read, but cost more than that.)
template <int kDim>
struct BlockBounds {
  i4 upper[kDim / 64], lower[kDim / 64];
  float scale;
  __device__ __forceinline__ void fetch(const KvView &kv, int head, int slot, bool &bad) {
    const bool fine = (unsigned)slot < (unsigned)kv.num_slots;
    bad |= !fine;
    const char *const chunk = kv.base + (fine ? slot : 0) * kv.slot_stride;
    const char *const from = chunk + bounds_at(kv, head) + 16 * (lane_id() >> 4);
#pragma unroll
    for (int s = 0; s < kDim / 64; ++s) {
      upper[s] = *reinterpret_cast<const i4 *>(from + 64 * s);
      lower[s] = *reinterpret_cast<const i4 *>(from + kv.kv_stride + 64 * s);
    }
    scale = *reinterpret_cast<const float *>(chunk + scale_at(kv, head));
  }
};

// The larger of a lane's and that of the lane 16 or 32 further, for both.
__device__ __forceinline__ float larger16(float x) {
  const auto y = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(y[0]), __uint_as_float(y[1]));
}
__device__ __forceinline__ float larger32(float x) {
  const auto y = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(y[0]), __uint_as_float(y[1]));
}

template <int kTurn>
__device__ __forceinline__ float larger_turned(float x) {  // among the 16 lanes of a row
  const int y = __float_as_int(x);
  return fmaxf(x, __int_as_float(__builtin_amdgcn_update_dpp(y, y, 0x120 + kTurn, 0xf, 0xf, false)));
}
// The largest of a wave.
__device__ __forceinline__ float wave_largest(float x) {
  return larger32(larger16(larger_turned<1>(larger_turned<2>(larger_turned<4>(larger_turned<8>(x))))));
}

// A row set of a wave: whole queries, and where its tokens' scores go.  kWide: a
// set is a part (`part`) of one token's query heads.
template <int kType, int kDim, bool kWide>
struct RowSet {
  Operand<kDim> q;
  float weight[4];  // of rows 4 (lane / 16) .. relative to the largest of a token's; NaN where there is no head
  float *to;        // the score of the lane's first token and block lane % 16
  int left;         // tokens from there on

  static __device__ __forceinline__ int token_of(const Select &a, int tile) {
    return kWide ? tile : (tile << (4 - a.shift)) + ((lane_id() & 15) >> a.shift);
  }
  static __device__ __forceinline__ int head_of(const Select &a, int part) {
    const int n = lane_id() & 15;
    return kWide ? 16 * part + n : n & ((1 << a.shift) - 1);
  }
  static __device__ __forceinline__ bool valid(const Select &a, const KvRequest &r, int tile, int part) {
    return token_of(a, tile) < r.count && head_of(a, part) < a.group;
  }
  static __device__ __forceinline__ void load(Query<kType, kDim> &raw, const Select &a, const KvRequest &r, int head,
                                              int tile, int part) {
    raw.load(a, r, head, token_of(a, tile), head_of(a, part), valid(a, r, tile, part));
  }
  // `top_all`: the largest exponent of a token whose heads take several sets
  __device__ __forceinline__ void make(Query<kType, kDim> &raw, const Select &a, const KvRequest &r, int i, int head,
                                       int tile, int part, int top_all, bool &bad) {
    const int lane = lane_id(), g = lane >> 4, shift = kWide ? 4 : a.shift;
    const bool in = valid(a, r, tile, part);
    const int e = raw.exponent(bad);
    q.round(raw, e);
    // relative to the largest of the token's heads: every product is exact, and none overflows
    int top = in ? e : kMinExponent;
    for (int m = 1; m < 1 << shift; m <<= 1) top = max(top, __shfl_xor(top, m));
    if (kWide) top = top_all;
    // the larger of NaN and a number is the number
    const float w = in ? __uint_as_float((unsigned)(127 + max(e - top, -126)) << 23) : __builtin_nanf("");
#pragma unroll
    for (int k = 0; k < 4; ++k) weight[k] = __shfl(w, 4 * g + k);
    const int first = kWide ? tile : (tile << (4 - shift)) + (4 * g >> shift);
    to = scores_of(a, r, i, first, head) + (lane & 15);
    left = (4 * g & ((1 << shift) - 1)) == 0 ? r.count - first : 0;
  }
  // The products with 16 blocks' bounds of dims 64 s ..
  __device__ __forceinline__ i4 add(const i4 &upper, const i4 &lower, int s, i4 sum) const {
    sum = __builtin_amdgcn_mfma_i32_16x16x64_i8(q.plus[s], upper, sum, 0, 0, 0);
    return __builtin_amdgcn_mfma_i32_16x16x64_i8(q.minus[s], lower, sum, 0, 0, 0);
  }
  // The scores of 16 blocks from `b` on by the sums of their products with `kTiles` sets; `in`:
  // the lane's is one.  `next` lies between two tokens' scores.  `add`, `more`: of a token's heads
  // these are not the first, not the last.  The largest of all heads is scaled, not each part's: by a
  // scale that is not finite the larger of two scaled ones would be another.  (Step by step for all
  // sets, each of which has a step's latency to itself otherwise.)
  template <int kTiles>
  static __device__ __forceinline__ void score(const Select &a, const RowSet (&set)[kTiles], const i4 (&sum)[kTiles],
                                               float scale, int b, bool in, int64_t next, bool add, bool more) {
    const int shift = kWide ? 4 : a.shift;
    float x[kTiles][4];
#pragma unroll
    for (int t = 0; t < kTiles; ++t)
#pragma unroll
      for (int k = 0; k < 4; ++k) x[t][k] = (float)sum[t][k] * set[t].weight[k];
    // over the heads of a token: rows 4 (lane / 16) + k of the set
    auto put = [&](int k, const float (&x)[kTiles]) {
#pragma unroll
      for (int t = 0; t < kTiles; ++t) {
        float *const at = set[t].to + k * next + b;
        if (in && k < set[t].left) {
          const float y = kWide && add ? fmaxf(*at, x[t]) : x[t];
          *at = kWide && more ? y : __builtin_fmaf(y, scale, 0.f);  // no -0
        }
      }
    };
    float y[kTiles];
    if (shift >= 2) {
#pragma unroll
      for (int t = 0; t < kTiles; ++t) y[t] = fmaxf(fmaxf(x[t][0], x[t][1]), fmaxf(x[t][2], x[t][3]));
      if (shift >= 3) {
#pragma unroll
        for (int t = 0; t < kTiles; ++t) y[t] = larger16(y[t]);
      }
      if (shift >= 4) {
#pragma unroll
        for (int t = 0; t < kTiles; ++t) y[t] = larger32(y[t]);
      }
      put(0, y);
    } else if (shift == 1) {
#pragma unroll
      for (int k = 0; k < 4; k += 2) {
#pragma unroll
        for (int t = 0; t < kTiles; ++t) y[t] = fmaxf(x[t][k], x[t][k + 1]);
        put(k / 2, y);
      }
    } else {
#pragma unroll
      for (int k = 0; k < 4; ++k) {
#pragma unroll
        for (int t = 0; t < kTiles; ++t) y[t] = x[t][k];
        put(k, y);
      }
    }
  }
};

// The scores of a wave's row set over blocks begin .. end of request i, 16 blocks
// a step: it is the other waves that keep memory busy.  A token whose heads
// take several sets has them one after another.
template <int kType, int kDim, bool kWide>
__device__ __forceinline__ void score_blocks(const Select &a, const KvRequest &r, int i, int head, int tile,
                                             int begin, int end) {
  const int n16 = lane_id() & 15, parts = kWide ? a.padded / 16 : 1;
  const int32_t *const slots = a.slots + r.row;
  const int64_t next = (int64_t)a.kv.kv_heads * score_pitch(a, r);
  bool bad_query = false, bad_slot = false;
  auto look = [&](int b0) { return slots[min(b0 + n16, end - 1)]; };
  int top_all = kMinExponent;
  if (kWide) {
    for (int p = 0; p < parts; ++p) {
      Query<kType, kDim> raw;
      RowSet<kType, kDim, kWide>::load(raw, a, r, head, tile, p);
      const int e = raw.exponent(bad_query);
      top_all = max(top_all, RowSet<kType, kDim, kWide>::valid(a, r, tile, p) ? e : kMinExponent);
    }
#pragma unroll
    for (int m = 8; m; m >>= 1) top_all = max(top_all, __shfl_xor(top_all, m));
  }
  for (int p = 0; p < parts; ++p) {
    int slot = look(begin);
    BlockBounds<kDim> bounds;
    RowSet<kType, kDim, kWide> sets[1], &set = sets[0];
    {
      Query<kType, kDim> raw;
      set.load(raw, a, r, head, tile, p);
      bounds.fetch(a.kv, head, slot, bad_slot);
      slot = look(begin + 16);
      set.make(raw, a, r, i, head, tile, p, top_all, bad_query);
    }
#pragma unroll 1
    for (int b0 = begin; b0 < end; b0 += 16) {
      i4 sum[1] = {i4{0, 0, 0, 0}};
#pragma unroll
      for (int s = 0; s < kDim / 64; ++s) sum[0] = set.add(bounds.upper[s], bounds.lower[s], s, sum[0]);
      set.score(a, sets, sum, bounds.scale, b0, b0 + n16 < end, next, p > 0, p + 1 < parts);
      if (b0 + 16 < end) {
        bounds.fetch(a.kv, head, slot, bad_slot);
        slot = look(b0 + 32);
      }
    }
  }
  if (__any(bad_query || bad_slot)) kv_report(a.status);
}

// The bounds of a stage of 32 blocks and a head in LDS, for all waves: each brings
// those of 8 blocks, by whole lines (16 lanes that ask for 16 blocks are answered one
// line at a time, which with several row sets a block took longer than the products).
template <int kDim>
struct BoundStage {
  static constexpr int kBlocks = 32, kMine = kBlocks / kWaves, kChunks = kDim / 16, kLoads = kDim / 64;
  static constexpr int kSlots = kDim == 256 ? 2 : 1;  // a lane's loads of a side are of as many blocks
  static constexpr int kBytes = 2 * kBlocks * kDim + 4 * kBlocks;
  u4 raw[kLoads];
  float scale;
  int slot[kSlots], scale_slot;
  // of load k: the side, the block among the wave's, the chunk of 16 bytes
  static __device__ __forceinline__ int side_of(int k) { return (64 * k + lane_id()) / (kMine * kChunks); }
  static __device__ __forceinline__ int block_of(int k) { return (64 * k + lane_id()) / kChunks % kMine; }
  static __device__ __forceinline__ int chunk_of() { return lane_id() % kChunks; }
  // 16 lanes that read a chunk of 16 blocks meet few banks twice
  static __device__ __forceinline__ int place(int side, int block, int chunk) {
    const int turn = kDim == 64 ? block >> 1 & 3 : block & (kChunks - 1);
    return side * kBlocks * kDim + (block * kChunks + (chunk ^ turn)) * 16;
  }
  __device__ __forceinline__ void look(const int32_t *slots, int b0, int end) {
    const int first = b0 + kMine * wave_id();
#pragma unroll
    for (int k = 0; k < kSlots; ++k) slot[k] = slots[min(first + block_of(k), end - 1)];
    scale_slot = slots[min(first + lane_id() % kMine, end - 1)];
  }
  __device__ __forceinline__ void fetch(const KvView &kv, int head, bool &bad) {
    const char *const from = kv.base + bounds_at(kv, head) + 16 * chunk_of();
#pragma unroll
    for (int k = 0; k < kLoads; ++k) {
      const int s = slot[k % kSlots];
      const bool fine = (unsigned)s < (unsigned)kv.num_slots;
      bad |= !fine;
      raw[k] = *reinterpret_cast<const u4 *>(from + (fine ? s : 0) * kv.slot_stride + side_of(k) * kv.kv_stride);
    }
    const int s = (unsigned)scale_slot < (unsigned)kv.num_slots ? scale_slot : 0;
    scale = *reinterpret_cast<const float *>(kv.base + scale_at(kv, head) + s * kv.slot_stride);
  }
  __device__ __forceinline__ void put(char *lds) const {
    const int first = kMine * wave_id();
#pragma unroll
    for (int k = 0; k < kLoads; ++k)
      *reinterpret_cast<u4 *>(lds + place(side_of(k), first + block_of(k), chunk_of())) = raw[k];
    if (lane_id() < kMine) reinterpret_cast<float *>(lds + 2 * kBlocks * kDim)[first + lane_id()] = scale;
  }
  static __device__ __forceinline__ void get(const char *lds, int half, i4 (&upper)[kLoads], i4 (&lower)[kLoads],
                                             float &scale) {
    const int block = 16 * half + (lane_id() & 15), g = lane_id() >> 4;
#pragma unroll
    for (int s = 0; s < kLoads; ++s) {
      upper[s] = *reinterpret_cast<const i4 *>(lds + place(0, block, 4 * s + g));
      lower[s] = *reinterpret_cast<const i4 *>(lds + place(1, block, 4 * s + g));
    }
    scale = reinterpret_cast<const float *>(lds + 2 * kBlocks * kDim)[block];
  }
};

// The scores of `kTiles` row sets a wave, neighbouring ones of a head, over blocks
// begin .. end.  Called by all waves; `lds` holds two stages.
template <int kType, int kDim, int kTiles>
__device__ __forceinline__ void score_sets(const Select &a, const KvRequest &r, int i, int head, int tile0, int begin,
                                           int end, char *lds) {
  typedef BoundStage<kDim> Stage;
  const int32_t *const slots = a.slots + r.row;
  const int64_t next = (int64_t)a.kv.kv_heads * score_pitch(a, r);
  bool bad_query = false, bad_slot = false;
  Stage stage;
  RowSet<kType, kDim, false> set[kTiles];
  stage.look(slots, begin, end);
  {
    Query<kType, kDim> raw[kTiles];
#pragma unroll
    for (int t = 0; t < kTiles; ++t) set[t].load(raw[t], a, r, head, tile0 + t, 0);
    stage.fetch(a.kv, head, bad_slot);
    stage.look(slots, begin + Stage::kBlocks, end);
#pragma unroll
    for (int t = 0; t < kTiles; ++t) set[t].make(raw[t], a, r, i, head, tile0 + t, 0, 0, bad_query);
  }
  char *from = lds, *to = lds + Stage::kBytes;
  __syncthreads();  // what was read of it before
  stage.put(from);
  stage.fetch(a.kv, head, bad_slot);  // past the end the last block's
  stage.look(slots, begin + 2 * Stage::kBlocks, end);
  __syncthreads();
#pragma unroll 1
  for (int b0 = begin; b0 < end; b0 += Stage::kBlocks) {
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      const int b = b0 + 16 * half;
      i4 upper[kDim / 64], lower[kDim / 64];
      float scale;
      Stage::get(from, half, upper, lower, scale);
      i4 sum[kTiles];  // a product waits for the one before it: those of other sets go between
#pragma unroll
      for (int t = 0; t < kTiles; ++t) sum[t] = i4{0, 0, 0, 0};
#pragma unroll
      for (int s = 0; s < kDim / 64; ++s)
#pragma unroll
        for (int t = 0; t < kTiles; ++t) sum[t] = set[t].add(upper[s], lower[s], s, sum[t]);
      set[0].score(a, set, sum, scale, b, b + (lane_id() & 15) < end, next, false, false);
    }
    stage.put(to);
    stage.fetch(a.kv, head, bad_slot);
    stage.look(slots, b0 + 3 * Stage::kBlocks, end);
    __syncthreads();
    char *const was = from;
    from = to;
    to = was;
  }
  if (__any(bad_query || bad_slot)) kv_report(a.status);
}

// The blocks of a request that have to be scored: none if its last token keeps
// all that it sees.
struct Candidates {
  int begin, end;
  __device__ __forceinline__ Candidates(const Select &a, int blocks) : begin(a.sink), end(blocks - a.recent) {
    if (blocks <= a.keep) end = begin;
  }
};

// Neighbouring pieces of work on one XCD (workgroups go to the 8 in turn; blockIdx.x is one of a multiple of 8).
__device__ __forceinline__ int piece() { return (blockIdx.x & 7) * (gridDim.x >> 3) + (blockIdx.x >> 3); }

// Entries span .. of the table, the requests in them one after another, with the
// tokens of the run as their new ones.  Requests up to where offsets fall: their entries and
// scores are in order and apart, whatever comes behind them.
template <typename F>
__device__ __forceinline__ void each_request(const Select &a, int span, int first_token, int *lds, F f) {
  if ((int64_t)span * a.span >= a.batch.n_entries) return;
  const int e0 = span * a.span, e1 = e0 + min(a.span, a.batch.n_entries - e0);
  int first[2];  // that ends behind e0, and whose end is before its begin
  first_of(a.batch.n, first, lds, [&](int i, bool (&found)[2]) {
    const int end = a.row_offsets[i + 1];
    found[0] = end > e0;
    found[1] = (end < a.row_offsets[i]) | (a.batch.token_offsets[i + 1] < a.batch.token_offsets[i]);
  });
  const int limit = __builtin_amdgcn_readfirstlane(first[1]);
  if (blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) *a.limit = limit;
  for (int i = __builtin_amdgcn_readfirstlane(first[0]); i < limit && uniform_load(a.row_offsets + i) < e1; ++i) {
    KvRequest r = kv_request<true>(a.batch, a.row_offsets, a.kv.block_shift, i);
    r.first += a.first;
    r.count = min(r.count - a.first, a.run);
    const int blocks = blocks_of(r, a.kv.block_shift);
    if (!r.ok || blocks > a.most || first_token >= r.count) continue;
    const Candidates c(a, blocks);
    const int begin = max(c.begin, e0 - r.row), end = min(c.end, e1 - r.row);
    if (begin < end) f(r, i, begin, end);
  }
}

// A row set to a wave, which takes heads, or parts of the entries where there
// are few heads, so that what lies side by side is read at one time.
template <int kType, int kDim, bool kWide>
__global__ __launch_bounds__(kBlock, kDim == 256 ? 2 : 5) void score_kernel(Select a) {
  __shared__ int owners[2 * kWaves];
  const int wave = __builtin_amdgcn_readfirstlane(wave_id()), tile = blockIdx.y;
  each_request(a, piece(), tile * (16 >> a.shift), owners, [&](const KvRequest &r, int i, int begin, int end) {
    const int heads = a.kv.kv_heads, parts = heads >= kWaves ? 1 : kWaves / heads;
    const int each = ((end - begin + 16 * parts - 1) / (16 * parts)) * 16;
    for (int u = wave; u < heads * parts; u += kWaves) {
      const int from = begin + u / heads * each, to = min(from + each, end);
      if (from < to) score_blocks<kType, kDim, kWide>(a, r, i, u % heads, tile, from, to);
    }
  });
}

// Many row sets: `kTiles` to a wave, of one head.  An XCD has one head, or few, whose queries and
// bounds are then in its L2.
template <int kType, int kDim, int kTiles>
__global__ __launch_bounds__(kBlock, 2) void score_sets_kernel(Select a) {
  __shared__ int owners[2 * kWaves];
  __shared__ alignas(16) char stages[2 * BoundStage<kDim>::kBytes];
  const int wave = __builtin_amdgcn_readfirstlane(wave_id());
  const int at = piece(), head = at / (a.spans * a.sets), tile0 = at / a.spans % a.sets * kWaves * kTiles;
  if (head >= a.kv.kv_heads) return;
  each_request(a, at % a.spans, tile0 * (16 >> a.shift), owners, [&](const KvRequest &r, int i, int begin, int end) {
    score_sets<kType, kDim, kTiles>(a, r, i, head, tile0 + wave * kTiles, begin, end, stages);
  });
}

// ------------------------------------------------------------------ select

// Scores in ascending order as whole numbers above 0 and below 2^32 - 1, NaN last.
__device__ __forceinline__ unsigned ordered(float x) {
  const unsigned b = __float_as_uint(x);
  if ((b & 0x7fffffffu) > 0x7f800000u) return 0xfffffffeu;
  return b >> 31 ? ~b : b | 0x80000000u;
}

// A list's candidates, begin .. end, of which `want` stay beside the first `sink`
// and the last `recent` blocks; none if there is no choice.
struct Row {
  const float *score;
  int32_t *out;
  int begin, end, want;
};

// The row of token and KV head `row`, with what needs no choice written by
// threads `lane` of `width`.
__device__ __forceinline__ Row row_of(const Select &a, const KvRequest &q, int i, int token, int head, int lane,
                                      int width) {
  Row r = {nullptr, nullptr, 0, 0, 0};
  const int j = token - q.first, last = q.len - q.count + j;  // cached token
  const int blocks = last < 0 ? 0 : (last >> a.kv.block_shift) + 1;
  r.out = a.selected + ((int64_t)token * a.kv.kv_heads + head) * a.keep;
  if (blocks <= a.keep) {
    for (int k = lane; k < a.keep; k += width) r.out[k] = k < blocks ? k : -1;
  } else {
    KvRequest run = q;  // as each_request has it
    run.first += a.first;
    r.score = scores_of(a, run, i, j - a.first, head);
    r.begin = a.sink, r.end = blocks - a.recent, r.want = a.keep - a.sink - a.recent;
    for (int k = lane; k < a.sink; k += width) r.out[k] = k;
    for (int k = lane; k < a.recent; k += width) r.out[a.keep - a.recent + k] = r.end + k;
  }
  return r;
}

// The least key that stays, by its digits of 11, 11 and 10 bits from the front:
// histograms in LDS, with a place for what a lane does not count.
constexpr int kDigits = 2048;
typedef unsigned Hist[kDigits + 64];
__device__ __forceinline__ int digit_shift(int pass) { return pass == 0 ? 21 : pass == 1 ? 10 : 0; }
__device__ __forceinline__ unsigned digit_mask(int pass) { return pass == 2 ? 1023u : 2047u; }

// The digit of the key that has `rank` before it, largest first; `rank` becomes its
// rank among the `count` with that digit.
__device__ __forceinline__ unsigned find_digit(const unsigned *hist, unsigned &rank, unsigned &count) {
  const int lane = lane_id();
  // 32 digits to a lane, from the largest; lanes begin at different ones, as they share banks
  unsigned sum = 0;
  const unsigned *const high = hist + kDigits - 32 * (lane + 1);
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const uint4 h = *reinterpret_cast<const uint4 *>(high + 4 * ((j + lane) & 7));
    sum += (h.x + h.y) + (h.z + h.w);
  }
  unsigned before = wave_inclusive_sum(sum) - sum;
  int from = __ffsll((unsigned long long)__ballot(rank >= before && rank < before + sum)) - 1;
  rank -= lane_value(before, from);
  // and of those a digit to a lane
  const int top = kDigits - 1 - 32 * from;
  sum = lane < 32 ? hist[top - lane] : 0;
  before = wave_inclusive_sum(sum) - sum;
  from = __ffsll((unsigned long long)__ballot(rank >= before && rank < before + sum)) - 1;
  rank -= lane_value(before, from);
  count = lane_value(sum, from);
  return top - from;
}

struct Threshold {
  unsigned key = 0, known = 0;  // its digits so far
  unsigned rank;                // of it among those that share them
  unsigned equal = ~0u;         // how many of the keys that share all known digits stay

  // Keys of no candidate are 0.
  __device__ __forceinline__ void count(unsigned *hist, int pass, unsigned x) const {
    const bool in = x && ((x ^ key) & known) == 0;
    atomicAdd(&hist[in ? x >> digit_shift(pass) & digit_mask(pass) : kDigits + lane_id()], 1u);
  }
  // Takes the next digit; false if it is the last that is needed.  By each wave for itself.
  __device__ __forceinline__ bool next(const unsigned *hist, int pass) {
    unsigned count;
    key |= find_digit(hist, rank, count) << digit_shift(pass);
    known |= digit_mask(pass) << digit_shift(pass);
    const bool all = rank + 1 == count;  // that share these digits stay
    equal = all ? ~0u : rank + 1;        // or the first of them
    return !all && pass < 2;
  }
};

__device__ __forceinline__ void wave_sync() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// The first request that is not taken.
__device__ __forceinline__ int limit_of(const Select &a) {
  const int limit = uniform_load(a.limit);
  return a.scored ? limit : a.batch.n;
}
// Whether a token is a new one of request i.
__device__ __forceinline__ bool has(const KvRequest &q, int i, int limit, int token) {
  return q.ok && i < limit && token >= q.first && token - q.first < q.count;
}
// Whether it is one of the run; reports a request of too many blocks.
__device__ __forceinline__ bool in_run(const Select &a, const KvRequest &q, int token) {
  if (blocks_of(q, a.kv.block_shift) > a.most) {
    kv_report(a.status);
    return false;
  }
  return (unsigned)(token - q.first - a.first) < (unsigned)a.run;
}

// Writes those of 64 blocks that stay, in order, and moves on: the ones above the
// threshold and the first of the ones at it.
__device__ __forceinline__ void put(const Row &r, uint64_t above, uint64_t at, unsigned equal, int first,
                                    unsigned &place, unsigned &ties) {
  if (!(above | at)) return;
  const bool tie = (at >> lane_id() & 1) && ties + rank_in_mask(at) < equal;
  const uint64_t stay = above | __ballot(tie);
  if (stay >> lane_id() & 1) r.out[place + rank_in_mask(stay)] = first + lane_id();
  place += __popcll(stay);
  ties += __popcll(at);
}
__device__ __forceinline__ void put(const Row &r, const Threshold &t, unsigned x, int first, unsigned &place,
                                    unsigned &ties) {
  put(r, __ballot((x & t.known) > t.key), __ballot((x & t.known) == t.key), t.equal, first, place, ties);
}

// The score with `rank` before it, largest first, of up to 64 finite ones in LDS, and how many of those
// equal to it stay.
struct Few {
  float threshold;
  unsigned equal;
  __device__ __forceinline__ Few(const float *few, unsigned count, unsigned rank) {
    const int lane = lane_id();
    const float mine = lane < (int)count ? few[lane] : -__builtin_inff();
    unsigned above = 0, at = 0;
    for (int j = 0; j < (int)count; ++j) {
      const float other = few[j];
      above += other > mine, at += other == mine;
    }
    const int from = __ffsll((unsigned long long)__ballot(rank >= above && rank < above + at)) - 1;
    threshold = __shfl(mine, from);
    equal = rank + 1 - lane_value(above, from);
  }
};

// A token and head to a wave, its candidates in registers, no barriers: for
// many rows.
constexpr int kHeld = 32, kRun = 16;  // registers, and those between two looks at the row's end
__global__ __launch_bounds__(kBlock) void select_wave_kernel(Select a) {
  if (blockIdx.x == gridDim.x - 1) {
    check_requests(a.batch, a.row_offsets, a.kv.block_shift, a.status);
    return;
  }
  __shared__ alignas(16) Hist hists[kWaves];
  __shared__ int owners[kWaves];
  const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(wave_id());
  const int limit = limit_of(a);
  const int64_t row = (int64_t)blockIdx.x * kWaves + wave;
  const int token = (int)(row / a.kv.kv_heads), head = (int)(row % a.kv.kv_heads);
  int i = owner_of(a.batch.token_offsets, a.batch.n, (int)((int64_t)blockIdx.x * kWaves / a.kv.kv_heads), owners);
  while (i < a.batch.n && a.batch.token_offsets[i + 1] <= token) ++i;
  if (i >= a.batch.n || token >= a.batch.n_tokens) return;
  const KvRequest q = kv_request(a.batch, a.row_offsets, a.kv.block_shift, i);
  if (!has(q, i, limit, token) || !in_run(a, q, token)) return;
  const Row r = row_of(a, q, i, token, head, lane, 64);
  if (r.want == 0) return;
  const int m = __builtin_amdgcn_readfirstlane(r.end - r.begin);
  float x[kHeld];
  auto each_run = [&](auto f) {
#pragma unroll
    for (int k0 = 0; k0 < kHeld; k0 += kRun) {
      if (64 * k0 >= m) break;
#pragma unroll
      for (int k = k0; k < k0 + kRun; ++k) f(k);
    }
  };
  float least = __builtin_inff(), most = -__builtin_inff();
  bool odd = false;  // a score that is no number
  each_run([&](int k) {
    x[k] = r.score[r.begin + min(64 * k + lane, m - 1)];
    odd |= !__builtin_isfinite(x[k]);
  });
  each_run([&](int k) {
    least = fminf(least, x[k]), most = fmaxf(most, x[k]);
    x[k] = 64 * k + lane < m ? x[k] : __builtin_nanf("");  // no candidate
  });
  unsigned *const hist = hists[wave];
  auto clear = [&] {
#pragma unroll
    for (int j = 0; j < kDigits / 256; ++j) reinterpret_cast<uint4 *>(hist)[64 * j + lane] = uint4{0, 0, 0, 0};
    wave_sync();
  };
  clear();
  // equal parts of the scores' range as digits: fewer scores share one than share
  // 11 bits, adds to one place in LDS take turns, and one pass leaves few
  least = -wave_largest(-least), most = wave_largest(most);
  const float per = (kDigits - 1) / (most - least);
  unsigned place = a.sink, ties = 0;
  if (!__any(odd) && __builtin_isfinite(per)) {
    unsigned place_of[kHeld];  // a place behind the digits is no candidate's
    each_run([&](int k) {
      const unsigned digit = min((unsigned)((x[k] - least) * per), kDigits - 1u);
      place_of[k] = 64 * k + lane < m ? digit : kDigits + lane;
      atomicAdd(&hist[place_of[k]], 1u);
    });
    wave_sync();
    unsigned rank = r.want - 1, count;
    const unsigned digit = find_digit(hist, rank, count);
    if (count <= 64) {
      wave_sync();
      float *const few = reinterpret_cast<float *>(hist);
      unsigned n = 0;
      each_run([&](int k) {
        const uint64_t in = __ballot(place_of[k] == digit);
        if (!in) return;
        if (in >> lane & 1) few[n + rank_in_mask(in)] = x[k];
        n += __popcll(in);
      });
      wave_sync();
      const Few found(few, count, rank);
      each_run([&](int k) {
        put(r, __ballot(x[k] > found.threshold), __ballot(x[k] == found.threshold), found.equal, r.begin + 64 * k,
            place, ties);
      });
      return;
    }
    wave_sync();
    clear();
  }
  Threshold t;
  t.rank = r.want - 1;
  auto key_of = [&](int k) { return 64 * k + lane < m ? ordered(r.score[r.begin + 64 * k + lane]) : 0; };
#pragma unroll 1
  for (int pass = 0;; ++pass) {
    for (int k = 0; 64 * k < m; ++k) t.count(hist, pass, key_of(k));
    wave_sync();
    if (!t.next(hist, pass)) break;
    wave_sync();
    clear();
  }
  for (int k = 0; 64 * k < m; ++k) put(r, t, key_of(k), r.begin + 64 * k, place, ties);
}

// A token and head to a workgroup: for few rows, or long ones.  A wave has a
// run of candidates, 64 at a time, the first kKept of them in registers.
template <int kKept>
__global__ __launch_bounds__(kBlock) void select_block_kernel(Select a) {
  if (blockIdx.x == gridDim.x - 1) {
    check_requests(a.batch, a.row_offsets, a.kv.block_shift, a.status);
    return;
  }
  __shared__ alignas(16) Hist hists[3];
  __shared__ int owners[kWaves];
  __shared__ unsigned marks[2][kWaves], listed;
  __shared__ float widths[2][kWaves];
  const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(wave_id());
  const int token = blockIdx.x / a.kv.kv_heads, head = blockIdx.x % a.kv.kv_heads;
  auto clear = [&](Hist &h) {
    for (int d = threadIdx.x; d < (int)(sizeof(Hist) / 16); d += kBlock)
      reinterpret_cast<uint4 *>(h)[d] = uint4{0, 0, 0, 0};
  };
  for (Hist &h : hists) clear(h);
  if (threadIdx.x == 0) listed = 0;
  // single tokens are their requests' numbers, and one request has them all: look there first
  const int limit = limit_of(a);
  int i = min(token, a.batch.n - 1);
  KvRequest q = kv_request<true>(a.batch, a.row_offsets, a.kv.block_shift, i);
  if (!has(q, i, limit, token)) {
    i = __builtin_amdgcn_readfirstlane(owner_of(a.batch.token_offsets, a.batch.n, token, owners));
    if (i >= a.batch.n) return;
    q = kv_request<true>(a.batch, a.row_offsets, a.kv.block_shift, i);
    if (!has(q, i, limit, token)) return;
  }
  if (!in_run(a, q, token)) return;
  const Row r = row_of(a, q, i, token, head, threadIdx.x, kBlock);
  if (r.want == 0) return;
  if (r.end - r.begin <= 64) {  // one wave's, a score to a lane: how many are above it?
    if (wave) return;
    const int m = r.end - r.begin;
    const unsigned x = lane < m ? ordered(r.score[r.begin + lane]) : 0;
    unsigned above = 0;
#pragma unroll 8
    for (int j = 0; j < m; ++j) above += lane_value(x, j) > x;
    uint64_t stay = __ballot(lane < m && above < (unsigned)r.want);
    if (__popcll(stay) > r.want) {  // the last of them are equal: the first of these
      const unsigned last = (unsigned)wave_largest(stay >> lane & 1 ? (float)above : 0.f);
      const uint64_t at = __ballot(lane < m && above == last);
      stay &= ~at;
      const bool tie = (at >> lane & 1) && (int)rank_in_mask(at) < r.want - __popcll(stay);
      stay |= __ballot(tie);
    }
    if (stay >> lane & 1) r.out[a.sink + rank_in_mask(stay)] = r.begin + lane;
    return;
  }
  const int each = ((r.end - r.begin + kBlock - 1) / kBlock) * 64;
  const int from = __builtin_amdgcn_readfirstlane(min(r.begin + wave * each, r.end));
  const int to = __builtin_amdgcn_readfirstlane(min(from + each, r.end));
  float kept[kKept];
#pragma unroll
  for (int k = 0; k < kKept; ++k) kept[k] = from + 64 * k < to ? r.score[min(from + 64 * k + lane, to - 1)] : 0.f;
  // f(score, whether it is one, block of lane 0)
  auto each_score = [&](auto f) {
#pragma unroll
    for (int k = 0; k < kKept; ++k)
      if (from + 64 * k < to) f(kept[k], from + 64 * k + lane < to, from + 64 * k);
    for (int b0 = from + 64 * kKept; b0 < to; b0 += 64) f(r.score[min(b0 + lane, to - 1)], b0 + lane < to, b0);
  };
  // where the waves before this one put theirs, by what each has above the threshold and at it
  unsigned place = a.sink, ties = 0;
  auto begin_at = [&](unsigned above, unsigned at, unsigned equal) {
    if (lane == 0) marks[0][wave] = above, marks[1][wave] = at;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      if (w < wave) {
        place += marks[0][w] + min(marks[1][w], equal - min(equal, ties));
        ties += marks[1][w];
      }
    }
  };

  // equal parts of the scores' range as digits, as in select_wave_kernel
  float least = __builtin_inff(), most = -__builtin_inff();
  bool odd = false;
  each_score([&](float x, bool, int) {
    odd |= !__builtin_isfinite(x);
    least = fminf(least, x), most = fmaxf(most, x);
  });
  if (__any(odd)) least = -__builtin_inff(), most = __builtin_inff();
  least = -wave_largest(-least), most = wave_largest(most);
  if (lane == 0) widths[0][wave] = least, widths[1][wave] = most;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kWaves; ++w) least = fminf(least, widths[0][w]), most = fmaxf(most, widths[1][w]);
  const float width = most - least, per = (kDigits - 1) / width;
  if (__builtin_isfinite(width) && __builtin_isfinite(per)) {
    auto digit_of = [&](float x) { return min((unsigned)((x - least) * per), kDigits - 1u); };
    each_score([&](float x, bool in, int) { atomicAdd(&hists[0][in ? digit_of(x) : kDigits + lane], 1u); });
    __syncthreads();
    unsigned rank = r.want - 1, count;
    const unsigned digit = find_digit(hists[0], rank, count);
    if (count <= 64) {
      float *const few = reinterpret_cast<float *>(hists[1]);  // in any order
      each_score([&](float x, bool in, int) {
        const uint64_t these = __ballot(in && digit_of(x) == digit);
        if (!these) return;
        unsigned first = 0;
        if (lane == 0) first = atomicAdd(&listed, (unsigned)__popcll(these));
        first = __builtin_amdgcn_readfirstlane(first);
        if (these >> lane & 1) few[first + rank_in_mask(these)] = x;
      });
      __syncthreads();
      const Few found(few, count, rank);
      unsigned above = 0, at = 0;
      each_score([&](float x, bool in, int) {
        above += __popcll(__ballot(in && x > found.threshold));
        at += __popcll(__ballot(in && x == found.threshold));
      });
      begin_at(above, at, found.equal);
      each_score([&](float x, bool in, int first) {
        put(r, __ballot(in && x > found.threshold), __ballot(in && x == found.threshold), found.equal, first, place,
            ties);
      });
      return;
    }
  }
  // the scores' bits, where that leaves many or there is no range; rare, so kept small
  auto each_key = [&](auto f) {
#pragma unroll 1
    for (int b0 = from; b0 < to; b0 += 64) f(b0 + lane < to ? ordered(r.score[b0 + lane]) : 0u, b0);
  };
  Threshold t;
  t.rank = r.want - 1;
#pragma unroll 1
  for (int pass = 0;; ++pass) {
    if (pass == 1) clear(hists[0]);  // for the last pass
    unsigned *const hist = hists[(pass + 1) % 3];
    each_key([&](unsigned x, int) { t.count(hist, pass, x); });
    __syncthreads();
    if (!t.next(hist, pass)) break;
  }
  unsigned above = 0, at = 0;
  each_key([&](unsigned x, int) {
    above += __popcll(__ballot((x & t.known) > t.key));
    at += __popcll(__ballot((x & t.known) == t.key));
  });
  begin_at(above, at, t.equal);
  each_key([&](unsigned x, int first) { put(r, t, x, first, place, ties); });
}

// ------------------------------------------------------------------- host

bool bounds_fit(const cascade_kv_pool_t *p, const cascade_kv_format_t *f) {
  return p->chunk_bytes >= kv_chunk_bytes(f) + (int64_t)f->kv_heads * f->head_dim;
}

// Places for the scores of one new token of each request.
size_t score_bytes(const cascade_kv_format_t *f, const cascade_kv_batch_t *b) {
  return sizeof(float) * ((size_t)b->n_entries + 16 * (size_t)b->n) * f->kv_heads;
}
constexpr size_t kRoom = 256;      // of a workspace before them
constexpr int kMostRun = 32768;    // new tokens of a request that are scored at one time: a grid's second dimension
// The most new tokens of a request.
int most_tokens(const cascade_kv_batch_t *b) { return std::min(b->max_new, b->n_tokens); }

// Row sets of a wave where there are many: what its registers hold.
constexpr int many_sets(int dim) { return dim == 256 ? 2 : 4; }

template <int kType, int kDim>
void score(const Select &a, bool many, dim3 grid, hipStream_t stream) {
  auto kernel = a.padded > 16 ? score_kernel<kType, kDim, true>
                : many        ? score_sets_kernel<kType, kDim, many_sets(kDim)>
                              : score_kernel<kType, kDim, false>;
  hipLaunchKernelGGL(kernel, grid, dim3(kBlock), 0, stream, a);
}
template <int kType>
void score(const Select &a, bool many, dim3 grid, hipStream_t stream) {
  switch (a.kv.head_dim) {
    case 64: score<kType, 64>(a, many, grid, stream); break;
    case 128: score<kType, 128>(a, many, grid, stream); break;
    default: score<kType, 256>(a, many, grid, stream);
  }
}

}  // namespace
}  // namespace cascade

using namespace cascade;

extern "C" size_t cascade_kv_bounds_bytes(const cascade_kv_format_t *format) {
  return kv_format_ok(format) ? (size_t)format->kv_heads * format->head_dim : 0;
}

extern "C" int cascade_kv_bounds(const cascade_kv_pool_t *pool, int32_t layer, const cascade_kv_format_t *format,
                                 const cascade_kv_batch_t *batch, const cascade_block_table_t *table, int32_t whole,
                                 int32_t *status_dev, void *stream) {
  if (!kv_pool_ok(pool, layer, format) || !bounds_fit(pool, format) || !kv_batch_ok(batch, table) ||
      (whole != 0 && whole != 1))
    return CASCADE_EINVAL;
  Bounds a = {};
  a.units = whole ? batch->n_entries : batch->n_tokens;
  if (batch->n == 0 || a.units == 0) return CASCADE_OK;
  a.kv = kv_view(pool, layer, format);
  a.batch = *batch;
  a.row_offsets = table->row_offsets;
  a.slots = table->slots;
  a.whole = whole;
  a.group = a.units <= 2048 ? 1 : whole ? 4 : 16;
  while ((a.units - 1) / a.group >= INT32_MAX / kBlock - 1) a.group *= 2;  // a launch has below 2^32 threads
  a.status = status_dev;
  const int grid = (a.units - 1) / a.group + 2;  // the last one checks the batch
  auto kernel = format->head_dim == 64    ? bounds_kernel<64>
                : format->head_dim == 128 ? bounds_kernel<128>
                                          : bounds_kernel<256>;
  // few workgroups: a head to a wave
  const int heads = grid <= 1024 ? (format->kv_heads + kWaves - 1) / kWaves : 1;
  hipLaunchKernelGGL(kernel, dim3(grid, heads), dim3(kBlock), 0, static_cast<hipStream_t>(stream), a);
  return hipGetLastError() == hipSuccess ? CASCADE_OK : CASCADE_EHIP;
}

extern "C" size_t cascade_kv_select_workspace_bytes(const cascade_kv_format_t *format,
                                                    const cascade_kv_batch_t *batch) {
  if (!kv_format_ok(format) || !batch || batch->n < 0 || batch->max_new < 0 || batch->n_tokens < 0 ||
      batch->n_entries < 0)
    return 0;
  return score_bytes(format, batch) * std::min(most_tokens(batch), kMostRun) + kRoom;
}

extern "C" int cascade_kv_select(const cascade_kv_pool_t *pool, int32_t layer, const cascade_kv_format_t *format,
                                 const cascade_kv_batch_t *batch, const cascade_block_table_t *table,
                                 const cascade_select_t *args, void *workspace, size_t workspace_bytes,
                                 int32_t *status_dev, void *stream) {
  if (!kv_pool_ok(pool, layer, format) || !bounds_fit(pool, format) || !kv_batch_ok(batch, table) || !args)
    return CASCADE_EINVAL;
  if ((args->dtype != CASCADE_BF16 && args->dtype != CASCADE_F16) || args->q_heads < 1 ||
      args->q_heads % format->kv_heads || args->q_heads / format->kv_heads > 128 || args->sink < 0 ||
      args->recent < 1 || args->most_blocks < 0 || args->keep > 65536 ||
      (int64_t)args->sink + args->recent > args->keep)
    return CASCADE_EINVAL;
  if (!workspace || ((uintptr_t)workspace & 255)) return CASCADE_EINVAL;
  const int64_t rows = (int64_t)batch->n_tokens * format->kv_heads;
  if (rows >= INT32_MAX / kBlock) return CASCADE_EINVAL;
  // by tokens where that takes less, and is known to fit
  const size_t one = score_bytes(format, batch), all = one * std::min(most_tokens(batch), kMostRun);
  const int64_t lines = ((int64_t)args->most_blocks + 15) & ~15;
  const size_t by_tokens = sizeof(float) * rows * lines;
  const bool known = args->most_blocks > 0 && by_tokens <= all && workspace_bytes >= by_tokens + kRoom;
  if (!known && workspace_bytes < one * std::min(most_tokens(batch), 1) + kRoom) return CASCADE_ENOSPC;
  if (batch->n == 0 || batch->n_tokens == 0 || batch->max_new == 0) return CASCADE_OK;
  if (!kv_rows_ok(&args->q) || !args->selected) return CASCADE_EINVAL;
  Select a = {};
  a.kv = kv_view(pool, layer, format);
  a.batch = *batch;
  a.row_offsets = table->row_offsets;
  a.slots = table->slots;
  a.q = QRows{static_cast<const char *>(args->q.data), 2 * args->q.token_stride, 2 * args->q.head_stride};
  a.group = args->q_heads / format->kv_heads;
  a.padded = a.group > 16 ? (a.group + 15) & ~15 : 1;
  while (a.padded < a.group) a.padded *= 2;
  a.shift = a.padded >= 16 ? 4 : __builtin_ctz((unsigned)a.padded);
  a.keep = args->keep;
  a.sink = args->sink;
  a.recent = args->recent;
  a.scores = reinterpret_cast<float *>(static_cast<char *>(workspace) + kRoom);
  a.selected = args->selected;
  a.status = status_dev;
  const auto s = static_cast<hipStream_t>(stream);
  // As many tokens at a time as the workspace holds, by 64, which fill a workgroup's row sets; where
  // every token keeps all that it sees there are no scores.
  const bool scored = batch->n_entries > a.keep;
  const int tokens = most_tokens(batch);
  a.limit = static_cast<int *>(workspace);
  a.scored = scored;
  a.most = args->most_blocks ? args->most_blocks : INT32_MAX;
  a.pitch = known ? (int)lines : 0;
  a.run = scored ? std::min(tokens, kMostRun) : tokens;
  if (scored && !known) a.run = (int)std::min<size_t>((workspace_bytes - kRoom) / one, a.run);
  if (a.run < tokens && a.run > 64) a.run &= -64;
  const int tiles = (a.run - 1) / (16 >> a.shift) + 1;
  const bool many = tiles >= 4 && a.padded <= 16;
  const int each = many ? many_sets(format->head_dim) * kWaves : 1, sets = (tiles - 1) / each + 1;
  // One round of workgroups where there are many sets: each begins with 5 us of loads and of rounding its
  // queries, and 32 blocks more take 2 us (512 tokens, 64 heads: of 4000 blocks 61 us, with at most 256
  // entries to a workgroup 81; of 2001 blocks 39 and 45).  Small where there is little to share:
  // one request's next token takes 6.6 us by 32 and 8.6 by 64, 128 requests' 48 and 50.  One form for
  // the whole batch, by its longest run: 128 single tokens 47 us, a chunk of 512 57, both in one call 208.
  const int64_t share = (int64_t)batch->n_entries * format->kv_heads * sets / 512;
  a.span = many ? (int)std::min<int64_t>(std::max<int64_t>((share + 31) / 32 * 32, 32), 1024) : 32;
  a.spans = (batch->n_entries - 1) / a.span + 1;
  a.sets = sets;
  const int64_t pieces = ((many ? (int64_t)a.spans * sets * format->kv_heads : a.spans) + 7) / 8 * 8;
  if (scored && pieces > INT32_MAX / kBlock) return CASCADE_EINVAL;
  // A wave to a row where all rows fit its registers (none has more candidates than the
  // table has entries) and there are enough of them to fill the GPU.
  const bool waves = batch->n_entries <= 64 * kHeld && rows >= 2048;
  // Else a workgroup, with registers for 2048 candidates, or 4096 where requests have more on average: 192
  // rows of 4000 9.4 us, else 13.2; 8 rows of 2044 7.1 and 7.9, 1024 of 660 8.8 and 9.7 (more code to fetch).
  const bool longer = batch->n_entries > (int64_t)64 * kWaves * 8 * batch->n;
  const int64_t groups = waves ? (rows + kWaves - 1) / kWaves : rows;
  auto kernel = waves ? select_wave_kernel : longer ? select_block_kernel<16> : select_block_kernel<8>;
  for (a.first = 0; a.first < tokens; a.first += a.run) {
    if (scored) {
      const dim3 grid((unsigned)pieces, many ? 1 : sets);
      args->dtype == CASCADE_BF16 ? score<CASCADE_BF16>(a, many, grid, s) : score<CASCADE_F16>(a, many, grid, s);
    }
    hipLaunchKernelGGL(kernel, dim3((unsigned)groups + 1), dim3(kBlock), 0, s, a);  // the last one checks the batch
  }
  return hipGetLastError() == hipSuccess ? CASCADE_OK : CASCADE_EHIP;
}
