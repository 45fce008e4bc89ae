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
// applies the block's power-of-two scale exactly (in float16 as much of it as
// the type holds, the rest in 32 bits: Units).
//
// m follows the row's maximum only when a score exceeds it by 2^8: most tiles
// then rescale nothing and need no exchange between lanes; sums stay below
// 2^8 times a row's length.
//
// Work is the list of (request, head, row tile) segments, each as long as
// its last row sees tokens, cut into ranges of equal cost, one per
// workgroup.  Every workgroup derives the list from the batch's lengths by
// itself (a scan), so ragged batches need neither a host plan nor another launch.  A
// segment that one workgroup covers is written at once; parts of a cut one go
// to the workspace and a second launch joins them.
//
// Few rows of a request are bound by reading the cache: 4 requests of 115 Ki
// tokens, 32 heads over 8 of 128 dims, 947 MB in 177 us (1043 MB fetched, 5.9
// TB/s; a large read reaches 6.2) and 8 for the join; 128 requests of 582 tokens,
// 64 heads, 157 MB in 35 to 37 us (4.5 TB/s: 4 us are the list, and short segments
// fill and drain), the join and the weights 10 more.  Drafts of up to 32 rows wait
// half of their cycles at two waves a SIMD: 32 requests of 7 Ki tokens, 462 MB in 109
// us.  Many rows are bound by the products and the softmax beside them
// (tile_kernel).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <cmath>
#include <limits>

#include "attention_work.h"
#include "cascade.h"
#include "device_util.h"
#include "kv_format.h"

namespace cascade {
namespace {

typedef float f2 __attribute__((ext_vector_type(2)));
typedef float f4 __attribute__((ext_vector_type(4)));
typedef float f16v __attribute__((ext_vector_type(16)));
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
  static constexpr bool kBounded = false;  // holds a code times any scale
  typedef bf2 v2;
  typedef bf8 v8;
  static __device__ __forceinline__ unsigned widen_lo(unsigned w, float s) {
    return __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, s, false));
  }
  static __device__ __forceinline__ unsigned widen_hi(unsigned w, float s) {
    return __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, s, true));
  }
  // c plus both of w
  static __device__ __forceinline__ float add2(unsigned w, float c) {
    return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(v2, w), __builtin_bit_cast(v2, 0x3f803f80u), c, false);
  }
  static __device__ __forceinline__ f4 mfma(v8 a, v8 b, f4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
  }
  static __device__ __forceinline__ f16v mfma(v8 a, v8 b, f16v c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
  }
};
template <> struct El<CASCADE_F16> {
  static constexpr bool kBounded = true;
  typedef h2 v2;
  typedef h8 v8;
  static __device__ __forceinline__ unsigned widen_lo(unsigned w, float s) {
    return __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, s, false));
  }
  static __device__ __forceinline__ unsigned widen_hi(unsigned w, float s) {
    return __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, s, true));
  }
  static __device__ __forceinline__ float add2(unsigned w, float c) {
    return __builtin_amdgcn_fdot2(__builtin_bit_cast(v2, w), __builtin_bit_cast(v2, 0x3c003c00u), c, false);
  }
  static __device__ __forceinline__ f4 mfma(v8 a, v8 b, f4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
  }
  static __device__ __forceinline__ f16v mfma(v8 a, v8 b, f16v c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
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

// What O is multiplied by so that it is an average by the weights as they were
// rounded, `used` their sum, and not by the weights of `sum`: a row that one
// token dominates is exact then, where the rounding of its weight would stay.
// 8 heads over 777 tokens of bfloat16: relative error 1.8e-3 to 2.2e-3 (of
// which the result's own rounding is 1.4e-3 to 1.7e-3), without it up to
// 2.7e-3.  It costs row tiles 3 % where log sums are wanted too, else nothing.
__device__ __forceinline__ float evened(float sum, float used) {
  return used > 0.f && used < __builtin_inff() ? sum / used : 1.f;
}

// A block's scale as the part that the conversion applies and the rest, for
// 32 bits.  float16 holds every code times 2^-15 (the least is 2^-24) to 2^7 (the
// largest is 57344); beyond, keys' scores are multiplied by the rest, and O is
// kept in units of it while a block's values are added.  Asking whether there is
// a rest costs float16 rows, of bfloat16's times: 32 requests with draft rows
// 117.9 us against 117.1, 4 of 115 Ki tokens 185 against 182, row tiles 1 to 2 %
// (of 256 dims 22 %: the compiler moves more of O between its register files).
__device__ __forceinline__ float applied(float scale, float &rest) {
  const int bits = __builtin_bit_cast(int, scale), held = min(max(bits, (127 - 15) << 23), (127 + 7) << 23);
  rest = __builtin_bit_cast(float, bits - held + (127 << 23));
  return __builtin_bit_cast(float, held);
}
// Of values a rest under 2^-24 counts as that: they are under 2^-30, and a
// result's last place is 2^-24.  So O over a rest stays finite unless the result
// is over the type's largest anyway.
__device__ __forceinline__ float unit_of(float rest) { return fmaxf(rest, 0x1p-24f); }
__device__ __forceinline__ float inverse_unit(float unit) {  // of a power of two
  return __builtin_bit_cast(float, (254 << 23) - __builtin_bit_cast(int, unit));
}
// The scales of the two sub-blocks of a step.
template <int kType>
struct Units {
  float scale[2], rest[2];
  bool odd = false;  // a rest is not 1
  __device__ __forceinline__ Units(const float (&s)[2]) {
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      scale[b] = s[b];
      if (El<kType>::kBounded) {
        const float held = applied(s[b], rest[b]);  // the same in all lanes
        scale[b] = __builtin_bit_cast(float, __builtin_amdgcn_readfirstlane(__builtin_bit_cast(int, held)));
        odd |= __builtin_amdgcn_readfirstlane(__builtin_bit_cast(int, rest[b])) != 127 << 23;
      }
    }
  }
};

struct Rows {
  char *data;
  int64_t token_stride, head_stride;  // bytes
};

// tanh(x / cap) by tanh(y) = 1 - 2 / (exp(2 y) + 1): off by 2^-23 of the cap,
// however small the score, which up to kNarrowLimit is within the scores' other
// errors.  Wider caps take tanh(y) = y (1 - y^2/3 + ...) for |y| under 1/2,
// off by 2^-23 of the score (the series' next term is 1e-8 of it), in kernels of
// their own: 16 chunks of 512 tokens, 64 heads, take 3.24 ms by that, 2.34 without.
enum class Cap { kNone, kNarrow, kWide };
constexpr float kNarrowLimit = 64.f;
template <Cap kCap>
__device__ __forceinline__ float capped(float x, float cap_in, float cap_y, float qk, float cap) {
  const float t = 1.f - 2.f * __builtin_amdgcn_rcpf(__builtin_amdgcn_exp2f(x * cap_in) + 1.f);
  if (kCap == Cap::kNarrow) return t;
  const float y = x * cap_y, z = y * y;
  float series = -929569.f / 638512875.f;
  series = __builtin_fmaf(series, z, 21844.f / 6081075.f);
  series = __builtin_fmaf(series, z, -1382.f / 155925.f);
  series = __builtin_fmaf(series, z, 62.f / 2835.f);
  series = __builtin_fmaf(series, z, -17.f / 315.f);
  series = __builtin_fmaf(series, z, 2.f / 15.f);
  series = __builtin_fmaf(series, z, -1.f / 3.f);
  series = __builtin_fmaf(series, z, 1.f);
  return fabsf(y) < 0.5f ? x * qk * series : cap * t;
}

struct Attention : Cuts {
  KvView kv;
  cascade_kv_batch_t batch;
  const int32_t *row_offsets, *slots;
  Rows q, out;
  int q_heads, group;      // query heads, and those of one KV head
  float scale;             // of q.k, or of the capped score; in log2 units, >= 0
  float cap_in;            // softcap: exp2 argument per q.k
  float cap_y, qk, cap;    // Cap::kWide: per q.k of the cap, and both in log2 units (`scale` is 1)
  unsigned keep, flip;     // q's bits: none where the scale was 0, turned signs where it was negative
  float *lse;              // [n_tokens][q_heads] or NULL
  float *logs;             // log2 of weights over runs of tokens, or NULL
  int log_shift;           // log2 of such a run
  int window;
  int64_t min_rows, max_rows;  // requests with min_rows < rows <= max_rows are taken
  Split *splits;           // [gridDim]
  float *parts;            // [gridDim][2][rows][kDim]
  float *part_sums;        // [gridDim][2][rows][2]: m and sum
  int32_t *status;
};

// ---------------------------------------------------------------- the work

// Log sums are kept of each 32 tokens, or 16 in blocks of no more (32 requests
// with draft rows and weights of 8 tokens: 118 us, by 16 123).  They lie as
// [run][KV head][window][head of the group], so that a segment's tile writes
// whole lines.  A row's place in a run's, for the head `of_group` of the token
// `back` before its request's last:
__device__ __forceinline__ int log_place(const Attention &a, int kv_head, int back, int of_group) {
  return (kv_head * a.window + back) * a.group + of_group;
}
// and those of a request's first run:
__device__ __forceinline__ float *first_logs(const Attention &a, int first_entry) {
  return a.logs + ((int64_t)first_entry << (a.kv.block_shift - a.log_shift)) * a.window * a.q_heads;
}

// A lane's place, as wave-uniform numbers.
__device__ __forceinline__ Place uniform(const Place &p, int lane = 0) {
  return {__builtin_amdgcn_readlane(p.item, lane), __builtin_amdgcn_readlane(p.head, lane),
          __builtin_amdgcn_readlane(p.tile, lane), __builtin_amdgcn_readlane(p.key, lane)};
}

__device__ __forceinline__ long long first_lane(unsigned long long x) {
  const unsigned lo = __builtin_amdgcn_readfirstlane((unsigned)x);
  return (long long)((unsigned long long)__builtin_amdgcn_readfirstlane((unsigned)(x >> 32)) << 32 | lo);
}

// The part of the work that a workgroup takes.
struct Range {
  Place begin, end;
  int items;  // requests in the list
  int group;  // which range it is

  // Fills the list and finds the range; false if there is none.  Called by all
  // threads.  Records the segment that the range's begin is the first cut of.
  template <int kW>
  __device__ __forceinline__ bool find(const Attention &a, const List &list, unsigned long long *scan) {
    const int lane = lane_id();
    int n = 0;
    long long total = 0;
    for (int i0 = 0; i0 < a.batch.n; i0 += 64 * kW) {
      const int i = i0 + threadIdx.x;
      unsigned long long v[2] = {0, 0}, all[2];
      KvRequest r = {};
      if (i < a.batch.n) {
        r = kv_request(a.batch, a.row_offsets, a.kv.block_shift, i);
        if (!r.ok) {
          kv_report(a.status);
        } else {
          const int64_t rows = (int64_t)r.count * a.group;
          if (rows > a.min_rows && rows <= a.max_rows)
            v[0] = Segments(r.len, r.count, a.tile_tokens).total() * a.kv.kv_heads;
        }
      }
      const unsigned long long cost = v[0];
      v[1] = cost > 0;
      block_exclusive_scan<2, unsigned long long, kW>(v, all, scan);
      if (cost) {
        const int at = n + (int)v[1];
        list.before[at] = total + v[0];
        list.ids[at] = i;
        list.len[at] = r.len;
        list.count[at] = r.count;
      }
      n += __builtin_amdgcn_readfirstlane((int)all[1]);
      total += first_lane(all[0]);
    }
    if (threadIdx.x == 0) list.before[n] = total;
    __syncthreads();

    // this workgroup's range: neighbours in cost on one XCD (workgroups go to
    // the 8 XCDs in turn), where heads and row tiles of a request share its L2
    const int groups = ranges(a, total, gridDim.x);
    const int block = blockIdx.x;
    if (block >= groups || n == 0) {
      if (threadIdx.x == 0) a.splits[block] = Split{-1, 0, 0, 0};
      return false;
    }
    const int w = groups >= 8 ? (block & 7) * (groups >> 3) + (block >> 3) : block;
    // lanes 0, 1, 2: this range's begin, its end, the one before's begin
    const int which = lane == 1 ? w + 1 : lane == 2 ? max(w - 1, 0) : w;
    const Place found =
        locate(a, a.kv.kv_heads, list, n, uncut_keys(a, total, groups), cut(total, which, groups));
    const Place at = uniform(found, 0), prev = uniform(found, 2);
    begin = at;
    end = uniform(found, 1);
    items = n;
    group = w;

    if (threadIdx.x == 0) a.splits[w] = first_cut(a, list, at, prev, total, groups);
    return true;
  }
};

// ------------------------------------------------------------- one wave

// What a wave keeps of 16 * kTiles query rows.
template <int kType, int kDim, int kTiles, Cap kCap>
struct Rowset {
  typedef typename El<kType>::v8 v8;
  f4 o[kTiles][kDim / 16];
  float m[kTiles], sum[kTiles];
  float used[kTiles];   // sum of the weights as they are rounded for the product
  int limit[kTiles];    // last cached token that the lane's row sees
  int log_at[kTiles];   // the row's place in a run's log sums, -1 for none

  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int t = 0; t < kTiles; ++t) {
      m[t] = kLowest;
      sum[t] = used[t] = 0.f;
#pragma unroll
      for (int d = 0; d < kDim / 16; ++d) o[t][d] = f4{0.f, 0.f, 0.f, 0.f};
    }
  }

  // Scores of kB sub-blocks of 16 tokens; `k(b, d)` gives the operand of
  // sub-block b and dims step d, `q(t, d)` that of row set t.
  template <int kB, typename KOp, typename QOp>
  __device__ __forceinline__ void scores(KOp k, QOp q, f4 (&s)[kTiles][kB]) const {
#pragma unroll
    for (int b = 0; b < kB; ++b)
#pragma unroll
      for (int t = 0; t < kTiles; ++t) s[t][b] = f4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int d = 0; d < kDim / 32; ++d) {
      v8 x[kTiles];
#pragma unroll
      for (int t = 0; t < kTiles; ++t) x[t] = q(t, d);
#pragma unroll
      for (int b = 0; b < kB; ++b) {
        const v8 y = k(b, d);
#pragma unroll
        for (int t = 0; t < kTiles; ++t) s[t][b] = El<kType>::mfma(y, x[t], s[t][b]);
      }
    }
  }

  // Their weights, for tokens from `key` on; m, sum and o follow.  `masked`:
  // some row does not see all of the tokens.
  template <int kB>
  __device__ __forceinline__ void weights(const Attention &a, f4 (&s)[kTiles][kB], v8 (&p)[kTiles][kB / 2],
                                          int key, int len, bool masked, float *logs) {
    const int lane = lane_id(), g = lane >> 4;
    if (kCap != Cap::kNone) {
#pragma unroll
      for (int t = 0; t < kTiles; ++t)
#pragma unroll
        for (int b = 0; b < kB; ++b)
#pragma unroll
          for (int i = 0; i < 4; ++i) s[t][b][i] = capped<kCap>(s[t][b][i], a.cap_in, a.cap_y, a.qk, a.cap);
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
    float top[kTiles];
    bool over = false;
#pragma unroll
    for (int t = 0; t < kTiles; ++t) {
      top[t] = s[t][0][0];
#pragma unroll
      for (int i = 1; i < 4 * kB; ++i) top[t] = fmaxf(top[t], s[t][i >> 2][i & 3]);
      top[t] *= a.scale;
      over |= top[t] > m[t] + kSlack;
    }
    if (__any(over)) {
#pragma unroll
      for (int t = 0; t < kTiles; ++t) {
        top[t] = fmaxf(top[t], __shfl_xor(top[t], 16));
        top[t] = fmaxf(top[t], __shfl_xor(top[t], 32));
        const float now = fmaxf(m[t], top[t]), f = __builtin_amdgcn_exp2f(m[t] - now);
        m[t] = now;
        sum[t] *= f;
        used[t] *= f;
#pragma unroll
        for (int d = 0; d < kDim / 16; ++d) o[t][d] *= f;
      }
    }
    float part[kTiles][kB];
#pragma unroll
    for (int t = 0; t < kTiles; ++t) {
#pragma unroll
      for (int b = 0; b < kB; ++b) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
          s[t][b][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[t][b][i], a.scale, -m[t]));
        part[t][b] = (s[t][b][0] + s[t][b][1]) + (s[t][b][2] + s[t][b][3]);
        sum[t] += part[t][b];
      }
#pragma unroll
      for (int b = 0; b < kB; b += 2) {
        const u4 w = {narrow2<kType>(s[t][b][0], s[t][b][1]), narrow2<kType>(s[t][b][2], s[t][b][3]),
                      narrow2<kType>(s[t][b + 1][0], s[t][b + 1][1]),
                      narrow2<kType>(s[t][b + 1][2], s[t][b + 1][3])};
        p[t][b / 2] = __builtin_bit_cast(v8, w);
#pragma unroll
        for (int i = 0; i < 4; ++i) used[t] = El<kType>::add2(w[i], used[t]);
      }
    }
    if (logs) {
      static_assert(kB == 2, "one run of 32 tokens, or two of 16");
      const int64_t run = (int64_t)a.window * a.q_heads;
      float *const to = logs + (key >> a.log_shift) * run;
#pragma unroll
      for (int t = 0; t < kTiles; ++t) {
        auto keep = [&](float x, float *to) {
          x += __shfl_xor(x, 16);
          x += __shfl_xor(x, 32);
          if (g == 0 && log_at[t] >= 0) to[log_at[t]] = __builtin_amdgcn_logf(x) + m[t];
        };
        if (a.log_shift == 5) {
          keep(part[t][0] + part[t][1], to);
        } else {
          keep(part[t][0], to);
          if (key + 16 < len) keep(part[t][1], to + run);
        }
      }
    }
  }

  // O of 32 tokens; `v(d)` gives the operand of dims 16 d, with 0 for tokens
  // past the cache's end, which may be anything.
  template <typename VOp>
  __device__ __forceinline__ void add(VOp v, const v8 (&p)[kTiles][1]) {
#pragma unroll
    for (int d = 0; d < kDim / 16; ++d) {
      const v8 x = v(d);
#pragma unroll
      for (int t = 0; t < kTiles; ++t) o[t][d] = El<kType>::mfma(x, p[t][0], o[t][d]);
    }
  }

  __device__ __forceinline__ void scale_o(float f) {
#pragma unroll
    for (int t = 0; t < kTiles; ++t)
#pragma unroll
      for (int d = 0; d < kDim / 16; ++d) o[t][d] *= f;
  }
};

// Where a request's head lies in the cache.
template <int kDim>
struct Cache : SubBlocks {
  const char *base;    // the head's codes in slot 0
  int64_t kv_stride, slot_stride, scales;  // `scales`: from the codes to the head's scale
  const int32_t *slots;
  int num_slots;
  // of the tokens before `end`, a request's length at most, and above 0
  __device__ __forceinline__ Cache(const Attention &a, const KvRequest &r, int head, int end)
      : SubBlocks(a.kv.block_shift, end), base(a.kv.base + ((int64_t)head << a.kv.block_shift) * kDim),
        kv_stride(a.kv.kv_stride), slot_stride(a.kv.slot_stride),
        scales(((int64_t)(a.kv.kv_heads - head) << a.kv.block_shift) * kDim + 4 * head),
        slots(a.slots + r.row), num_slots(a.kv.num_slots) {}
  // slot of sub-block `sub`, or of the last one
  __device__ __forceinline__ int slot(int sub) const { return uniform_load(slots + entry(sub)); }
  // from slot 0 to a slot
  __device__ __forceinline__ int64_t offset(int slot, bool &bad) const {
    const bool fine = (unsigned)slot < (unsigned)num_slots;
    bad |= !fine;
    return (fine ? slot : 0) * slot_stride;
  }
  // the head's codes in a slot; one outside the pool counts as slot 0 and sets `bad`
  __device__ __forceinline__ const char *block(int slot, bool &bad) const { return base + offset(slot, bad); }
  // a sub-block within its block's codes
  __device__ __forceinline__ int place(int sub) const { return within(sub) * 16 * kDim; }
  __device__ __forceinline__ const char *codes(const char *block, int sub) const { return block + place(sub); }
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
  bool bad = false;
  __device__ __forceinline__ void fetch_k(const Cache<kDim> &c, const int (&slot)[2], int key) {
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      const char *block = c.block(slot[b], bad), *at = c.codes(block, (key >> 4) + b);
#pragma unroll
      for (int i = 0; i < kDim / 64; ++i) k[b][i] = *reinterpret_cast<const u4 *>(at + 1024 * i + k_place());
      ks[b] = c.k_scale(block);
    }
  }
  __device__ __forceinline__ void fetch_v(const Cache<kDim> &c, const int (&slot)[2], int key) {
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      const char *block = c.block(slot[b], bad), *at = c.codes(block, (key >> 4) + b) + c.kv_stride;
#pragma unroll
      for (int i = 0; i < kDim / 64; ++i) v[b][i] = *reinterpret_cast<const u4 *>(at + 1024 * i + v_place());
      vs[b] = c.v_scale(block);
    }
  }
};

// ------------------------------------------------------------- the kernel

// A tile of up to 16 * kTiles rows; kWaves waves share its tokens and combine in LDS.
// As many waves as its registers allow without scratch; 64 rows of 128 dims
// spill 30 registers at two and are faster so (32 requests of 64 draft rows a
// head over 7 Ki tokens: 157 us, without scratch at one wave 205), others that
// could be pressed further are slower (32 rows of 128 dims at three waves: 132
// us, at two 128; of 256 at two: 243, at one 234).
constexpr int waves_per_simd(int dim, int tiles) {
  const int held = dim * tiles;  // of o in registers
  return held <= 64 ? 5 : tiles == 1 && held <= 128 ? 4 : held <= 128 ? 3 : held <= 256 || tiles == 4 ? 2 : 1;
}
template <int kType, int kDim, int kTiles, Cap kCap>
__global__ __launch_bounds__(kBlock, waves_per_simd(kDim, kTiles)) void attention_kernel(Attention a) {
  constexpr int kRows = 16 * kTiles;
  constexpr int kPart = kDim < 128 ? kDim : 128;  // dims that one combination takes
  constexpr int kPitch = kPart + 4;
  typedef typename El<kType>::v8 v8;
  extern __shared__ __align__(16) char lds[];
  __shared__ unsigned long long scan[2 * kWaves];
  const List list(lds, a.batch.n);
  // the waves' m and sum, and their O or before it q
  float *const ms = reinterpret_cast<float *>(lds + list_bytes(a.batch.n)), *const os = ms + 2 * kWaves * 16;
  char *const qs = reinterpret_cast<char *>(os);
  static_assert(kRows * kDim * 2 <= 4 * kWaves * 16 * kPitch, "q fits the place of O");
  const int lane = lane_id(), g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(wave_id());
  Range range;
  if (!range.find<kWaves>(a, list, scan)) return;
  Place at = range.begin;
  const Place end = uniform(range.end);
  const int n = __builtin_amdgcn_readfirstlane(range.items), w = __builtin_amdgcn_readfirstlane(range.group);
  const int kv_heads = a.kv.kv_heads;

  Rowset<kType, kDim, kTiles, kCap> r;
  while (at.item < n) {
    at = uniform(at);  // the compiler does not see that it is
    const int id = __builtin_amdgcn_readfirstlane(list.ids[at.item]);
    const KvRequest req = kv_request<true>(a.batch, a.row_offsets, a.kv.block_shift, id);
    const Segments seg(req.len, req.count, a.tile_tokens);
    const int length = (int)seg.length(at.tile);
    const bool last = end.item == at.item && end.head == at.head && end.tile == at.tile;
    const int stop = last ? end.key : length;
    if (last && stop == at.key) break;

    // rows: lane n of row set t has row 16 t + n of the tile
    const int tile_rows = a.tile_tokens * a.group, shown = req.len - req.count;
    bool any = false;
#pragma unroll
    for (int t = 0; t < kTiles; ++t) {
      const int row = 16 * t + (lane & 15), token = at.tile * a.tile_tokens + row / a.group;
      const bool valid = row < tile_rows && token < req.count;
      r.limit[t] = valid ? shown + token : -1;
      const int back = req.count - 1 - token;
      r.log_at[t] = a.logs && valid && back < a.window ? log_place(a, at.head, back, row % a.group) : -1;
      any |= r.log_at[t] >= 0;
    }
    float *const logs = __any(any) ? first_logs(a, req.row) : nullptr;
    r.clear();

    // every row sees the tokens before clear_end, none those from key_end on
    const int first_token = at.tile * a.tile_tokens;
    const int last_token = min(first_token + a.tile_tokens, req.count) - 1;
    const int clear_end = __builtin_amdgcn_readfirstlane(shown + first_token + 1);
    const int key_end = __builtin_amdgcn_readfirstlane(min(min(stop, req.len), shown + last_token + 1));
    const int len = __builtin_amdgcn_readfirstlane(req.len);
    // the same in all waves; a request may have no blocks where nothing is seen
    if (at.key < key_end) {
      const Cache<kDim> cache(a, req, at.head, key_end);
      // each wave takes every fourth 32 tokens, straight into registers: the next K
      // codes are requested when these have been taken, V codes likewise, and the
      // slots are known a step ahead of them.  No load hangs on a condition (a wait
      // after the ways meet again would wait for too much): past the end the last
      // sub-block is read again, from a cache.
      constexpr int kStride = 32 * kWaves;
      int key = __builtin_amdgcn_readfirstlane(at.key + 32 * wave);
      Codes<kDim> c;
      int slot[2];
      auto look = [&](int key) {
        slot[0] = cache.slot(key >> 4);
        slot[1] = cache.slot((key >> 4) + 1);
      };
      look(key);
      // the waves share the rows' q, which lies in operand order in LDS
      constexpr int kQs = kTiles * (kDim / 32), kMine = (kQs + kWaves - 1) / kWaves;
      u4 q[kMine];
#pragma unroll
      for (int i = 0; i < kMine; ++i) {
        const int e = min(i * kWaves + wave, kQs - 1), d = e % (kDim / 32);
        const int row = e / (kDim / 32) * 16 + (lane & 15);
        const int token = at.tile * a.tile_tokens + row / a.group, head = at.head * a.group + row % a.group;
        const bool valid = row < tile_rows && token < req.count;
        q[i] = *reinterpret_cast<const u4 *>(a.q.data + (int64_t)(req.first + (valid ? token : 0)) * a.q.token_stride +
                                             (valid ? head : 0) * a.q.head_stride + 32 * g + 128 * (d >> 1) +
                                             16 * (d & 1));
        q[i] = valid ? (q[i] & a.keep) ^ a.flip : u4{0, 0, 0, 0};
      }
      __builtin_amdgcn_sched_barrier(0);
      c.fetch_k(cache, slot, key);
      // K before V, as in the loop: waits count the loads that follow
      __builtin_amdgcn_sched_barrier(0);
      c.fetch_v(cache, slot, key);
      __builtin_amdgcn_sched_barrier(0);
      look(key + kStride);
#pragma unroll
      for (int i = 0; i < kMine; ++i)
        *reinterpret_cast<u4 *>(qs + (min(i * kWaves + wave, kQs - 1) * 64 + lane) * 16) = q[i];
      __syncthreads();
      if (key < key_end) {
        while (true) {
          if (key + 32 > len) {
            const unsigned live[2] = {live_bytes(key + 4 * g, len), live_bytes(key + 16 + 4 * g, len)};
#pragma unroll
            for (int i = 0; i < kDim / 64; ++i)
#pragma unroll
              for (int b = 0; b < 2; ++b) c.v[b][i] &= live[b];
          }
          f4 x[kTiles][2];
          int q_at = lane * 16;
          asm volatile("" : "+v"(q_at));  // or the loads of q move out of the loop, into registers
          const Units<kType> ku(c.ks);
          r.template scores<2>(
              [&](int b, int d) {
                const u4 w = c.k[b][d >> 1];
                return widen8<kType>(w[2 * (d & 1)], w[2 * (d & 1) + 1], ku.scale[b], ku.scale[b]);
              },
              [&](int t, int d) {
                return *reinterpret_cast<const v8 *>(qs + (t * (kDim / 32) + d) * 1024 + q_at);
              },
              x);
          if (__builtin_expect(ku.odd, false)) {
#pragma unroll
            for (int t = 0; t < kTiles; ++t)
#pragma unroll
              for (int b = 0; b < 2; ++b) x[t][b] *= ku.rest[b];
          }
          c.fetch_k(cache, slot, key + kStride);
          v8 p[kTiles][1];
          r.template weights<2>(a, x, p, key, len, key + 32 > clear_end, logs);
          const Units<kType> vu(c.vs);
          // at once, or sub-block by sub-block where their values have rests
          v8 part[kTiles][1];
#pragma unroll
          for (int t = 0; t < kTiles; ++t) part[t][0] = p[t][0];
          for (int b = 0;; ++b) {
            if (__builtin_expect(vu.odd, false)) {
              r.scale_o(inverse_unit(unit_of(vu.rest[b])));
#pragma unroll
              for (int t = 0; t < kTiles; ++t) {
                u4 w = __builtin_bit_cast(u4, p[t][0]);
#pragma unroll
                for (int i = 0; i < 4; ++i) w[i] = i / 2 == b ? w[i] : 0;
                part[t][0] = __builtin_bit_cast(v8, w);
              }
            }
            float s0 = vu.scale[0], s1 = vu.scale[1];
            if (El<kType>::kBounded) asm volatile("" : "+s"(s0), "+s"(s1));  // or all of V is widened before the loop
            r.add(
                [&](int d) { return widen8<kType>(c.v[0][d >> 2][d & 3], c.v[1][d >> 2][d & 3], s0, s1); },
                part);
            if (__builtin_expect(!vu.odd, true)) break;
            r.scale_o(unit_of(vu.rest[b]));
            if (b) break;
          }
          c.fetch_v(cache, slot, key + kStride);
          look(key + 2 * kStride);
          key += kStride;
          if (key >= key_end) break;
        }
        if (c.bad) kv_report(a.status);
      }
    }

#pragma unroll
    for (int t = 0; t < kTiles; ++t) {
      r.sum[t] += __shfl_xor(r.sum[t], 16);
      r.sum[t] += __shfl_xor(r.sum[t], 32);
      r.used[t] += __shfl_xor(r.used[t], 16);
      r.used[t] += __shfl_xor(r.used[t], 32);
    }
    const bool whole = at.key == 0 && stop == length;
    const int64_t part = ((int64_t)w * 2 + (at.key > 0 ? 0 : 1)) * kRows;
    // one row set at a time
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
      const float f = __builtin_amdgcn_exp2f(r.m[t] - top) * evened(r.sum[t], r.used[t]);
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

// A tile of many rows: 32 to a wave, and all of a workgroup's waves share the
// tokens.  A stage of them (64; 32 for the longest heads) is widened once, a
// sub-block's K or V by each wave, into LDS in operand order, two stages in turn.
// The products are taken as 32x32x16: one such instruction leaves room for 6
// vector instructions in its 32 cycles, two 16x16x32 for 2 each, and the softmax
// has about as many cycles as the products.  8 waves on a stage: with 4 each wave
// widens twice as much and takes 4 % longer.  16 chunks of 512 tokens, 64 heads over
// 8 of 128 dims, contexts of 7 k: 1.8 to 1.9 ms, 0.95 PFLOP/s of the 1.24 that a large
// matrix product reaches; the matrix units are busy for 45 % of the cycles.  Builds
// that leave parts out take 1.1 ms for the products alone, 1.2 with their operands'
// reads from LDS, 1.5 with the softmax, and 2.0 with the widening (before the last
// steps).  64 rows to a wave halve the LDS reads, but leave one wave to a SIMD and
// take 25 % longer.
constexpr int stage_tokens(int dim) { return dim == 256 ? 32 : 64; }
constexpr int tile_waves(int dim) { return 2 * stage_tokens(dim) / 16; }
constexpr int tile_rows(int dim) { return 32 * tile_waves(dim); }
// of LDS: K, V, and what of their scales the type does not hold
constexpr int stage_bytes(int type, int dim) {
  return stage_tokens(dim) * dim * 4 + (type == CASCADE_F16 ? stage_tokens(dim) / 16 * 8 : 0);
}
template <int kType, int kDim, Cap kCap>
__global__ __launch_bounds__(64 * tile_waves(kDim), kDim == 256 ? 1 : 2) void tile_kernel(Attention a) {
  typedef El<kType> E;
  typedef typename E::v8 v8;
  constexpr int kSlices = kDim / 64, kOut = kDim / 32, kTW = tile_waves(kDim);
  constexpr int kStage = stage_tokens(kDim), kSubs = kStage / 16, kHalves = kStage / 32;
  constexpr int kSide = kStage * kDim * 2;  // bytes of a stage's K or V operands
  constexpr bool kBounded = E::kBounded;
  extern __shared__ __align__(16) char lds[];
  __shared__ unsigned long long scan[2 * kTW];
  const List list(lds, a.batch.n);
  char *const stages = lds + list_bytes(a.batch.n);
  const int lane = lane_id(), n32 = lane & 31, hg = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(wave_id());
  Range range;
  if (!range.find<kTW>(a, list, scan)) return;
  Place at = range.begin;
  const Place end = uniform(range.end);
  const int items = __builtin_amdgcn_readfirstlane(range.items), w = __builtin_amdgcn_readfirstlane(range.group);

  while (at.item < items) {
    at = uniform(at);  // the compiler does not see that it is
    const int id = __builtin_amdgcn_readfirstlane(list.ids[at.item]);
    const KvRequest req = kv_request<true>(a.batch, a.row_offsets, a.kv.block_shift, id);
    const Segments seg(req.len, req.count, a.tile_tokens);
    const int length = (int)seg.length(at.tile);
    const bool last = end.item == at.item && end.head == at.head && end.tile == at.tile;
    const int stop = last ? end.key : length;
    if (last && stop == at.key) break;

    // the lane's row: 32 wave + lane % 32 of the tile
    const int row = 32 * wave + n32, shown = req.len - req.count;
    const int token = at.tile * a.tile_tokens + row / a.group, head = at.head * a.group + row % a.group;
    const bool valid = row < a.tile_tokens * a.group && token < req.count;
    const int limit = valid ? shown + token : -1;  // last cached token that it sees
    v8 q[kDim / 16];
    const char *from_q = a.q.data + (int64_t)(req.first + (valid ? token : 0)) * a.q.token_stride +
                         (valid ? head : 0) * a.q.head_stride + 16 * hg;
#pragma unroll
    for (int d = 0; d < kDim / 16; ++d) {
      u4 x = *reinterpret_cast<const u4 *>(from_q + 32 * d);
      if (!valid) x = u4{0, 0, 0, 0};
      q[d] = __builtin_bit_cast(v8, (x & a.keep) ^ a.flip);
    }
    const int back = req.count - 1 - token;
    const int log_at =
        a.logs && valid && back < a.window ? log_place(a, at.head, back, head - at.head * a.group) : -1;
    float *const logs = __any(log_at >= 0) ? first_logs(a, req.row) : nullptr;
    // every row of the wave sees the tokens before clear_end, no row of the tile those from block_end on
    const int clear_end = __builtin_amdgcn_readfirstlane(shown + at.tile * a.tile_tokens + 32 * wave / a.group + 1);
    const int block_end = __builtin_amdgcn_readfirstlane(
        min(stop, min(req.len, shown + min((at.tile + 1) * a.tile_tokens, req.count))));
    const int first_key = __builtin_amdgcn_readfirstlane(at.key), len = __builtin_amdgcn_readfirstlane(req.len);

    f16v o[kOut];
#pragma unroll
    for (int d = 0; d < kOut; ++d)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[d][i] = 0.f;
    float m = kLowest, sum = 0.f, used = 0.f;
    const bool exact = a.lse != nullptr;  // only log sums need the sum of the weights unrounded
    if (first_key < block_end) {
      // a wave carries one sub-block's K or V, a stage ahead.  Slots and scales by vector
      // loads, whose waits count in order (a wait for scalar loads waits for all
      // and for LDS), and no load hangs on a condition (a value that arrives on
      // one way only is waited for where the ways meet): past the end the
      // last sub-block is read again.
      const Cache<kDim> cache(a, req, at.head, block_end);
      u4 own[kSlices];
      float own_scale;
      int own_key = 0, slot;
      bool bad = false;
      const int sub = wave % kSubs, side = wave / kSubs;
      const char *const lane_codes = cache.base + side * cache.kv_stride + (side ? v_place() : k_place());
      const char *const lane_scale = cache.base + side * cache.kv_stride + cache.scales;
      auto look = [&](int key) { slot = vector_load(cache.slots + cache.entry((key >> 4) + sub)); };
      auto fetch = [&](int key) {
        const int64_t from = cache.offset(slot, bad), codes = from + cache.place((key >> 4) + sub);
        own_key = key + 16 * sub;
#pragma unroll
        for (int c = 0; c < kSlices; ++c) own[c] = *reinterpret_cast<const u4 *>(lane_codes + codes + 1024 * c);
        own_scale = *reinterpret_cast<const float *>(lane_scale + from);
        look(key + kStage);
      };
      // of 32 tokens (a half): K operand [16 dims][lane], lane = token + 32 * (which 8
      // of them); V operand [16 tokens][32 dims][lane], lane = dim + 32 * hg, of tokens
      // 4 hg + 0..3 and 8 + 4 hg + 0..3
      constexpr int kHalf = 32 * kDim * 2;
      const int own_place = (sub >> 1) * kHalf + (side ? kSide + ((sub & 1) * kOut * 64 + 32 * (lane >> 4 & 1) + (lane & 15)) * 16 + 8 * (lane >> 5)
                                                      : ((lane >> 4) * 64 + 16 * (sub & 1) + (lane & 15)) * 16);
      auto put = [&](char *to) {
        float scale = own_scale;
        if (kBounded) {
          float rest;
          scale = applied(own_scale, rest);
          if (lane == 0) reinterpret_cast<float *>(to + 2 * kSide)[side * kSubs + sub] = rest;
        }
        to += own_place;
        if (side == 0) {
#pragma unroll
          for (int c = 0; c < kSlices; ++c)
#pragma unroll
            for (int h = 0; h < 2; ++h)
              *reinterpret_cast<v8 *>(to + (4 * c * 64 + 32 * h) * 16) =
                  widen8<kType>(own[c][2 * h], own[c][2 * h + 1], scale, scale);
        } else {
          if (own_key + 16 > len) {  // codes past the end may be anything
            const unsigned live = live_bytes(own_key + 4 * (lane >> 4), len);
#pragma unroll
            for (int c = 0; c < kSlices; ++c) own[c] &= live;
          }
#pragma unroll
          for (int c = 0; c < kSlices; ++c)
#pragma unroll
            for (int j = 0; j < 4; ++j)
              *reinterpret_cast<u2 *>(to + ((2 * c + (j >> 1)) * 64 + 16 * (j & 1)) * 16) =
                  u2{E::widen_lo(own[c][j], scale), E::widen_hi(own[c][j], scale)};
        }
      };
      v8 kop[kDim / 16], vop[2][kOut];
      auto load_k = [&](const char *from, int h) {
#pragma unroll
        for (int d = 0; d < kDim / 16; ++d)
          kop[d] = *reinterpret_cast<const v8 *>(from + h * kHalf + (d * 64 + lane) * 16);
      };
      auto load_v = [&](const char *from, int h) {
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int d = 0; d < kOut; ++d)
            vop[u][d] = *reinterpret_cast<const v8 *>(from + kSide + h * kHalf + ((u * kOut + d) * 64 + lane) * 16);
      };
      auto scores = [&](f16v &x) {
#pragma unroll
        for (int i = 0; i < 16; ++i) x[i] = 0.f;
#pragma unroll
        for (int d = 0; d < kDim / 16; ++d) x = E::mfma(kop[d], q[d], x);
      };
      // score i of a lane is token key + 8 * (i / 4) + 4 * hg + i % 4
      auto limits = [&](f16v &x, int key) {
        if (kCap != Cap::kNone) {
#pragma unroll
          for (int i = 0; i < 16; ++i) x[i] = capped<kCap>(x[i], a.cap_in, a.cap_y, a.qk, a.cap);
        }
        if (key + 32 > clear_end) {
          const int seen = limit - key - 4 * hg;
#pragma unroll
          for (int i = 0; i < 16; ++i) x[i] = 8 * (i >> 2) + (i & 3) <= seen ? x[i] : -__builtin_inff();
        }
      };
      auto raise = [&](const f16v (&x)[kHalves]) {
        float part[4];
#pragma unroll
        for (int h = 0; h < kHalves; ++h)
#pragma unroll
          for (int i = 0; i < 16; ++i) part[i & 3] = h + i < 4 && h == 0 ? x[h][i] : fmaxf(part[i & 3], x[h][i]);
        float top = fmaxf(fmaxf(part[0], part[1]), fmaxf(part[2], part[3])) * a.scale;
        if (__any(top > m + kSlack)) {
          top = fmaxf(top, __shfl_xor(top, 32));
          const float now = fmaxf(m, top), f = __builtin_amdgcn_exp2f(m - now);
          m = now;
          sum *= f;
          used *= f;
#pragma unroll
          for (int d = 0; d < kOut; ++d) o[d] *= f;
        }
      };
      auto weigh = [&](f16v &x, v8 (&p)[2], int key) {
#pragma unroll
        for (int i = 0; i < 16; ++i) x[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[i], a.scale, -m));
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const u4 b = {narrow2<kType>(x[8 * u], x[8 * u + 1]), narrow2<kType>(x[8 * u + 2], x[8 * u + 3]),
                        narrow2<kType>(x[8 * u + 4], x[8 * u + 5]), narrow2<kType>(x[8 * u + 6], x[8 * u + 7])};
          p[u] = __builtin_bit_cast(v8, b);
#pragma unroll
          for (int i = 0; i < 4; ++i) used = E::add2(b[i], used);
        }
        if (!exact) return;
        float part[2];
#pragma unroll
        for (int u = 0; u < 2; ++u)
          part[u] = ((x[8 * u] + x[8 * u + 1]) + (x[8 * u + 2] + x[8 * u + 3])) +
                    ((x[8 * u + 4] + x[8 * u + 5]) + (x[8 * u + 6] + x[8 * u + 7]));
        sum += part[0] + part[1];
        if (logs) {
          const int64_t run = (int64_t)a.window * a.q_heads;
          float *const to = logs + (key >> a.log_shift) * run;
          auto keep = [&](float x, float *to) {
            x += __shfl_xor(x, 32);
            if (hg == 0 && log_at >= 0) to[log_at] = __builtin_amdgcn_logf(x) + m;
          };
          if (a.log_shift == 5) {
            if (key < len) keep(part[0] + part[1], to);
          } else {
            if (key < len) keep(part[0], to);
            if (key + 16 < len) keep(part[1], to + run);
          }
        }
      };
      // what a stage's scales leave to 32 bits
      auto rest = [&](const char *from, int side, int sub) {
        return reinterpret_cast<const float *>(from + 2 * kSide)[side * kSubs + sub];
      };
      auto scale_o = [&](float f) {
#pragma unroll
        for (int d = 0; d < kOut; ++d) o[d] *= f;
      };
      auto add = [&](const v8 (&p)[2], const char *from, int h, bool apart) {
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          if (__builtin_expect(apart, false)) scale_o(inverse_unit(unit_of(rest(from, 1, 2 * h + u))));
#pragma unroll
          for (int d = 0; d < kOut; ++d) o[d] = E::mfma(vop[u][d], p[u], o[d]);
          if (__builtin_expect(apart, false)) scale_o(unit_of(rest(from, 1, 2 * h + u)));
        }
      };
      char *from = stages, *to = stages + stage_bytes(kType, kDim);
      look(first_key);
      fetch(first_key);
      put(from);
      fetch(first_key + kStage);
      __syncthreads();
      for (int key = first_key; key < block_end; key += kStage) {
        f16v x[kHalves];
        v8 p[kHalves][2];
        // a lane for each of the stage's, K's and V's
        const float any_rest = kBounded ? rest(from, 0, lane % (2 * kSubs)) : 1.f;
#pragma unroll
        for (int h = 0; h < kHalves; ++h) {
          load_k(from, h);
          scores(x[h]);
        }
        const unsigned odd = kBounded ? (unsigned)__ballot(any_rest != 1.f) : 0;
        if (__builtin_expect(odd & ((1u << kSubs) - 1), 0)) {
#pragma unroll
          for (int h = 0; h < kHalves; ++h)
#pragma unroll
            for (int i = 0; i < 16; ++i) x[h][i] *= rest(from, 0, 2 * h + (i >> 3));
        }
        load_v(from, 0);
#pragma unroll
        for (int h = 0; h < kHalves; ++h) limits(x[h], key + 32 * h);
        raise(x);
#pragma unroll
        for (int h = 0; h < kHalves; ++h) weigh(x[h], p[h], key + 32 * h);
        put(to);
        fetch(key + 2 * kStage);
        const bool apart = odd >> kSubs & ((1u << kSubs) - 1);
        add(p[0], from, 0, apart);
        if (kHalves > 1) {
          load_v(from, kHalves - 1);
          add(p[kHalves - 1], from, kHalves - 1, apart);
        }
        __syncthreads();
        char *const was = from;
        from = to;
        to = was;
      }
      if (__any(bad)) kv_report(a.status);
      __syncthreads();
    }

    sum += __shfl_xor(sum, 32);
    used += __shfl_xor(used, 32);
    if (!exact) sum = used;
    const float even = evened(sum, used);
    if (valid && at.key == 0 && stop == length) {
      const float f = (sum > 0.f ? 1.f / sum : sum == 0.f ? 0.f : sum) * even;
      char *out = a.out.data + (int64_t)(req.first + token) * a.out.token_stride + head * a.out.head_stride + 8 * hg;
#pragma unroll
      for (int d = 0; d < kOut; ++d)
#pragma unroll
        for (int j = 0; j < 4; ++j)
          *reinterpret_cast<u2 *>(out + 64 * d + 16 * j) =
              u2{narrow2<kType>(o[d][4 * j] * f, o[d][4 * j + 1] * f),
                 narrow2<kType>(o[d][4 * j + 2] * f, o[d][4 * j + 3] * f)};
      if (a.lse && hg == 0)
        a.lse[(int64_t)(req.first + token) * a.q_heads + head] = (m + __builtin_amdgcn_logf(sum)) * kLn2;
    } else if (valid) {
      const int64_t part = ((int64_t)w * 2 + (at.key > 0 ? 0 : 1)) * tile_rows(kDim) + row;
      float *to = a.parts + part * kDim + 4 * hg;
#pragma unroll
      for (int d = 0; d < kOut; ++d)
#pragma unroll
        for (int j = 0; j < 4; ++j)
          *reinterpret_cast<f4 *>(to + 32 * d + 8 * j) =
              f4{o[d][4 * j], o[d][4 * j + 1], o[d][4 * j + 2], o[d][4 * j + 3]} * even;
      if (hg == 0) *reinterpret_cast<f2 *>(a.part_sums + 2 * part) = f2{m, sum};
    }

    if (last) break;
    at.key = 0;
    if (++at.tile == seg.tiles()) {
      at.tile = 0;
      if (++at.head == a.kv.kv_heads) {
        at.head = 0;
        ++at.item;
      }
    }
  }
}

// Joins the parts of cut segments: a wave takes `each` rows, one after another.
template <int kType, int kDim>
__global__ __launch_bounds__(kBlock) void join_kernel(Attention a, int rows, int each) {
  constexpr int kLanes = kDim / 4, kParts = 64 / kLanes;
  const Split s = a.splits[blockIdx.x];
  if (s.request < 0) return;
  const int lane = lane_id();
  const int row0 = __builtin_amdgcn_readfirstlane(((int)blockIdx.y * kWaves + wave_id()) * each);
  const KvRequest req = kv_request(a.batch, a.row_offsets, a.kv.block_shift, s.request);
  // part 0 ends the range of the workgroup before the cut, the others begin theirs
  const int w = blockIdx.x, parts = s.last - w + 2;
  for (int row = row0; row < row0 + each; ++row) {
    const int token = s.tile * a.tile_tokens + row / a.group;
    if (row >= a.tile_tokens * a.group || token >= req.count) return;
    const int head = s.head * a.group + row % a.group;
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
}

// Adds to each table entry the weight that its request's last tokens gave it:
// one wave per entry, its runs' log sums against the rows' totals.
__global__ __launch_bounds__(kBlock) void weight_kernel(Attention a, float *block_weight) {
  __shared__ unsigned sums[kWaves];
  const int e0 = blockIdx.x * kWaves, lane = lane_id(), subs = a.kv.block_shift - a.log_shift;
  unsigned ended[1] = {0};
  for (int i = threadIdx.x; i < a.batch.n; i += kBlock) ended[0] += a.row_offsets[i + 1] <= e0;
  block_sum<1, unsigned>(ended, sums);
  int i = __builtin_amdgcn_readfirstlane((int)ended[0]);
  const int e = __builtin_amdgcn_readfirstlane(e0 + wave_id());
  while (i < a.batch.n && uniform_load(a.row_offsets + i + 1) <= e) ++i;
  if (i >= a.batch.n || e >= a.batch.n_entries) return;
  const KvRequest r = kv_request<true>(a.batch, a.row_offsets, a.kv.block_shift, i);
  if (!r.ok || e < r.row || (int64_t)(e - r.row) << a.kv.block_shift >= r.len || r.count == 0) return;
  const float *lse = a.lse + (int64_t)(r.first + r.count - 1) * a.q_heads;
  const float old = block_weight[e];
  float sum = 0.f;
  // 64 rows on: `step` of KV heads, tokens back and heads of the group
  int backs = 0, step[3], first[3];
  for (int s = 0; s < 1 << subs; ++s) {
    const int token = (((e - r.row) << subs) + s) << a.log_shift;  // the run's first
    // tokens more than `behind` back do not see it, and left no log sum
    const int behind = r.len - 1 - token;
    if (behind < 0) break;
    const int seen = min(min(a.window, r.count), behind + 1);
    if (seen != backs) {
      backs = seen;
      const int per = backs * a.group;
      step[0] = 64 / per, step[1] = 64 % per / a.group, step[2] = 64 % per % a.group;
      first[0] = lane / per, first[1] = lane % per / a.group, first[2] = lane % per % a.group;
    }
    const float *log = a.logs + (((int64_t)e << subs) + s) * a.window * a.q_heads;
    int kv_head = first[0], back = first[1], head = first[2];
#pragma unroll 4
    for (int j = lane; j < backs * a.q_heads; j += 64) {
      const float x = log[(kv_head * a.window + back) * a.group + head];
      sum += __builtin_amdgcn_exp2f(x - lse[kv_head * a.group + head - back * a.q_heads] * kLog2e);
      kv_head += step[0], back += step[1], head += step[2];
      if (head >= a.group) head -= a.group, ++back;
      if (back >= backs) back -= backs, ++kv_head;
    }
  }
#pragma unroll
  for (int d = 32; d; d >>= 1) sum += __shfl_xor(sum, d);
  if (lane == 0) block_weight[e] = old + sum;
}

// ------------------------------------------------------------------- host

constexpr int kCUs = 256;
// Up to this many tokens in the whole table nothing is cut, which saves the join
// (one request of 777 tokens: 11.8 us, cut 12.5; of 100: 8.0, with a join that
// finds nothing 11.4).  8 waves on a tile instead of 4 take 11.5 us for 777 tokens
// and 12.1 against 12.3 for 1024, but 10.4 against 9.9 for 512, 10.4 against 9.8
// for 777 of 64 dims, and no less for 2 to 4 requests.
constexpr int kUncut = 1024;
constexpr int kGroups = 4 * kCUs;      // workgroups of the kernel that splits tokens over waves
constexpr int kTileGroups = kCUs;   // of the kernel that splits rows over waves: one to a CU
constexpr int most_rows(int dim) { return dim == 256 ? 32 : 64; }  // of a request in the former

struct Workspace {
  size_t splits, tile_splits, parts, tile_parts, sums, tile_sums, lse, logs, total;
};

int log_shift(const cascade_kv_format_t *f) { return f->block_tokens >= 32 ? 5 : 4; }

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
  w.tile_parts = take(sizeof(float) * kTileGroups * 2 * tile_rows(f->head_dim) * f->head_dim);
  w.sums = take(sizeof(float) * kGroups * 2 * most_rows(f->head_dim) * 2);
  w.tile_sums = take(sizeof(float) * kTileGroups * 2 * tile_rows(f->head_dim) * 2);
  w.lse = take(window ? sizeof(float) * b->n_tokens * q_heads : 0);
  w.logs = take(window ? sizeof(float) * ((size_t)b->n_entries * f->block_tokens >> log_shift(f)) * window * q_heads : 0);
  w.total = at;
  return w;
}

bool heads_ok(const cascade_kv_format_t *f, int q_heads) {
  return q_heads >= 1 && q_heads % f->kv_heads == 0 && q_heads / f->kv_heads <= 128;
}

template <int kType, int kDim, int kTiles>
void start(const Attention &a, int grid, Cap cap, hipStream_t stream) {
  const size_t mix = sizeof(float) * kWaves * 16 * (2 + (kDim < 128 ? kDim : 128) + 4);
  auto kernel =
      cap == Cap::kWide     ? attention_kernel<kType, kDim, kTiles, Cap::kWide>
      : cap == Cap::kNarrow ? attention_kernel<kType, kDim, kTiles, Cap::kNarrow>
                            : attention_kernel<kType, kDim, kTiles, Cap::kNone>;
  hipLaunchKernelGGL(kernel, dim3(grid), dim3(64 * kWaves), list_bytes(a.batch.n) + mix, stream, a);
}

template <int kType, int kDim>
void start_tiles(const Attention &a, Cap cap, hipStream_t stream) {
  auto kernel = cap == Cap::kWide     ? tile_kernel<kType, kDim, Cap::kWide>
                : cap == Cap::kNarrow ? tile_kernel<kType, kDim, Cap::kNarrow>
                                      : tile_kernel<kType, kDim, Cap::kNone>;
  hipLaunchKernelGGL(kernel, dim3(kTileGroups), dim3(64 * tile_waves(kDim)),
                     list_bytes(a.batch.n) + 2 * stage_bytes(kType, kDim), stream, a);
}

template <int kType, int kDim>
int run(Attention a, char *ws, const Workspace &w, Cap cap, float *block_weight, hipStream_t s) {
  const int64_t most = (int64_t)a.batch.max_new * a.group;  // rows of a request and KV head
  const int64_t table = (int64_t)a.batch.n_entries << a.kv.block_shift;  // no request is longer
  const int64_t keys = table * a.kv.kv_heads;
  // few rows: 4 waves share a tile's tokens.  More: row tiles, and requests of
  // up to 32 rows beside them in the first kernel.
  const bool tiled = most > most_rows(kDim);
  const int small = most <= 16 ? 16 : most <= 32 || tiled ? 32 : 64;
  if (!tiled || a.batch.n > 1) {
    a.min_rows = 0;
    a.max_rows = small;
    a.tile_tokens = small / a.group > 0 ? small / a.group : 1;
    // Up to 512 tokens a cut costs more than it evens out (128 requests of 582
    // tokens on average, 64 heads: 57 us, with every cut made 64).
    a.least_keys = a.atomic_keys = table <= kUncut ? kUncut : 512;
    a.cut_keys = 32;
    a.range_keys = 256;
    a.splits = reinterpret_cast<Split *>(ws + w.splits);
    a.parts = reinterpret_cast<float *>(ws + w.parts);
    a.part_sums = reinterpret_cast<float *>(ws + w.sums);
    // as many workgroups as there is work for (a segment's fixed cost counts: 8
    // requests of 100 tokens 8.0 us, without it 15.1) and as fit the GPU at once
    const int64_t room = kCUs * waves_per_simd(kDim, small / 16);
    const int64_t work = (keys + (int64_t)a.batch.n * a.kv.kv_heads * kFixedKeys) / a.range_keys;
    const int grid = (int)std::min(std::min<int64_t>(kGroups, room), std::max<int64_t>(8, work));
    if (small == 16)
      start<kType, kDim, 1>(a, grid, cap, s);
    else if (small == 32)
      start<kType, kDim, 2>(a, grid, cap, s);
    else if constexpr (kDim < 256)
      start<kType, kDim, 4>(a, grid, cap, s);
    if (table > a.atomic_keys)  // else none is cut
      hipLaunchKernelGGL((join_kernel<kType, kDim>), dim3(grid, small / kWaves), dim3(kBlock), 0, s, a, small, 1);
  }
  if (tiled) {
    a.min_rows = a.batch.n > 1 ? small : 0;
    a.max_rows = INT64_MAX;
    a.tile_tokens = tile_rows(kDim) / a.group;
    // shorter ones are cut where there are few (64 rows of each of 8 KV heads, 2000
    // tokens: 37 us, uncut 61), but not those of up to 16 stages (512 rows of 600
    // tokens: 29 us, cut 35)
    a.least_keys = 16 * stage_tokens(kDim);
    a.atomic_keys = 2048;
    a.cut_keys = stage_tokens(kDim);
    a.range_keys = 256;
    a.splits = reinterpret_cast<Split *>(ws + w.tile_splits);
    a.parts = reinterpret_cast<float *>(ws + w.tile_parts);
    a.part_sums = reinterpret_cast<float *>(ws + w.tile_sums);
    start_tiles<kType, kDim>(a, cap, s);
    if (table > a.least_keys)
      hipLaunchKernelGGL((join_kernel<kType, kDim>), dim3(kTileGroups, tile_rows(kDim) / (2 * kWaves)), dim3(kBlock),
                         0, s, a, tile_rows(kDim), 2);
  }
  if (block_weight)
    hipLaunchKernelGGL(weight_kernel, dim3((a.batch.n_entries + kWaves - 1) / kWaves), dim3(kBlock), 0,
                       s, a, block_weight);
  return hipGetLastError() == hipSuccess ? CASCADE_OK : CASCADE_EHIP;
}

template <int kType>
int run(const Attention &a, char *ws, const Workspace &w, Cap cap, float *block_weight, hipStream_t s) {
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
  const Cap cap = args->softcap > kNarrowLimit ? Cap::kWide : args->softcap > 0 ? Cap::kNarrow : Cap::kNone;
  // softmax(-s q.k) is softmax(s (-q).k): the largest score is then that of
  // the largest product
  const double scale = std::fabs(args->scale), softcap = args->softcap;
  const auto held = [](double x) { return (float)std::min<double>(x, std::numeric_limits<float>::max()); };
  a.flip = args->scale < 0 ? 0x80008000u : 0u;
  a.keep = scale > 0 ? ~0u : 0u;
  a.scale = cap == Cap::kWide ? 1.f : held((cap == Cap::kNarrow ? softcap : scale > 0 ? scale : 1) * kLog2e);
  if (cap != Cap::kNone) {
    a.cap_in = held(2 * kLog2e * scale / softcap);
    a.cap_y = held(scale / softcap);
    a.qk = held(scale * kLog2e);
    a.cap = held(softcap * kLog2e);
  }
  char *ws = static_cast<char *>(workspace);
  a.window = args->weight_window;
  a.lse = args->lse ? args->lse : a.window ? reinterpret_cast<float *>(ws + w.lse) : nullptr;
  a.log_shift = log_shift(format);
  a.logs = a.window && batch->n_entries ? reinterpret_cast<float *>(ws + w.logs) : nullptr;
  a.status = status_dev;
  const auto s = static_cast<hipStream_t>(stream);
  float *weight = a.logs ? args->block_weight : nullptr;
  return args->dtype == CASCADE_BF16 ? run<CASCADE_BF16>(a, ws, w, cap, weight, s)
                                     : run<CASCADE_F16>(a, ws, w, cap, weight, s);
}
