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
// a token in a lane, and halves the dims it answers for at each exchange.
// score: a wave holds the queries of 16 rows (tokens and heads of a group) as the
// first operand and takes 16 blocks at a time as the second, so a lane has one
// block's scores of 4 rows, and the largest over a group's heads is taken in
// registers.  select: a workgroup takes one token and head, finds the
// least score that stays by a radix selection in LDS, and writes the blocks in
// order by ballots.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "cascade.h"
#include "device_util.h"
#include "kv_format.h"

namespace cascade {
namespace {

typedef int i4 __attribute__((ext_vector_type(4)));
typedef unsigned u4 __attribute__((ext_vector_type(4)));
typedef _Float16 h2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf2 __attribute__((ext_vector_type(2)));

constexpr int kMinExponent = -100;  // of a row of whole queries

// From a chunk's begin to its head's bounds.
__device__ __forceinline__ int64_t bounds_at(const KvView &kv, int head) {
  const int64_t codes = (int64_t)kv.kv_heads * kv.head_dim << kv.block_shift;
  return codes + (4 * kv.kv_heads + 15) / 16 * 16 + (int64_t)head * kv.head_dim;
}
__device__ __forceinline__ int64_t scale_at(const KvView &kv, int head) {
  return ((int64_t)kv.kv_heads * kv.head_dim << kv.block_shift) + 4 * head;
}

// The request that unit `at` of a list lies in, by the ends of the requests'
// parts: how many end at or before it.  Called by all threads.
__device__ __forceinline__ int owner_of(const int32_t *offsets, int n, int at, unsigned *lds) {
  unsigned ended[1] = {0};
  for (int i = threadIdx.x; i < n; i += kBlock) ended[0] += offsets[i + 1] <= at;
  block_sum<1, unsigned>(ended, lds);
  return (int)ended[0];
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
  for (int t0 = 0; t0 < tokens; t0 += 16) {
    if (t0 + lane / 4 >= tokens) continue;
#pragma unroll
    for (int c = 0; c < kDim / 64; ++c) {
      const u4 w = *reinterpret_cast<const u4 *>(codes + t0 * kDim + 1024 * c + 16 * lane);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const h2 x = __builtin_bit_cast(h2, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w[i], 1.f, false));
        const h2 y = __builtin_bit_cast(h2, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w[i], 1.f, true));
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
#pragma unroll
    for (int keep = 4, mask = 32; keep; keep >>= 1, mask >>= 1) {
      const bool upper = lane & mask;
#pragma unroll
      for (int i = 0; i < keep; ++i) {
        const h2 mine = upper ? top[c][keep + i] : top[c][i], give = upper ? top[c][i] : top[c][keep + i];
        top[c][i] = larger(mine, other_lane(give, mask));
        const h2 mine_low = upper ? low[c][keep + i] : low[c][i], give_low = upper ? low[c][i] : low[c][keep + i];
        low[c][i] = smaller(mine_low, other_lane(give_low, mask));
      }
      first += upper ? keep : 0;
    }
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
    check_requests(a.batch, a.row_offsets, a.kv.block_shift, a.status);
    return;
  }
  __shared__ unsigned sums[kWaves];
  const int u0 = blockIdx.x * a.group, u1 = min(u0 + a.group, a.units);
  int i = owner_of(a.whole ? a.row_offsets : a.batch.token_offsets, a.batch.n, u0, sums);
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
      for (int head = wave_id(); head < a.kv.kv_heads; head += kWaves) bound_block<kDim>(a, slot, head, tokens);
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
  int keep, sink, recent;
  int span;    // table entries of a workgroup
  float *scores;  // request by request [token][KV head][block], as many as max_new tokens would take
  int32_t *selected;
  int32_t *status;
};

__device__ __forceinline__ int blocks_of(const KvRequest &r, int block_shift) {
  return (int)(((long long)r.len + (1 << block_shift) - 1) >> block_shift);
}
__device__ __forceinline__ float *scores_of(const Select &a, const KvRequest &r, int token, int head) {
  const int64_t first = (int64_t)r.row * a.batch.max_new * a.kv.kv_heads;
  return a.scores + first + ((int64_t)token * a.kv.kv_heads + head) * blocks_of(r, a.kv.block_shift);
}

template <int kType>
__device__ __forceinline__ void widen2(unsigned w, float &a, float &b) {
  if constexpr (kType == CASCADE_BF16) {
    const bf2 x = __builtin_bit_cast(bf2, w);
    a = (float)x[0], b = (float)x[1];
  } else {
    const h2 x = __builtin_bit_cast(h2, w);
    a = (float)x[0], b = (float)x[1];
  }
}

// 16 rows of queries in whole numbers, in operand order: lane % 16 is the row, lane
// / 16 its dims 16 (lane / 16) of each 64.
template <int kType, int kDim>
struct Queries {
  i4 plus[kDim / 64], minus[kDim / 64];
  int exponent;  // of the lane's row
  bool bad = false;

  __device__ __forceinline__ void load(const Select &a, const KvRequest &r, int head, int token, int of_group,
                                       bool valid) {
    const char *from = a.q.data + (int64_t)(r.first + (valid ? token : 0)) * a.q.token_stride +
                       (int64_t)(head * a.group + (valid ? of_group : 0)) * a.q.head_stride + 32 * (lane_id() >> 4);
    float x[kDim / 64][16], most = 0.f;
#pragma unroll
    for (int s = 0; s < kDim / 64; ++s)
#pragma unroll
      for (int v = 0; v < 2; ++v) {
        const u4 w = *reinterpret_cast<const u4 *>(from + 128 * s + 16 * v);
#pragma unroll
        for (int i = 0; i < 4; ++i) widen2<kType>(w[i], x[s][8 * v + 2 * i], x[s][8 * v + 2 * i + 1]);
      }
#pragma unroll
    for (int s = 0; s < kDim / 64; ++s)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const bool fine = __builtin_isfinite(x[s][i]);
        bad |= valid && !fine;
        x[s][i] = valid && fine ? x[s][i] : 0.f;
        most = fmaxf(most, fabsf(x[s][i]));
      }
    most = fmaxf(most, __shfl_xor(most, 16));
    most = fmaxf(most, __shfl_xor(most, 32));
    // the least with most <= 127 * 2^exponent; 127 is 1.984375 * 2^6
    const unsigned b = __float_as_uint(most);
    exponent = max((int)(b >> 23) - 127 - 6 + ((b & 0x7fffffu) > 0x7e0000u ? 1 : 0), kMinExponent);
    const float inverse = __uint_as_float((unsigned)(127 - exponent) << 23);
#pragma unroll
    for (int s = 0; s < kDim / 64; ++s)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        int p = 0, m = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int n = (int)__builtin_rintf(x[s][4 * i + j] * inverse);
          p |= max(n, 0) << 8 * j;
          m |= (min(n, 0) & 255) << 8 * j;
        }
        plus[s][i] = p, minus[s][i] = m;
      }
  }
};

// The scores of a wave's `kTiles` row sets over blocks begin .. end of a request.
template <int kType, int kDim, int kTiles>
__device__ __forceinline__ void score_blocks(const Select &a, const KvRequest &r, int head, int tile0, int begin,
                                             int end) {
  constexpr int kSteps = kDim / 64;
  const int lane = lane_id(), n16 = lane & 15, g = lane >> 4;
  const bool wide = a.padded > 16;  // a token's heads take several row sets, one after another
  const int per_tile = wide ? 1 : 16 / a.padded, passes = wide ? a.padded / 16 : 1;
  int top_all = kMinExponent;
  if (wide) {
    for (int p = 0; p < passes; ++p) {
      Queries<kType, kDim> q;
      const int of_group = 16 * p + n16;
      const bool valid = of_group < a.group && tile0 < r.count;
      q.load(a, r, head, tile0, of_group, valid);
      top_all = max(top_all, valid ? q.exponent : kMinExponent);
    }
#pragma unroll
    for (int m = 8; m; m >>= 1) top_all = max(top_all, __shfl_xor(top_all, m));
  }
  bool bad_query = false, bad_slot = false;
  for (int p = 0; p < passes; ++p) {
    Queries<kType, kDim> q[kTiles];
    float weight[kTiles][4], pad[kTiles][4];
#pragma unroll
    for (int t = 0; t < kTiles; ++t) {
      const int tile = tile0 + t, token = tile * per_tile + (wide ? 0 : n16 / a.padded);
      const int of_group = wide ? 16 * p + n16 : n16 & (a.padded - 1);
      const bool valid = token < r.count && of_group < a.group;
      q[t].load(a, r, head, token, of_group, valid);
      bad_query |= q[t].bad;
      // relative to the largest of the token's heads: every product is exact, and none overflows
      int top = valid ? q[t].exponent : kMinExponent;
      for (int m = 1; m < min(a.padded, 16); m <<= 1) top = max(top, __shfl_xor(top, m));
      if (wide) top = top_all;
      const float w = valid ? __uint_as_float((unsigned)(127 + max(q[t].exponent - top, -126)) << 23) : 0.f;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        weight[t][i] = __shfl(w, 4 * g + i);
        pad[t][i] = weight[t][i] > 0.f ? 0.f : -__builtin_inff();
      }
    }
    for (int b0 = begin; b0 < end; b0 += 16) {
      const int b = b0 + n16;
      int slot = a.slots[r.row + min(b, end - 1)];
      if ((unsigned)slot >= (unsigned)a.kv.num_slots) bad_slot = true, slot = 0;
      const char *const chunk = a.kv.base + slot * a.kv.slot_stride;
      const char *const from = chunk + bounds_at(a.kv, head) + 16 * g;
      i4 upper[kSteps], lower[kSteps];
#pragma unroll
      for (int s = 0; s < kSteps; ++s) {
        upper[s] = *reinterpret_cast<const i4 *>(from + 64 * s);
        lower[s] = *reinterpret_cast<const i4 *>(from + a.kv.kv_stride + 64 * s);
      }
      const float scale = *reinterpret_cast<const float *>(chunk + scale_at(a.kv, head));
#pragma unroll
      for (int t = 0; t < kTiles; ++t) {
        i4 sum = {0, 0, 0, 0};
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
          sum = __builtin_amdgcn_mfma_i32_16x16x64_i8(q[t].plus[s], upper[s], sum, 0, 0, 0);
          sum = __builtin_amdgcn_mfma_i32_16x16x64_i8(q[t].minus[s], lower[s], sum, 0, 0, 0);
        }
        float x[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = __builtin_fmaf((float)sum[i], weight[t][i], pad[t][i]);
        // over the heads of a token: rows 4 g + i of the set
        int tokens = 4;  // of the lane's 4 rows
        if (a.padded >= 2) x[0] = fmaxf(x[0], x[1]), x[1] = fmaxf(x[2], x[3]), tokens = 2;
        if (a.padded >= 4) x[0] = fmaxf(x[0], x[1]), tokens = 1;
        if (a.padded >= 8) x[0] = fmaxf(x[0], __shfl_xor(x[0], 16));
        if (a.padded >= 16) x[0] = fmaxf(x[0], __shfl_xor(x[0], 32));
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int token = wide ? tile0 : (tile0 + t) * per_tile + (4 * g + i * (4 / tokens)) / a.padded;
          const bool first = (4 * g & (min(a.padded, 16) - 1)) == 0;  // of a token's lanes
          if (i >= tokens || !first || token >= r.count || b >= end) continue;
          float *const to = scores_of(a, r, token, head) + b;
          const float y = x[i] * scale + 0.f;  // no -0
          *to = p ? fmaxf(*to, y) : y;
        }
      }
    }
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

template <int kType, int kDim, int kTiles>
__global__ __launch_bounds__(kBlock) void score_kernel(Select a) {
  __shared__ unsigned sums[kWaves];
  const int e0 = blockIdx.x * a.span, e1 = min(e0 + a.span, a.batch.n_entries);
  const int per_tile = a.padded > 16 ? 1 : 16 / a.padded;
  for (int i = owner_of(a.row_offsets, a.batch.n, e0, sums); i < a.batch.n && a.row_offsets[i] < e1; ++i) {
    const KvRequest r = kv_request(a.batch, a.row_offsets, a.kv.block_shift, i);
    const int tile0 = blockIdx.y * kTiles;
    if (!r.ok || tile0 * per_tile >= r.count) continue;
    const Candidates c(a, blocks_of(r, a.kv.block_shift));
    const int begin = max(c.begin, e0 - r.row), end = min(c.end, e1 - r.row);
    if (begin >= end) continue;
    for (int head = wave_id(); head < a.kv.kv_heads; head += kWaves)
      score_blocks<kType, kDim, kTiles>(a, r, head, tile0, begin, end);
  }
}

// ------------------------------------------------------------------ select

// Scores in ascending order as whole numbers, NaN last.
__device__ __forceinline__ unsigned ordered(float x) {
  const unsigned b = __float_as_uint(x);
  if ((b & 0x7fffffffu) > 0x7f800000u) return 0xffffffffu;
  return b >> 31 ? ~b : b | 0x80000000u;
}

constexpr int kHeld = 8;     // scores of a thread that stay in registers
constexpr int kDigits = 2048;

__global__ __launch_bounds__(kBlock) void select_kernel(Select a) {
  if (blockIdx.x == gridDim.x - 1) {
    check_requests(a.batch, a.row_offsets, a.kv.block_shift, a.status);
    return;
  }
  __shared__ unsigned hist[kDigits], scan[kWaves], found[3], marks[2][kWaves];
  const int token = blockIdx.x / a.kv.kv_heads, head = blockIdx.x % a.kv.kv_heads;
  const int i = owner_of(a.batch.token_offsets, a.batch.n, token, scan);
  if (i >= a.batch.n) return;
  const KvRequest r = kv_request(a.batch, a.row_offsets, a.kv.block_shift, i);
  if (!r.ok || token < r.first || token - r.first >= r.count) return;
  const int j = token - r.first, last = r.len - r.count + j;  // cached token
  const int blocks = last < 0 ? 0 : (last >> a.kv.block_shift) + 1;
  int32_t *const out = a.selected + ((int64_t)token * a.kv.kv_heads + head) * a.keep;
  const int tid = threadIdx.x, lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(wave_id());
  if (blocks <= a.keep) {
    for (int k = tid; k < a.keep; k += kBlock) out[k] = k < blocks ? k : -1;
    return;
  }
  const int begin = a.sink, end = blocks - a.recent, want = a.keep - a.sink - a.recent;
  for (int k = tid; k < a.sink; k += kBlock) out[k] = k;
  for (int k = tid; k < a.recent; k += kBlock) out[a.keep - a.recent + k] = end + k;
  if (want == 0) return;

  // each wave has a run of candidates, 64 at a time
  const float *const score = scores_of(a, r, j, head);
  const int each = ((end - begin + kBlock - 1) / kBlock) * 64;
  const int from = begin + wave * each, to = min(from + each, end);
  unsigned held[kHeld];
#pragma unroll
  for (int k = 0; k < kHeld; ++k) {
    const int b = from + 64 * k + lane;
    held[k] = b < to ? ordered(score[b]) : 0;
  }
  auto each_key = [&](auto f) {
#pragma unroll
    for (int k = 0; k < kHeld; ++k)
      if (from + 64 * k < to) f(held[k], from + 64 * k + lane);
    for (int b0 = from + 64 * kHeld; b0 < to; b0 += 64) {
      const int b = b0 + lane;
      f(b < to ? ordered(score[b]) : 0, b);
    }
  };
  // the want-th largest: its digits as far as they are needed
  unsigned key = 0, known = 0, rank = want - 1, equal = ~0u;
#pragma unroll 1
  for (int pass = 0; pass < 3; ++pass) {
    const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0;
    const unsigned mask = pass == 2 ? 1023u : 2047u;
    for (int d = tid; d < kDigits; d += kBlock) hist[d] = 0;
    __syncthreads();
    each_key([&](unsigned k, int b) {
      if (b < to && ((k ^ key) & known) == 0) atomicAdd(&hist[k >> shift & mask], 1u);
    });
    __syncthreads();
    // 8 digits to a thread, from the largest
    unsigned h[8], sum[1] = {0}, all[1];
#pragma unroll
    for (int d = 0; d < 8; ++d) sum[0] += h[d] = hist[kDigits - 1 - 8 * tid - d];
    const unsigned mine = sum[0];
    block_exclusive_scan<1, unsigned>(sum, all, scan);
    unsigned at = sum[0];
    if (rank >= at && rank < at + mine) {
#pragma unroll
      for (int d = 0; d < 8; ++d) {
        if (rank >= at && rank < at + h[d]) {
          found[0] = kDigits - 1 - 8 * tid - d;
          found[1] = rank - at;
          found[2] = h[d];
        }
        at += h[d];
      }
    }
    __syncthreads();
    key |= found[0] << shift;
    known |= mask << shift;
    rank = found[1];
    if (rank + 1 == found[2]) {  // all that share these digits stay
      equal = ~0u;
      break;
    }
    equal = rank + 1;  // the first of those that share all digits
    __syncthreads();
  }
  // above the key, and equal to it as far as its digits are known
  unsigned above = 0, same = 0;
  each_key([&](unsigned k, int b) {
    above += __popcll(__ballot(b < to && (k & known) > key));
    same += __popcll(__ballot(b < to && (k & known) == key));
  });
  if (lane == 0) marks[0][wave] = above, marks[1][wave] = same;
  __syncthreads();
  unsigned place = a.sink, ties = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    if (w < wave) place += marks[0][w] + min(marks[1][w], equal - min(equal, ties)), ties += marks[1][w];
  }
  each_key([&](unsigned k, int b) {
    const uint64_t same = __ballot(b < to && (k & known) == key);
    const bool tie = (same >> lane & 1) && ties + rank_in_mask(same) < equal;
    const uint64_t stay = __ballot((b < to && (k & known) > key) || tie);
    if (stay >> lane & 1) out[place + rank_in_mask(stay)] = b;
    place += __popcll(stay);
    ties += __popcll(same);
  });
}

// ------------------------------------------------------------------- host

bool bounds_fit(const cascade_kv_pool_t *p, const cascade_kv_format_t *f) {
  return p->chunk_bytes >= kv_chunk_bytes(f) + (int64_t)f->kv_heads * f->head_dim;
}

size_t score_bytes(const cascade_kv_format_t *f, const cascade_kv_batch_t *b) {
  return (sizeof(float) * b->n_entries * b->max_new * f->kv_heads + 255) & ~(size_t)255;
}

template <int kType, int kTiles>
void score(const Select &a, dim3 grid, hipStream_t stream) {
  auto kernel = a.kv.head_dim == 64    ? score_kernel<kType, 64, kTiles>
                : a.kv.head_dim == 128 ? score_kernel<kType, 128, kTiles>
                                       : score_kernel<kType, 256, kTiles>;
  hipLaunchKernelGGL(kernel, grid, dim3(kBlock), 0, stream, a);
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
  a.status = status_dev;
  const int grid = (a.units - 1) / a.group + 2;  // the last one checks the batch
  auto kernel = format->head_dim == 64    ? bounds_kernel<64>
                : format->head_dim == 128 ? bounds_kernel<128>
                                          : bounds_kernel<256>;
  hipLaunchKernelGGL(kernel, dim3(grid), dim3(kBlock), 0, static_cast<hipStream_t>(stream), a);
  return hipGetLastError() == hipSuccess ? CASCADE_OK : CASCADE_EHIP;
}

extern "C" size_t cascade_kv_select_workspace_bytes(const cascade_kv_format_t *format,
                                                    const cascade_kv_batch_t *batch) {
  if (!kv_format_ok(format) || !batch || batch->max_new < 0 || batch->n_entries < 0) return 0;
  return score_bytes(format, batch) + 256;
}

extern "C" int cascade_kv_select(const cascade_kv_pool_t *pool, int32_t layer, const cascade_kv_format_t *format,
                                 const cascade_kv_batch_t *batch, const cascade_block_table_t *table,
                                 const cascade_select_t *args, void *workspace, size_t workspace_bytes,
                                 int32_t *status_dev, void *stream) {
  if (!kv_pool_ok(pool, layer, format) || !bounds_fit(pool, format) || !kv_batch_ok(batch, table) || !args)
    return CASCADE_EINVAL;
  if ((args->dtype != CASCADE_BF16 && args->dtype != CASCADE_F16) || args->q_heads < 1 ||
      args->q_heads % format->kv_heads || args->q_heads / format->kv_heads > 128 || args->sink < 0 ||
      args->recent < 1 || args->keep > 65536 || (int64_t)args->sink + args->recent > args->keep)
    return CASCADE_EINVAL;
  if (!workspace || ((uintptr_t)workspace & 255)) return CASCADE_EINVAL;
  if (workspace_bytes < cascade_kv_select_workspace_bytes(format, batch)) return CASCADE_ENOSPC;
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
  a.keep = args->keep;
  a.sink = args->sink;
  a.recent = args->recent;
  a.scores = static_cast<float *>(workspace);
  a.selected = args->selected;
  a.status = status_dev;
  const int64_t rows = (int64_t)batch->n_tokens * format->kv_heads;
  if (rows >= INT32_MAX) return CASCADE_EINVAL;
  const auto s = static_cast<hipStream_t>(stream);
  const int per_tile = a.padded > 16 ? 1 : 16 / a.padded;
  const int tiles = (batch->max_new + per_tile - 1) / per_tile;
  const bool many = tiles >= 4 && a.padded <= 16;
  const int sets = many ? (tiles + 3) / 4 : tiles;
  if (sets > 65535) return CASCADE_EINVAL;
  a.span = 64;
  if (batch->n_entries > a.keep) {  // else every token keeps all that it sees
    const dim3 grid((batch->n_entries + a.span - 1) / a.span, sets);
    if (args->dtype == CASCADE_BF16) {
      if (many) score<CASCADE_BF16, 4>(a, grid, s); else score<CASCADE_BF16, 1>(a, grid, s);
    } else {
      if (many) score<CASCADE_F16, 4>(a, grid, s); else score<CASCADE_F16, 1>(a, grid, s);
    }
  }
  hipLaunchKernelGGL(select_kernel, dim3((unsigned)rows + 1), dim3(kBlock), 0, s, a);
  return hipGetLastError() == hipSuccess ? CASCADE_OK : CASCADE_EHIP;
}
