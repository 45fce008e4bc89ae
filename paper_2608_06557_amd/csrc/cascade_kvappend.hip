// cascade_kvappend.hip -- new tokens into the 8-bit paged KV cache on gfx950.
//
// One launch rotates the queries and writes keys and values.  A unit of a row
// is 16 dims, 8 of them at two places `reach` apart (half layout) or side by
// side (interleaved), so that a lane holds both members of its 8 pairs.
//
// Angles: position * freq in 64 bits is the fraction of a turn in 2^-64,
// whole turns dropped by the wrap; its high half as a float is exact to 2^-24
// of itself, and the sine unit takes turns.
//
// Keys and values go by runs: the new tokens of one request that share a
// block.  One wave owns a run of one head's K or V, so it alone reads and
// writes that block's codes and scale.  It takes the largest magnitude, the
// scale 2^ceil(log2(max / 448)), and rounds once from 32 bits.  Codes are
// gathered in LDS in the layout of the cache and leave 16 bytes a lane.  When a block's scale
// grows, the codes of its older tokens are multiplied by the (exact) ratio
// and rounded again, which changes only those that fall below E4M3's normal
// range: with powers of two a block rounds an element at most once there per
// doubling.
//
// Bound by HBM: 8192 tokens of 32 query and 8 KV heads of 128 dims, 185 MB in
// 43 to 46 us (4.1 to 4.3 TB/s; a large copy reaches 4.7).  Single tokens are
// bound by the latency of dependent loads (128 requests: 8 us), since a run
// reads its block's scale and codes before it writes.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <cmath>

#include "cascade.h"
#include "device_util.h"
#include "kv_format.h"

namespace cascade {
namespace {

constexpr int kMinExponent = -100;  // of a scale

typedef float f2 __attribute__((ext_vector_type(2)));
typedef unsigned u4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf2 __attribute__((ext_vector_type(2)));
typedef _Float16 h2 __attribute__((ext_vector_type(2)));

template <int kType> struct Pair { typedef bf2 type; };
template <> struct Pair<CASCADE_F16> { typedef h2 type; };

template <int kType>
__device__ __forceinline__ void widen(u4 raw, float (&x)[8]) {
  typedef typename Pair<kType>::type P;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const P p = __builtin_bit_cast(P, (unsigned)raw[i]);
    x[2 * i] = (float)p[0];
    x[2 * i + 1] = (float)p[1];
  }
}

template <int kType>
__device__ __forceinline__ u4 narrow(const float (&x)[8]) {
  typedef typename Pair<kType>::type P;
  u4 raw;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const f2 f = {x[2 * i], x[2 * i + 1]};
    raw[i] = __builtin_bit_cast(unsigned, __builtin_convertvector(f, P));
  }
  return raw;
}

struct Rope {
  const uint64_t *freq;
  const int32_t *positions;
  int dim;  // 0: no rotation
  int interleaved;
  float scale;
};

// The two places of 8 dims that unit `u` of a row covers.
__device__ __forceinline__ void unit_dims(const Rope &r, int u, int &a, int &b) {
  if (16 * u < r.dim && !r.interleaved) {
    a = 8 * u;
    b = a + r.dim / 2;
  } else {
    a = 16 * u;
    b = a + 8;
  }
}

__device__ __forceinline__ void turn(const Rope &r, int j, int p, float &a, float &b) {
  const uint64_t t = (uint64_t)(uint32_t)p * r.freq[j];
  const float turns = (float)(int32_t)(t >> 32) * 0x1p-32f;
  const float c = __builtin_amdgcn_cosf(turns) * r.scale;
  const float s = __builtin_amdgcn_sinf(turns) * r.scale;
  const float a0 = a, b0 = b;
  a = a0 * c - b0 * s;
  b = b0 * c + a0 * s;
}

// Turns the 8 pairs of unit u (x: first place, y: second) at position p.
__device__ __forceinline__ void rotate_unit(const Rope &r, int u, int p, float (&x)[8],
                                            float (&y)[8]) {
  if (16 * u >= r.dim) return;
  if (r.interleaved) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      turn(r, 8 * u + j, p, x[2 * j], x[2 * j + 1]);
      turn(r, 8 * u + 4 + j, p, y[2 * j], y[2 * j + 1]);
    }
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) turn(r, 8 * u + j, p, x[j], y[j]);
  }
}

__device__ __forceinline__ float codes_max(float a, float b) { return fmaxf(a, fabsf(b)); }

// Exponent e of the smallest power of two with amax <= 448 * 2^e, amax >= 0
// finite.  448 = 1.75 * 2^8.
__device__ __forceinline__ int scale_exponent(float amax) {
  const unsigned b = __float_as_uint(amax);
  const int e = (int)(b >> 23) - 127 - 8 + ((b & 0x7fffffu) > 0x600000u ? 1 : 0);
  return e < kMinExponent ? kMinExponent : e;
}
__device__ __forceinline__ float power_of_two(int e) { return __uint_as_float((unsigned)(e + 127) << 23); }

__device__ __forceinline__ unsigned codes4(float a, float b, float c, float d) {
  int r = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  r = __builtin_amdgcn_cvt_pk_fp8_f32(c, d, r, true);
  return (unsigned)r;
}

__device__ __forceinline__ unsigned rescale4(unsigned w, float ratio) {
  const f2 lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false);
  const f2 hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
  return codes4(lo[0] * ratio, lo[1] * ratio, hi[0] * ratio, hi[1] * ratio);
}

__device__ __forceinline__ void wave_sync() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

struct Rows {
  char *data;
  int64_t token_stride, head_stride;  // bytes
};
__device__ __forceinline__ u4 load_row(const Rows &r, int t, int h, int d) {
  return *reinterpret_cast<const u4 *>(r.data + t * r.token_stride + h * r.head_stride + 2 * d);
}

struct Append {
  KvView kv;
  cascade_kv_batch_t batch;
  const int32_t *row_offsets, *slots;
  Rows q, q_out, k, v;
  Rope rope;
  int q_heads;
  int q_blocks;  // leading workgroups that rotate queries
  int group;     // tokens whose runs one workgroup looks for
  int32_t *status;
};

template <int kType, int kDim>
__device__ __forceinline__ void rotate_queries(const Append &a) {
  constexpr int kUnits = kDim / 16;
  const int64_t id = (int64_t)blockIdx.x * kBlock + threadIdx.x;
  const int u = (int)(id % kUnits);
  const int64_t row = id / kUnits;
  const int t = (int)(row / a.q_heads), h = (int)(row % a.q_heads);
  if (t >= a.batch.n_tokens) return;
  const int p = a.rope.dim ? a.rope.positions[t] : 0;
  int da, db;
  unit_dims(a.rope, u, da, db);
  float x[8], y[8];
  widen<kType>(load_row(a.q, t, h, da), x);
  widen<kType>(load_row(a.q, t, h, db), y);
  if (p < 0) {
    kv_report(a.status);
    return;
  }
  rotate_unit(a.rope, u, p, x, y);
  char *out = a.q_out.data + t * a.q_out.token_stride + h * a.q_out.head_stride;
  *reinterpret_cast<u4 *>(out + 2 * da) = narrow<kType>(x);
  *reinterpret_cast<u4 *>(out + 2 * db) = narrow<kType>(y);
}

// One wave: tokens t .. t + m of a request, at places o .. o + m of a block,
// head `head` of K (side 0) or V (side 1).  `tile` is 16 * kDim bytes of LDS.
template <int kType, int kDim>
__device__ __forceinline__ void write_run(const Append &a, int t, int m, int o, int slot, int head,
                                          int side, char *tile) {
  constexpr int kUnits = kDim / 16, kTokens = 64 / kUnits, kPasses = 16 / kTokens;
  const int lane = lane_id(), u = lane % kUnits, tl = lane / kUnits;
  const Rows &rows = side ? a.v : a.k;
  const int bt = 1 << a.kv.block_shift;
  char *chunk = const_cast<char *>(a.kv.base) + side * a.kv.kv_stride + slot * a.kv.slot_stride;
  char *codes = chunk + (int64_t)head * bt * kDim;
  float *scale_at = reinterpret_cast<float *>(chunk + (int64_t)a.kv.kv_heads * bt * kDim) + head;
  const float old_scale = o > 0 ? *scale_at : 0.f;
  Rope rope = a.rope;
  if (side) rope.dim = 0;
  int da, db;
  unit_dims(rope, u, da, db);

  float x[kPasses][8], y[kPasses][8];
  bool bad = false;
  // the run's tokens in sub-block s, zeros in other places
  auto load = [&](int s) {
#pragma unroll
    for (int p = 0; p < kPasses; ++p) {
      const int j = 16 * s + p * kTokens + tl - o;
      const bool in = j >= 0 && j < m;
      const int at = t + (in ? j : 0);
      widen<kType>(load_row(rows, at, head, da), x[p]);
      widen<kType>(load_row(rows, at, head, db), y[p]);
      if (rope.dim) rotate_unit(rope, u, rope.positions[at], x[p], y[p]);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const bool fx = __builtin_isfinite(x[p][i]), fy = __builtin_isfinite(y[p][i]);
        bad |= in && !(fx && fy);
        x[p][i] = in && fx ? x[p][i] : 0.f;
        y[p][i] = in && fy ? y[p][i] : 0.f;
      }
    }
  };
  const int s0 = o >> 4, s1 = (o + m - 1) >> 4;
  float amax = 0.f;
  for (int s = s0; s <= s1; ++s) {
    load(s);
#pragma unroll
    for (int p = 0; p < kPasses; ++p)
#pragma unroll
      for (int i = 0; i < 8; ++i) amax = codes_max(codes_max(amax, x[p][i]), y[p][i]);
  }
#pragma unroll
  for (int d = 32; d; d >>= 1) amax = fmaxf(amax, __shfl_xor(amax, d));
  if (__any(bad)) {
    if (lane == 0) kv_report(a.status);
  }
  const float scale = fmaxf(old_scale, power_of_two(scale_exponent(amax)));
  const float inverse = 1.f / scale;  // exact: a power of two
  const bool grew = o > 0 && scale > old_scale;
  const float ratio = old_scale * inverse;
  for (int s = grew ? 0 : s0; s <= s1; ++s) {
    u4 *place = reinterpret_cast<u4 *>(codes + s * 16 * kDim) + lane;
    // the 16 bytes of a lane: a token's 16 dims of K, 4 tokens' 4 dims of V
    const int a0 = 16 * s + (side ? lane / 16 * 4 : lane / 4), a1 = a0 + (side ? 4 : 1);
    const bool has_new = a1 > o && a0 < o + m, all_new = a0 >= o && a1 <= o + m;
    const bool rescale = grew && a0 < o, store = has_new || rescale;
    if (store && !all_new) {
      // bytes of older tokens, among those that stay
      const unsigned older = a1 <= o ? ~0u : a0 < o ? (1u << 8 * (o - a0)) - 1 : 0u;
#pragma unroll
      for (int c = 0; c < kDim / 64; ++c) {
        u4 w = place[64 * c];
        if (rescale) {
#pragma unroll
          for (int i = 0; i < 4; ++i) w[i] = (rescale4(w[i], ratio) & older) | (w[i] & ~older);
        }
        reinterpret_cast<u4 *>(tile)[64 * c + lane] = w;
      }
    }
    if (s >= s0) {
      if (s1 > s0) load(s);
      wave_sync();
#pragma unroll
      for (int p = 0; p < kPasses; ++p) {
        const int tok = p * kTokens + tl, j = 16 * s + tok - o;
        if (j < 0 || j >= m) continue;
        unsigned w[4];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          w[i] = codes4(x[p][4 * i] * inverse, x[p][4 * i + 1] * inverse, x[p][4 * i + 2] * inverse,
                        x[p][4 * i + 3] * inverse);
          w[2 + i] = codes4(y[p][4 * i] * inverse, y[p][4 * i + 1] * inverse,
                            y[p][4 * i + 2] * inverse, y[p][4 * i + 3] * inverse);
        }
        if (!side) {
          unsigned *ka = reinterpret_cast<unsigned *>(tile + ((da >> 6) * 16 + tok) * 64 + (da & 63));
          unsigned *kb = reinterpret_cast<unsigned *>(tile + ((db >> 6) * 16 + tok) * 64 + (db & 63));
          ka[0] = w[0];
          ka[1] = w[1];
          kb[0] = w[2];
          kb[1] = w[3];
        } else {
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const int d = (i < 8 ? da : db) + (i & 7);
            tile[(((d >> 6) * 4 + tok / 4) * 16 + (d & 15)) * 16 + ((d & 63) >> 4) * 4 + tok % 4] =
                (char)(w[i >> 2] >> (8 * (i & 3)));
          }
        }
      }
    }
    wave_sync();
#pragma unroll
    for (int c = 0; c < kDim / 64; ++c)
      if (store) place[64 * c] = reinterpret_cast<u4 *>(tile)[64 * c + lane];
    wave_sync();
  }
  if (lane == 0 && (o == 0 || grew)) *scale_at = scale;
}

__device__ __forceinline__ bool writable(const KvRequest &r) { return r.ok && r.len >= r.count; }

template <int kType, int kDim>
__global__ __launch_bounds__(kBlock) void append_kernel(Append a) {
  if ((int)blockIdx.x < a.q_blocks) {
    rotate_queries<kType, kDim>(a);
    return;
  }
  if (blockIdx.x == gridDim.x - 1) {
    // the others meet only requests with new tokens
    for (int i = threadIdx.x; i < a.batch.n; i += kBlock)
      if (!writable(kv_request(a.batch, a.row_offsets, a.kv.block_shift, i))) kv_report(a.status);
    return;
  }
  __shared__ __align__(16) char tiles[kWaves][16 * kDim];
  __shared__ unsigned sums[kWaves];
  const int sides = 2 * a.kv.kv_heads, parts = (sides + kWaves - 1) / kWaves;
  const int w = (int)blockIdx.x - a.q_blocks;
  const int t0 = w / parts * a.group, t1 = min(t0 + a.group, a.batch.n_tokens);
  // the request of token t0: how many end at or before it
  unsigned ended[1] = {0};
  for (int i = threadIdx.x; i < a.batch.n; i += kBlock) ended[0] += a.batch.token_offsets[i + 1] <= t0;
  block_sum<1, unsigned>(ended, sums);
  const int unit = w % parts * kWaves + wave_id();
  if (unit >= sides) return;
  const int head = unit >> 1, side = unit & 1;
  const int bt = 1 << a.kv.block_shift;
  for (int i = (int)ended[0], t = t0; t < t1 && i < a.batch.n; ++i) {
    const KvRequest r = kv_request(a.batch, a.row_offsets, a.kv.block_shift, i);
    if (!writable(r)) continue;
    t = max(t, r.first);
    while (t < t1 && t < r.first + r.count) {
      const int at = r.len - r.count + (t - r.first);  // cache index
      const int o = at & (bt - 1);
      const int m = min(bt - o, r.first + r.count - t);
      if (t == r.first || o == 0) {  // otherwise the run began in an earlier group
        const int slot = a.slots[r.row + (at >> a.kv.block_shift)];
        bool fine = slot >= 0 && slot < a.kv.num_slots;
        if (a.rope.dim)
          for (int j = lane_id(); j < m; j += 64) fine &= a.rope.positions[t + j] >= 0;
        if (__all(fine))
          write_run<kType, kDim>(a, t, m, o, slot, head, side, tiles[wave_id()]);
        else
          kv_report(a.status);
      }
      t += m;
    }
  }
}

Rows rows_of(const cascade_rows_t *r) {
  return r ? Rows{static_cast<char *>(r->data), 2 * r->token_stride, 2 * r->head_stride}
           : Rows{nullptr, 0, 0};
}

template <int kType>
void launch(const Append &a, int blocks, int dim, hipStream_t stream) {
  auto kernel = dim == 64    ? append_kernel<kType, 64>
                : dim == 128 ? append_kernel<kType, 128>
                             : append_kernel<kType, 256>;
  hipLaunchKernelGGL(kernel, dim3(blocks), dim3(kBlock), 0, stream, a);
}

}  // namespace
}  // namespace cascade

using namespace cascade;

extern "C" size_t cascade_kv_chunk_bytes(const cascade_kv_format_t *format) {
  return kv_format_ok(format) ? (size_t)kv_chunk_bytes(format) : 0;
}

extern "C" int cascade_kv_append(const cascade_kv_pool_t *pool, int32_t layer,
                                 const cascade_kv_format_t *format,
                                 const cascade_kv_batch_t *batch,
                                 const cascade_block_table_t *table, int32_t dtype,
                                 int32_t q_heads, const cascade_rows_t *q,
                                 const cascade_rows_t *q_out, const cascade_rows_t *k,
                                 const cascade_rows_t *v, const cascade_rope_t *rope,
                                 const int32_t *positions, int32_t *status_dev, void *stream) {
  if (!kv_pool_ok(pool, layer, format) || !kv_batch_ok(batch, table)) return CASCADE_EINVAL;
  if (dtype != CASCADE_BF16 && dtype != CASCADE_F16) return CASCADE_EINVAL;
  if (!q != !q_out || (q && (q_heads < 1 || q_heads > 128 * format->kv_heads)))
    return CASCADE_EINVAL;
  if (rope && (rope->rotary_dim < 0 || rope->rotary_dim > format->head_dim ||
               rope->rotary_dim % 16 || !std::isfinite(rope->scale) ||
               (rope->rotary_dim > 0 && (!rope->freq || !positions))))
    return CASCADE_EINVAL;
  if (batch->n_tokens == 0 || batch->n == 0) return CASCADE_OK;
  if (!kv_rows_ok(k) || !kv_rows_ok(v) || (q && (!kv_rows_ok(q) || !kv_rows_ok(q_out))))
    return CASCADE_EINVAL;
  Append a;
  a.kv = kv_view(pool, layer, format);
  a.batch = *batch;
  a.row_offsets = table->row_offsets;
  a.slots = table->slots;
  a.q = rows_of(q);
  a.q_out = rows_of(q_out);
  a.k = rows_of(k);
  a.v = rows_of(v);
  a.rope = Rope{nullptr, nullptr, 0, 0, 1.f};
  if (rope && rope->rotary_dim > 0)
    a.rope = Rope{rope->freq, positions, rope->rotary_dim, rope->interleaved != 0, rope->scale};
  a.q_heads = q_heads;
  a.status = status_dev;
  const int64_t units = q ? (int64_t)batch->n_tokens * q_heads * (format->head_dim / 16) : 0;
  // A wave takes the runs that begin in a group's tokens one after another, and a
  // workgroup looks at its group's request first.  So groups are small where runs
  // are short, or few in all.  Groups of 1, 4 and 16 tokens take, in us, for
  //   single tokens, 64 query heads: 128 of them 7.0, 15.5, 50.6; 512 18, 22, 58;
  //     640 23, 26, 63; 1024 36, 31, 77; 2048 70, 58, 91
  //   chunks of 512 tokens: one 13.4, 7.6, 7.2; 16 130, 59, 44
  //   of 16: 4 of them 6.1, 5.9, 8.5; 32 13.5, 10.6, 10.0; 100 35, 23, 16
  //   of 12: 16 of them 7.1, 9.0, 12.1; 128 30, 18, 19
  const bool few = batch->n_tokens <= 512, runs = batch->n_tokens >= 16ll * batch->n;
  a.group = few ? (runs ? 4 : 1) : (runs ? 16 : 4);
  const int64_t q_blocks = (units + kBlock - 1) / kBlock;
  const int64_t kv_blocks = (int64_t)((batch->n_tokens + a.group - 1) / a.group) *
                            ((2 * format->kv_heads + kWaves - 1) / kWaves);
  const int64_t blocks = q_blocks + kv_blocks + 1;  // the last one checks the batch
  if (blocks > INT32_MAX / kBlock) return CASCADE_EINVAL;
  a.q_blocks = (int)q_blocks;
  const auto s = static_cast<hipStream_t>(stream);
  if (dtype == CASCADE_BF16)
    launch<CASCADE_BF16>(a, (int)blocks, format->head_dim, s);
  else
    launch<CASCADE_F16>(a, (int)blocks, format->head_dim, s);
  return hipGetLastError() == hipSuccess ? CASCADE_OK : CASCADE_EHIP;
}

extern "C" int cascade_rope_frequencies(const cascade_rope_spec_t *spec, uint64_t *freq,
                                        float *scale) {
  if (!spec || !freq || !scale) return CASCADE_EINVAL;
  const int R = spec->rotary_dim;
  if (R < 16 || R > 256 || R % 16 || spec->kind < CASCADE_ROPE_PLAIN ||
      spec->kind > CASCADE_ROPE_RAMP)
    return CASCADE_EINVAL;
  const double f = spec->factor, len = spec->original_len, pi = 3.14159265358979323846;
  if (!(spec->base > 1 && std::isfinite(spec->base)) || !(f >= 1 && std::isfinite(f)))
    return CASCADE_EINVAL;
  if (spec->kind >= CASCADE_ROPE_BANDS &&
      (!(len >= 1 && std::isfinite(len)) || !(spec->low > 0 && spec->high > spec->low) ||
       !std::isfinite(spec->high)))
    return CASCADE_EINVAL;
  const double base =
      spec->kind == CASCADE_ROPE_BASE ? spec->base * std::pow(f, R / (R - 2.0)) : spec->base;
  const auto pair = [&](double turns) {
    return R * std::log(len / (2 * pi * turns)) / (2 * std::log(base));
  };
  double from = 0, to = 0;
  if (spec->kind == CASCADE_ROPE_RAMP) {
    from = std::fmax(std::floor(pair(spec->high)), 0);
    to = std::fmin(std::ceil(pair(spec->low)), R - 1);
    if (to <= from) to = from + 0.001;
  }
  *scale = spec->kind == CASCADE_ROPE_RAMP ? (float)(0.1 * std::log(f) + 1) : 1.f;
  for (int j = 0; j < R / 2; ++j) {
    double theta = std::pow(base, -2.0 * j / R), kept = 1;  // share of the unstretched angle
    if (spec->kind == CASCADE_ROPE_LINEAR) kept = 0;
    if (spec->kind == CASCADE_ROPE_BANDS)
      kept = (len * theta / (2 * pi) - spec->low) / (spec->high - spec->low);
    if (spec->kind == CASCADE_ROPE_RAMP) kept = 1 - (j - from) / (to - from);
    kept = std::fmin(std::fmax(kept, 0), 1);
    theta *= kept + (1 - kept) / f;
    freq[j] = (uint64_t)std::ldexp(theta / (2 * pi), 64);  // under 1/6 of a turn
  }
  return CASCADE_OK;
}
