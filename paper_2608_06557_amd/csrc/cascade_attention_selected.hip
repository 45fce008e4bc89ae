// cascade_attention_selected.hip -- attention of a batch's new tokens over
// blocks that were selected for each token and KV head, on gfx950.
//
// The listed blocks' tokens, one behind the other, are a short cache of the
// token's own: place c is token c % block_tokens of the list's block c /
// block_tokens.  Blocks ascend, so only the last can hold tokens that the row does
// not see, and they are at the end.  The products are those of attention_tiles.h
// for few rows: 4 waves take 32 tokens each in turn and join in LDS.
//
// A workgroup has one token, KV head, row set and part of the list; the parts
// of one token are joined by a second launch.  It looks its slots up once,
// into LDS, and the loads of codes run a step ahead.
//
// 128 single tokens with lists of 128 blocks of 16 tokens, 64/8 heads of 128 dims, are bound by
// HBM: 104-106 us, 601 MB fetched (543 without what lines bring along), 5.7 TB/s.  512 tokens of
// one request, 64 blocks each, find codes in L2: 60 us for 1.07 GB in close succession (66 to 70 after a
// pause, before the clock has risen), of which 5.5 us for each of its rounds of workgroups go to
// slots, first loads and the join of waves.  One token: 6.6 us, join 4.2.
#include "attention_tiles.h"

namespace cascade {
namespace {

struct Selected : Attention {
  const int32_t *selected;  // [n_tokens][KV heads][places]
  int places;       // of a list
  int splits, per;  // parts of a list, and blocks of one
  int row_tiles;    // row sets of a KV head's query heads
};

constexpr int kMostListed = 4096;  // blocks of a part: their slots are in LDS

// Up to 8 query heads fill half of a product's 16 columns.  kHalves = 2 gives the
// other half to the second 16 tokens of a step: K_0 Q_0 + K_1 Q_1, where Q_0 has the
// heads in the first 8 columns and zeros in the others and Q_1 in the last 8, holds
// the scores of both in one operand's place, so the softmax has half the work.  A
// column's weights belong to its 16 tokens; each half keeps an m, a sum and an O of its
// own, and they are joined like those of two waves.
template <int kType, int kDim, Cap kCap>
struct Halves : Rowset<kType, kDim, 1, kCap> {
  typedef Rowset<kType, kDim, 1, kCap> Base;
  typedef typename El<kType>::v8 v8;
  // Weights of tokens key .. key + 32, the lane's half of them.
  __device__ __forceinline__ void weights(const Attention &a, f4 &s, v8 (&p)[1][1], int key, bool masked) {
    const int lane = lane_id(), half = lane >> 3 & 1;
    if (kCap != Cap::kNone) {
#pragma unroll
      for (int i = 0; i < 4; ++i) s[i] = capped<kCap>(s[i], a.cap_in, a.cap_y, a.qk, a.cap);
    }
    if (masked) {
      const int seen = this->limit[0] - key - 16 * half - 4 * (lane >> 4);
#pragma unroll
      for (int i = 0; i < 4; ++i) s[i] = i <= seen ? s[i] : -__builtin_inff();
    }
    float &m = this->m[0], &sum = this->sum[0], &used = this->used[0];
    float top = fmaxf(fmaxf(s[0], s[1]), fmaxf(s[2], s[3])) * a.scale;
    if (__any(top > m + kSlack)) {
      top = fmaxf(top, __shfl_xor(top, 16));
      top = fmaxf(top, __shfl_xor(top, 32));
      const float now = fmaxf(m, top), f = __builtin_amdgcn_exp2f(m - now);
      m = now;
      sum *= f;
      used *= f;
      this->scale_o(f);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) s[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i], a.scale, -m));
    sum += (s[0] + s[1]) + (s[2] + s[3]);
    const unsigned w0 = narrow2<kType>(s[0], s[1]), w1 = narrow2<kType>(s[2], s[3]);
    used = El<kType>::add2(w1, El<kType>::add2(w0, used));
    p[0][0] = __builtin_bit_cast(v8, u4{half ? 0 : w0, half ? 0 : w1, half ? w0 : 0, half ? w1 : 0});
  }
};

template <int kType, int kDim, int kTiles, Cap kCap, int kHalves = 1>
__global__ __launch_bounds__(kBlock, waves_per_simd(kDim, kTiles)) void selected_kernel(Selected a) {
  static_assert(kHalves == 1 || kTiles == 1, "half a row set");
  constexpr int kRows = 16 * kTiles / kHalves;
  constexpr int kPart = kDim < 128 ? kDim : 128;  // dims that one combination takes
  constexpr int kPitch = kPart + 4;
  typedef typename El<kType>::v8 v8;
  if (blockIdx.x == gridDim.x - 1) {
    if (blockIdx.y == 0) check_requests(a.batch, a.row_offsets, a.kv.block_shift, a.status);
    return;
  }
  extern __shared__ __align__(16) char lds[];
  __shared__ int owners[kWaves], ends[kWaves];
  int *const slot_list = reinterpret_cast<int *>(lds);
  float *const ms = reinterpret_cast<float *>(lds + (4 * a.per + 15 & ~15)), *const os = ms + 2 * kWaves * 16;
  char *const qs = reinterpret_cast<char *>(os);
  static_assert(16 * kTiles * kHalves * kDim * 2 <= 4 * kWaves * 16 * kPitch, "q fits the place of O");
  const int lane = lane_id(), g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(wave_id());
  const int kv_heads = a.kv.kv_heads;
  const int token = blockIdx.x / kv_heads, head = blockIdx.x % kv_heads;
  const int tile = blockIdx.y % a.row_tiles, split = blockIdx.y / a.row_tiles;

  // the part's first blocks, while the request is looked for
  const int32_t *const list = a.selected + ((int64_t)token * kv_heads + head) * a.places;
  const int k0 = split * a.per, k1 = min(k0 + a.per, a.places);
  int k = k0 + threadIdx.x;
  int block = k < k1 ? list[k] : -1, before = k > 0 && k < k1 ? list[k - 1] : 0;
  // single tokens are their requests' numbers, and one request has them all: look there first
  KvRequest req = kv_request<true>(a.batch, a.row_offsets, a.kv.block_shift, min(token, a.batch.n - 1));
  if (!req.ok || token < req.first || token - req.first >= req.count) {
    const int id = __builtin_amdgcn_readfirstlane(owner_of(a.batch.token_offsets, a.batch.n, token, owners));
    if (id >= a.batch.n) return;
    req = kv_request<true>(a.batch, a.row_offsets, a.kv.block_shift, id);
    if (!req.ok || token < req.first || token - req.first >= req.count) return;
  }
  const int last = __builtin_amdgcn_readfirstlane(req.len - req.count + token - req.first);  // cached token
  const int own = last < 0 ? -1 : last >> a.kv.block_shift, bt = 1 << a.kv.block_shift;

  // the part's slots, up to the list's end
  int end = k1 - k0;
  bool bad = false, partial = false;
  while (k < k1) {
    if (block < 0) {
      end = min(end, k - k0);
    } else if (block > own || (k > 0 && (before < 0 || before >= block))) {
      bad = true;  // not seen, behind the end or not in order
      slot_list[k - k0] = 0;
    } else {
      partial |= block == own;
      slot_list[k - k0] = a.slots[req.row + block];
    }
    k += kBlock;
    if (k < k1) block = list[k], before = list[k - 1];
  }
  __syncthreads();
#pragma unroll
  for (int m = 32; m; m >>= 1) end = min(end, __shfl_xor(end, m));
  // the last block of the part is the token's own, of which it sees a part
  const bool mine = __any(partial);
  if (lane == 0) ends[wave] = 2 * end + mine;
  __syncthreads();
  int listed = INT32_MAX, ended_own = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) listed = min(listed, ends[w] >> 1), ended_own |= ends[w] & 1;
  listed = __builtin_amdgcn_readfirstlane(listed);
  const int length = __builtin_amdgcn_readfirstlane((listed << a.kv.block_shift) -
                                                    (ended_own && listed ? bt - 1 - (last & (bt - 1)) : 0));
  if (__any(bad)) kv_report(a.status);

  typename std::conditional<kHalves == 2, Halves<kType, kDim, kCap>, Rowset<kType, kDim, kTiles, kCap>>::type r;
  const int first_row = tile * kRows;
#pragma unroll
  for (int t = 0; t < kTiles; ++t) {
    r.limit[t] = first_row + 16 * t + (lane & (16 / kHalves - 1)) < a.group ? length - 1 : -1;
    r.log_at[t] = -1;
  }
  r.clear();
  if (length > 0) {
    // as in attention_kernel
    const Cache<kDim> cache(a, req, head, length);
    constexpr int kStride = 32 * kWaves;
    int key = __builtin_amdgcn_readfirstlane(32 * wave);
    Codes<kDim> c;
    int slot[2];
    auto look = [&](int key) {
      slot[0] = __builtin_amdgcn_readfirstlane(slot_list[cache.entry(key >> 4)]);
      slot[1] = __builtin_amdgcn_readfirstlane(slot_list[cache.entry((key >> 4) + 1)]);
    };
    look(key);
    constexpr int kQs = kTiles * kHalves * (kDim / 32), kMine = (kQs + kWaves - 1) / kWaves;
    u4 q[kMine];
#pragma unroll
    for (int i = 0; i < kMine; ++i) {
      const int e = min(i * kWaves + wave, kQs - 1), d = e % (kDim / 32), set = e / (kDim / 32);
      const int row = first_row + (kHalves == 2 ? lane & 7 : set * 16 + (lane & 15));
      const bool valid = row < a.group && (kHalves == 1 || (lane >> 3 & 1) == set);
      q[i] = *reinterpret_cast<const u4 *>(a.q.data + (int64_t)token * a.q.token_stride +
                                           (int64_t)(head * a.group + (valid ? row : 0)) * a.q.head_stride + 32 * g +
                                           128 * (d >> 1) + 16 * (d & 1));
      q[i] = valid ? (q[i] & a.keep) ^ a.flip : u4{0, 0, 0, 0};
    }
    __builtin_amdgcn_sched_barrier(0);
    c.fetch_k(cache, slot, key);
    __builtin_amdgcn_sched_barrier(0);
    c.fetch_v(cache, slot, key);
    __builtin_amdgcn_sched_barrier(0);
    look(key + kStride);
#pragma unroll
    for (int i = 0; i < kMine; ++i)
      *reinterpret_cast<u4 *>(qs + (min(i * kWaves + wave, kQs - 1) * 64 + lane) * 16) = q[i];
    __syncthreads();
    if (key < length) {
      while (true) {
        if (key + 32 > length) {
          const unsigned live[2] = {live_bytes(key + 4 * g, length), live_bytes(key + 16 + 4 * g, length)};
#pragma unroll
          for (int i = 0; i < kDim / 64; ++i)
#pragma unroll
            for (int b = 0; b < 2; ++b) {
              c.v[b][i] &= live[b];
              // a score of one half adds the other's key, times 0
              if (kHalves == 2 && key + 16 * b + (lane & 15) >= length) c.k[b][i] = u4{0, 0, 0, 0};
            }
        }
        int q_at = lane * 16;
        asm volatile("" : "+v"(q_at));  // or the loads of q move out of the loop, into registers
        const Units<kType> ku(c.ks);
        auto k_of = [&](int b, int d) {
          const u4 w = c.k[b][d >> 1];
          return widen8<kType>(w[2 * (d & 1)], w[2 * (d & 1) + 1], ku.scale[b], ku.scale[b]);
        };
        auto q_of = [&](int t, int d) {
          return *reinterpret_cast<const v8 *>(qs + (t * (kDim / 32) + d) * 1024 + q_at);
        };
        v8 p[kTiles][1];
        if constexpr (kHalves == 2) {
          f4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int d = 0; d < kDim / 32; ++d)
#pragma unroll
            for (int b = 0; b < 2; ++b) x = El<kType>::mfma(k_of(b, d), q_of(b, d), x);
          if (__builtin_expect(ku.odd, false)) x *= lane & 8 ? ku.rest[1] : ku.rest[0];
          c.fetch_k(cache, slot, key + kStride);
          r.weights(a, x, p, key, key + 32 > length);
        } else {
          f4 x[kTiles][2];
          r.template scores<2>(k_of, q_of, x);
          if (__builtin_expect(ku.odd, false)) {
#pragma unroll
            for (int t = 0; t < kTiles; ++t)
#pragma unroll
              for (int b = 0; b < 2; ++b) x[t][b] *= ku.rest[b];
          }
          c.fetch_k(cache, slot, key + kStride);
          r.template weights<2>(a, x, p, key, length, key + 32 > length, nullptr);
        }
        const Units<kType> vu(c.vs);
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
          r.add([&](int d) { return widen8<kType>(c.v[0][d >> 2][d & 3], c.v[1][d >> 2][d & 3], s0, s1); }, part);
          if (__builtin_expect(!vu.odd, true)) break;
          r.scale_o(unit_of(vu.rest[b]));
          if (b) break;
        }
        c.fetch_v(cache, slot, key + kStride);
        look(key + 2 * kStride);
        key += kStride;
        if (key >= length) break;
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
#pragma unroll
  for (int t = 0; t < kTiles; ++t) {
    if (g == 0) {
      ms[(wave * 16 + lane) * 2] = r.m[t];
      ms[(wave * 16 + lane) * 2 + 1] = r.sum[t];
    }
    __syncthreads();
    // of a row: the waves', and their halves'
    constexpr int kJoined = kWaves * kHalves, kApart = 16 / kHalves;
    float top = kLowest;
#pragma unroll
    for (int k = 0; k < kJoined; ++k) top = fmaxf(top, ms[(k * kApart + lane % kApart) * 2]);
    const float f = __builtin_amdgcn_exp2f(r.m[t] - top) * evened(r.sum[t], r.used[t]);
#pragma unroll
    for (int d0 = 0; d0 < kDim; d0 += kPart) {
#pragma unroll
      for (int d = d0 / 16; d < (d0 + kPart) / 16; ++d)
        *reinterpret_cast<f4 *>(os + (wave * 16 + (lane & 15)) * kPitch + 16 * d - d0 + 4 * g) = r.o[t][d] * f;
      __syncthreads();
      for (int j = threadIdx.x; j < kApart * kPart / 4; j += kBlock) {
        const int n = j / (kPart / 4), d = j % (kPart / 4) * 4, row = first_row + 16 * t + n;
        if (row >= a.group) continue;
        f4 o = {0.f, 0.f, 0.f, 0.f};
        float m = kLowest, sum = 0.f;
#pragma unroll
        for (int k = 0; k < kJoined; ++k) {
          o += *reinterpret_cast<const f4 *>(os + (k * kApart + n) * kPitch + d);
          m = fmaxf(m, ms[(k * kApart + n) * 2]);
        }
#pragma unroll
        for (int k = 0; k < kJoined; ++k)
          sum += ms[(k * kApart + n) * 2 + 1] * __builtin_amdgcn_exp2f(ms[(k * kApart + n) * 2] - m);
        const int h = head * a.group + row;
        const int64_t at = (int64_t)token * a.q_heads + h;
        if (a.splits == 1) {
          const float inv = sum > 0.f ? 1.f / sum : sum == 0.f ? 0.f : sum;
          const u2 x = {narrow2<kType>(o[0] * inv, o[1] * inv), narrow2<kType>(o[2] * inv, o[3] * inv)};
          *reinterpret_cast<u2 *>(a.out.data + (int64_t)token * a.out.token_stride + (int64_t)h * a.out.head_stride +
                                  2 * (d0 + d)) = x;
          if (a.lse && d0 + d == 0) a.lse[at] = (m + __builtin_amdgcn_logf(sum)) * kLn2;
        } else {
          const int64_t to = at * a.splits + split;
          *reinterpret_cast<f4 *>(a.parts + to * kDim + d0 + d) = o;
          if (d0 + d == 0) *reinterpret_cast<f2 *>(a.part_sums + 2 * to) = f2{m, sum};
        }
      }
      __syncthreads();
    }
  }
}

// Joins the parts of each row: a row to a wave.
template <int kType, int kDim>
__global__ __launch_bounds__(kBlock) void join_selected_kernel(Selected a) {
  constexpr int kLanes = kDim / 4, kParts = 64 / kLanes;
  __shared__ int owners[kWaves];
  const int lane = lane_id();
  const int64_t row0 = (int64_t)blockIdx.x * kWaves, row = row0 + wave_id();
  const int token = (int)(row / a.q_heads), head = (int)(row % a.q_heads);
  // rows of no request stay as they are
  int id = __builtin_amdgcn_readfirstlane(
      owner_of(a.batch.token_offsets, a.batch.n, (int)(row0 / a.q_heads), owners));
  const int mine = __builtin_amdgcn_readfirstlane(token);
  while (id < a.batch.n && a.batch.token_offsets[id + 1] <= mine) ++id;
  if (id >= a.batch.n || mine >= a.batch.n_tokens) return;
  const KvRequest req = kv_request(a.batch, a.row_offsets, a.kv.block_shift, id);
  if (!req.ok || mine < req.first || mine - req.first >= req.count) return;
  const float *const part_sums = a.part_sums + 2 * row * a.splits;
  float top = kLowest;
  for (int p = lane; p < a.splits; p += 64) top = fmaxf(top, part_sums[2 * p]);
#pragma unroll
  for (int d = 32; d; d >>= 1) top = fmaxf(top, __shfl_xor(top, d));
  float sum = 0.f;
  for (int p = lane; p < a.splits; p += 64) sum += part_sums[2 * p + 1] * __builtin_amdgcn_exp2f(part_sums[2 * p] - top);
#pragma unroll
  for (int d = 32; d; d >>= 1) sum += __shfl_xor(sum, d);
  f4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
  for (int p = lane / kLanes; p < a.splits; p += kParts)
    o += *reinterpret_cast<const f4 *>(a.parts + (row * a.splits + p) * kDim + 4 * (lane % kLanes)) *
         __builtin_amdgcn_exp2f(part_sums[2 * p] - top);
#pragma unroll
  for (int d = 32; d >= kLanes; d >>= 1)
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] += __shfl_xor(o[i], d);
  if (lane < kLanes) {
    const float f = sum > 0.f ? 1.f / sum : sum == 0.f ? 0.f : sum;
    const u2 x = {narrow2<kType>(o[0] * f, o[1] * f), narrow2<kType>(o[2] * f, o[3] * f)};
    *reinterpret_cast<u2 *>(a.out.data + (int64_t)mine * a.out.token_stride + (int64_t)head * a.out.head_stride +
                            8 * lane) = x;
  }
  if (a.lse && lane == 0) a.lse[row] = (top + __builtin_amdgcn_logf(sum)) * kLn2;
}

// ------------------------------------------------------------------- host

// How a list is divided: into as many parts as fill the GPU, of 256 tokens at least.  That pays
// from 2 Ki listed tokens on: one token of 32/8 heads of 128 dims over 512, 1 Ki and 2 Ki 11.3, 11.2 and
// 11.2 us, in parts of 1 Ki at least 7.7, 9.8 and 14.0; 8 tokens 11.5, 13.1 and 16.6 against 8.2, 12.1
// and 16.8; 32 tokens 15.7, 21.2 and 31.8 against 11.1, 16.1 and 31.6.
struct Parts {
  int tiles, row_tiles, splits, per;
  size_t parts, sums, total;
  Parts(const cascade_kv_format_t *f, const cascade_kv_batch_t *b, int q_heads, int keep) {
    const int group = q_heads / f->kv_heads;
    tiles = group > 16 ? 2 : 1;
    row_tiles = (group + 16 * tiles - 1) / (16 * tiles);
    const int64_t work = std::max<int64_t>((int64_t)b->n_tokens * f->kv_heads * row_tiles, 1);
    const int64_t room = kCUs * waves_per_simd(f->head_dim, tiles);
    const int64_t useful = ((int64_t)keep * f->block_tokens + 255) / 256;
    int64_t n = std::max<int64_t>(std::min(useful, room / work), 1);
    n = std::max<int64_t>(n, (keep + kMostListed - 1) / kMostListed);
    per = (int)((keep + n - 1) / n);
    splits = (keep + per - 1) / per;
    // the same for every batch, so that one made for any serves all, but for longer lists
    const size_t forced = (keep + kMostListed - 1) / kMostListed;
    const size_t rows = std::max<size_t>(room * 16 * tiles, forced > 1 ? (size_t)b->n_tokens * q_heads * splits : 0);
    parts = 0;
    sums = aligned(sizeof(float) * rows * f->head_dim);
    total = sums + aligned(sizeof(float) * rows * 2) + 256;
  }
};

template <int kType, int kDim, int kTiles, int kHalves = 1>
void start(const Selected &a, Cap cap, hipStream_t stream) {
  const size_t lds = (4 * a.per + 15 & ~15) + sizeof(float) * kWaves * 16 * (2 + (kDim < 128 ? kDim : 128) + 4);
  auto kernel = cap == Cap::kWide     ? selected_kernel<kType, kDim, kTiles, Cap::kWide, kHalves>
                : cap == Cap::kNarrow ? selected_kernel<kType, kDim, kTiles, Cap::kNarrow, kHalves>
                                      : selected_kernel<kType, kDim, kTiles, Cap::kNone, kHalves>;
  const dim3 grid(a.batch.n_tokens * a.kv.kv_heads + 1, a.splits * a.row_tiles);  // the last one checks the batch
  hipLaunchKernelGGL(kernel, grid, dim3(kBlock), lds, stream, a);
  if (a.splits > 1) {
    const int64_t rows = (int64_t)a.batch.n_tokens * a.q_heads;
    hipLaunchKernelGGL((join_selected_kernel<kType, kDim>), dim3((unsigned)((rows + kWaves - 1) / kWaves)),
                       dim3(kBlock), 0, stream, a);
  }
}

template <int kType, int kDim>
void start(const Selected &a, const Parts &p, Cap cap, hipStream_t stream) {
  a.group <= 8 ? start<kType, kDim, 1, 2>(a, cap, stream)
  : p.tiles == 1 ? start<kType, kDim, 1>(a, cap, stream)
                 : start<kType, kDim, 2>(a, cap, stream);
}

template <int kType>
int start(const Selected &a, const Parts &p, Cap cap, hipStream_t s) {
  switch (a.kv.head_dim) {
    case 64: start<kType, 64>(a, p, cap, s); break;
    case 128: start<kType, 128>(a, p, cap, s); break;
    default: start<kType, 256>(a, p, cap, s);
  }
  return hipGetLastError() == hipSuccess ? CASCADE_OK : CASCADE_EHIP;
}

bool keep_ok(int keep) { return keep >= 1 && keep <= 65536; }

}  // namespace
}  // namespace cascade

using namespace cascade;

extern "C" size_t cascade_attention_selected_workspace_bytes(const cascade_kv_format_t *format,
                                                             const cascade_kv_batch_t *batch, int32_t q_heads,
                                                             int32_t keep) {
  if (!kv_format_ok(format) || !batch || batch->n_tokens < 0 || !heads_ok(format, q_heads) || !keep_ok(keep)) return 0;
  return Parts(format, batch, q_heads, keep).total;
}

extern "C" int cascade_attention_selected(const cascade_kv_pool_t *pool, int32_t layer,
                                          const cascade_kv_format_t *format, const cascade_kv_batch_t *batch,
                                          const cascade_block_table_t *table, const cascade_attention_t *args,
                                          const int32_t *selected, int32_t keep, void *workspace,
                                          size_t workspace_bytes, int32_t *status_dev, void *stream) {
  if (!kv_pool_ok(pool, layer, format) || !kv_batch_ok(batch, table) || !attention_ok(args, format) || !keep_ok(keep))
    return CASCADE_EINVAL;
  if (args->block_weight || args->weight_window) return CASCADE_EINVAL;
  if (!workspace || ((uintptr_t)workspace & 255)) return CASCADE_EINVAL;
  const Parts p(format, batch, args->q_heads, keep);
  if (workspace_bytes < p.total) return CASCADE_ENOSPC;
  if (batch->n == 0 || batch->n_tokens == 0 || batch->max_new == 0) return CASCADE_OK;
  if (!kv_rows_ok(&args->q) || !kv_rows_ok(&args->out) || !selected) return CASCADE_EINVAL;
  if ((int64_t)batch->n_tokens * args->q_heads > INT32_MAX / kBlock) return CASCADE_EINVAL;
  Cap cap;
  Selected a;
  static_cast<Attention &>(a) = attention_of(pool, layer, format, batch, table, args, status_dev, cap);
  a.selected = selected;
  a.places = keep;
  a.splits = p.splits;
  a.per = p.per;
  a.row_tiles = p.row_tiles;
  char *ws = static_cast<char *>(workspace);
  a.parts = reinterpret_cast<float *>(ws + p.parts);
  a.part_sums = reinterpret_cast<float *>(ws + p.sums);
  const auto s = static_cast<hipStream_t>(stream);
  return args->dtype == CASCADE_BF16 ? start<CASCADE_BF16>(a, p, cap, s) : start<CASCADE_F16>(a, p, cap, s);
}
