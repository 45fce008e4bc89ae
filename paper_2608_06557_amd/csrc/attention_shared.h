// attention_shared.h -- attention with shared prefixes for one type of rows,
// instantiated in a source file each.  Internal to the library.
#pragma once
#include "attention_tiles.h"

namespace cascade {

struct SharedCall {
  Attention attention;
  char *workspace;
  Workspace places;
  Cap cap;
  hipStream_t stream;
};
int shared_attention_bf16(const SharedCall &c);
int shared_attention_f16(const SharedCall &c);

// The parts of one kernel.
struct PartSet {
  const float *parts, *sums;
  int groups, rows;  // workgroups, rows of a tile
};
struct SharedJoin {
  PartSet of[2];
};

// Whether what `sources` says of a token was said by this call: a request that has
// it was taken, and the group if it is in one.  Called by all lanes, where
// something was refused.
__device__ __forceinline__ bool taken(const Attention &a, int token) {
  const int lane = lane_id();
  bool alone = false, found = false;
  int leader = -1;
  for (int i = lane; i < a.batch.n; i += 64) {
    const int what = a.taken[i];
    if (what == kRefused || token < a.batch.token_offsets[i] || token >= a.batch.token_offsets[i + 1]) continue;
    if (what == kAlone) alone = true;
    else leader = a.leader[i];
  }
  if (__any(alone)) return true;
  const uint64_t in = __ballot(leader >= 0);
  if (!in) return false;
  leader = __builtin_amdgcn_readlane(leader, __ffsll((unsigned long long)in) - 1);
  // the group's rows end where its last request's do
  const bool behind = token >= a.batch.token_offsets[leader];
  for (int i = lane; i < a.batch.n; i += 64)
    found |= behind && a.taken[i] == kGroup && a.leader[i] == leader && token < a.batch.token_offsets[i + 1];
  return __any(found);
}

// Joins what is known of each row, a row to a wave: the parts of its request's
// segment, or its state, and the same of its group's.  A chain of dependent loads,
// then the parts: 128 tokens of 64 heads of 128 dims 9 us behind 32 groups of 4 tokens, 12 where
// the row tiles of one group left 8 parts of each row, 33 MB.
template <int kType, int kDim>
__global__ __launch_bounds__(kBlock) void join_shared_kernel(Attention a, SharedJoin j) {
  constexpr int kLanes = kDim / 4, kHalves = 64 / kLanes;
  const int64_t rows = (int64_t)a.batch.n_tokens * a.q_heads;
  const int64_t row = (int64_t)blockIdx.x * kWaves + __builtin_amdgcn_readfirstlane(wave_id());
  if (row >= rows) return;
  const int lane = lane_id(), token = (int)(row / a.q_heads), head = (int)(row % a.q_heads);
  // rows of no request stay as they are
  const int refused = uniform_load(a.taken + a.batch.n);
  if (token < uniform_load(a.batch.token_offsets) || token >= uniform_load(a.batch.token_offsets + a.batch.n)) return;
  const float *parts[2], *sums[2];  // of the first of each
  int count[2], step[2];            // how many, and rows from one place to the next
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const int64_t at = ((k ? a.batch.n_tokens : 0) + (int64_t)token) * a.kv.kv_heads + head / a.group;
    const int *from = reinterpret_cast<const int *>(a.sources + at);
    const Source s = {uniform_load(from), uniform_load(from + 1), uniform_load(from + 2), uniform_load(from + 3)};
    if (k == 0 && s.kind == kWritten) return;
    const bool split = s.kind >= kParts;
    const PartSet &p = j.of[s.kind == kParts + 1];
    // within the workspace whatever was told
    const int w = min(max(s.w, 1), p.groups - 1);
    const int in_tile = min(max(s.row, 0) + head % a.group, p.rows - 1);
    const int64_t first = split ? (int64_t)(w - 1) * 2 * p.rows + in_tile : (k ? rows : 0) + row;
    parts[k] = (split ? p.parts : a.states) + first * kDim;
    sums[k] = (split ? p.sums : a.state_sums) + first * 2;
    count[k] = split ? min(max(s.last, w), p.groups - 1) - w + 2 : s.kind == kState;
    step[k] = split ? p.rows : 0;
  }
  if (__builtin_expect(refused, false) && !taken(a, token)) return;
  // two places a workgroup: part 0 ends its range, the others begin theirs
  const int all = count[0] + count[1];
  auto place = [&](int c, int &k) -> int64_t {
    k = c >= count[0];
    c -= k ? count[0] : 0;
    return (int64_t)step[k] * (2 * c + (c == 0));
  };
  auto sums_of = [&](int c) {
    int k;
    const int64_t at = place(c, k);
    return *reinterpret_cast<const f2 *>(sums[k] + 2 * at);
  };
  float top = kLowest;
  for (int c = lane; c < all; c += 64) top = fmaxf(top, sums_of(c)[0]);
#pragma unroll
  for (int d = 32; d; d >>= 1) top = fmaxf(top, __shfl_xor(top, d));
  float sum = 0.f;
  for (int c = lane; c < all; c += 64) {
    const f2 ms = sums_of(c);
    sum += ms[1] * __builtin_amdgcn_exp2f(ms[0] - top);
  }
#pragma unroll
  for (int d = 32; d; d >>= 1) sum += __shfl_xor(sum, d);
  f4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
  for (int c = lane / kLanes; c < all; c += kHalves) {
    int k;
    const int64_t at = place(c, k);
    o += *reinterpret_cast<const f4 *>(parts[k] + at * kDim + 4 * (lane % kLanes)) *
         __builtin_amdgcn_exp2f(sums[k][2 * at] - top);
  }
#pragma unroll
  for (int d = 32; d >= kLanes; d >>= 1)
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] += __shfl_xor(o[i], d);
  if (lane < kLanes) {
    const float f = sum > 0.f ? 1.f / sum : sum == 0.f ? 0.f : sum;
    const u2 x = {narrow2<kType>(o[0] * f, o[1] * f), narrow2<kType>(o[2] * f, o[3] * f)};
    *reinterpret_cast<u2 *>(a.out.data + (int64_t)token * a.out.token_stride + (int64_t)head * a.out.head_stride +
                            8 * lane) = x;
  }
  if (a.lse && lane == 0) a.lse[row] = (top + __builtin_amdgcn_logf(sum)) * kLn2;
}

template <int kType, int kDim>
void attend_shared(const SharedCall &c) {
  Attention a = c.attention;
  const int64_t most = (int64_t)std::max(a.max_tokens, a.batch.max_new) * a.group;  // rows of a request or group
  const bool tiled = most > most_rows(kDim);
  // Where groups need row tiles and no request has over 16 rows, those of up to 32
  // are groups: the requests' form is theirs alone.  128 single tokens of 611 tokens each
  // beside a group of 1024 rows 49 us, in the 32-row form 53.  Groups of 17 to 32 rows are row tiles
  // then, which costs more where there are many: one group of 128 tokens beside 31 of four, behind 8 and
  // 4 Ki tokens, 64/8 heads, 262 us, in the 32-row form 209; the 31 beside one of nine 145 and 136.
  const int64_t rest = (int64_t)a.batch.max_new * a.group;
  const int small = tiled && rest <= 16 ? 16 : few_rows(most, kDim);
  SharedJoin j = {};
  a.which = 0;
  const int grid = attend_few<Form::kShared, kType, kDim>(a, c.workspace, c.places, c.cap, small, c.stream);
  j.of[0] = j.of[1] = PartSet{a.parts, a.part_sums, grid, small};
  auto tiles = [&](auto stage) {
    constexpr int kStage = decltype(stage)::value;
    a.which = 1;
    attend_tiles<Form::kShared, kType, kDim, kStage>(a, c.workspace, c.places, c.cap, small, c.stream);
    j.of[1] = PartSet{a.parts, a.part_sums, kTileGroups * stage_tokens(kDim) / kStage, tile_rows(kStage)};
  };
  // Tiles of half the rows, unless a group fills four whole ones: 12 groups of 104
  // rows on average 102 us, in whole ones 166; a group of 1024 rows 60, in whole ones 52.  Between them
  // they are alike or whole ones faster: calls of four groups of 256, 384, 512, 768 and 1016 rows behind
  // 8 Ki tokens 114, 160, 194, 280 and 361 us, in whole ones 111, 161, 184, 265 and 338.
  if (tiled && most < 1024)
    tiles(std::integral_constant<int, 32>());
  else if (tiled)
    tiles(std::integral_constant<int, stage_tokens(kDim)>());
  const int64_t rows = (int64_t)a.batch.n_tokens * a.q_heads;
  hipLaunchKernelGGL((join_shared_kernel<kType, kDim>), dim3((unsigned)((rows + kWaves - 1) / kWaves)), dim3(kBlock),
                     0, c.stream, a, j);
}

template <int kType>
int attend_shared(const SharedCall &c) {
  switch (c.attention.kv.head_dim) {
    case 64: attend_shared<kType, 64>(c); break;
    case 128: attend_shared<kType, 128>(c); break;
    default: attend_shared<kType, 256>(c);
  }
  return hipGetLastError() == hipSuccess ? CASCADE_OK : CASCADE_EHIP;
}

}  // namespace cascade
