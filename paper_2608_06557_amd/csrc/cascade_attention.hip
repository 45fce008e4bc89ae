// cascade_attention.hip -- attention of a ragged batch's new tokens over the
// 8-bit paged KV cache, and the weight that it gives to blocks, on gfx950.
#include "attention_tiles.h"

namespace cascade {
namespace {

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

template <int kType, int kDim>
int run(Attention a, char *ws, const Workspace &w, Cap cap, float *block_weight, hipStream_t s) {
  const int64_t most = (int64_t)a.batch.max_new * a.group;  // rows of a request and KV head
  const int64_t table = (int64_t)a.batch.n_entries << a.kv.block_shift;
  const bool tiled = most > most_rows(kDim);
  const int small = few_rows(most, kDim);
  if (!tiled || a.batch.n > 1) {
    const int grid = attend_few<Form::kWhole, kType, kDim>(a, ws, w, cap, small, s);
    if (table > a.atomic_keys)  // else none is cut
      hipLaunchKernelGGL((join_kernel<kType, kDim>), dim3(grid, small / kWaves), dim3(kBlock), 0, s, a, small, 1);
  }
  if (tiled) {
    constexpr int kStage = stage_tokens(kDim), kRows = tile_rows(kStage);
    attend_tiles<Form::kWhole, kType, kDim, kStage>(a, ws, w, cap, a.batch.n > 1 ? small : 0, s);
    if (table > a.least_keys)
      hipLaunchKernelGGL((join_kernel<kType, kDim>), dim3(kTileGroups, kRows / (2 * kWaves)), dim3(kBlock), 0, s, a,
                         kRows, 2);
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
  if (!kv_pool_ok(pool, layer, format) || !kv_batch_ok(batch, table) || !attention_ok(args, format))
    return CASCADE_EINVAL;
  if (args->block_weight ? args->weight_window < 1 || args->weight_window > 64 : args->weight_window != 0)
    return CASCADE_EINVAL;
  if (!workspace || ((uintptr_t)workspace & 255)) return CASCADE_EINVAL;
  const Workspace w = layout(format, batch, args->q_heads, args->weight_window);
  if (workspace_bytes < w.total) return CASCADE_ENOSPC;
  if (batch->n == 0 || batch->n_tokens == 0 || batch->max_new == 0) return CASCADE_OK;
  if (!kv_rows_ok(&args->q) || !kv_rows_ok(&args->out)) return CASCADE_EINVAL;
  Cap cap;
  Attention a = attention_of(pool, layer, format, batch, table, args, status_dev, cap);
  char *ws = static_cast<char *>(workspace);
  a.window = args->weight_window;
  a.lse = args->lse ? args->lse : a.window ? reinterpret_cast<float *>(ws + w.lse) : nullptr;
  a.log_shift = log_shift(format);
  a.logs = a.window && batch->n_entries ? reinterpret_cast<float *>(ws + w.logs) : nullptr;
  const auto s = static_cast<hipStream_t>(stream);
  float *weight = a.logs ? args->block_weight : nullptr;
  return args->dtype == CASCADE_BF16 ? run<CASCADE_BF16>(a, ws, w, cap, weight, s)
                                     : run<CASCADE_F16>(a, ws, w, cap, weight, s);
}

