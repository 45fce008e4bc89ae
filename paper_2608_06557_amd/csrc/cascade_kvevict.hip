// cascade_kvevict.hip -- blocks with the least accumulated attention weight
// leave their requests, on gfx950.
//
// One workgroup per request.  How many blocks it drops follows from lengths
// and budgets alone, so every workgroup adds up the earlier requests' counts
// itself and knows where its rows and freed slots go: one launch, no
// hand-over.  Which ones: the count-th least weight by a radix selection, 8
// bits of the weights' ordered form a pass (histogram in LDS), then one pass
// in index order that drops what lies below it and the first of the equal
// ones.  A thread keeps its weights (one, or 8 neighbours of a request of more than
// 1024 blocks) in registers between the passes; the call is bound by latency (8192 blocks of each of 64 requests:
// FIGURE).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "cascade.h"
#include "device_util.h"
#include "kv_format.h"

namespace cascade {
namespace {

constexpr int kThreads = 1024;
constexpr int kEvictWaves = kThreads / 64;

struct Counts {
  int blocks, begin, end, gone;  // candidates begin .. end, `gone` of them dropped
  bool ok;
};

__device__ __forceinline__ Counts count_blocks(const cascade_evict_t &a, const int32_t *row_offsets,
                                               int i) {
  const int len = a.kv_len[i], keep = a.keep_blocks[i];
  const int row = row_offsets[i], row_end = row_offsets[i + 1];
  Counts c;
  c.blocks = (int)(((long long)len + a.block_tokens - 1) / a.block_tokens);
  c.ok = len >= 0 && len <= kMaxKvLen && keep >= 0 && row >= 0 && row_end >= row &&
         row_end <= a.n_entries && c.blocks <= row_end - row;
  if (!c.ok) c.blocks = 0;
  c.begin = min(a.sink, c.blocks);
  c.end = max(c.begin, c.blocks - min(a.recent, c.blocks));
  c.gone = min(max(c.blocks - keep, 0), c.end - c.begin);
  return c;
}

// Weights in ascending order as whole numbers: -0 as 0, NaN last.
__device__ __forceinline__ unsigned ordered(float w) {
  const unsigned b = __float_as_uint(w);
  if ((b & 0x7fffffffu) > 0x7f800000u) return 0xffffffffu;
  if ((b << 1) == 0) return 0x80000000u;
  return b >> 31 ? ~b : b | 0x80000000u;
}

// One request's blocks, kPer neighbours to a thread.
template <int kPer>
__device__ __forceinline__ void evict_blocks(const cascade_evict_t &a, const Counts &c, const float *weight,
                                             const int32_t *slot, const unsigned long long (&before)[2],
                                             unsigned *hist, unsigned *scan, unsigned *picked) {
  const int tid = threadIdx.x;
  // a thread's weights: kPer neighbours of the first kThreads * kPer blocks stay
  // in registers, those of longer requests are read again in every pass
  auto load = [&](int b0, float (&w)[kPer]) {
#pragma unroll
    for (int j = 0; j < kPer; ++j) w[j] = b0 + j < c.blocks ? weight[b0 + j] : 0.f;
  };
  float first[kPer];
  load(tid * kPer, first);

  // the gone-th least: `key` once all digits are known, of which `equal` go
  unsigned key = 0, equal = 0;
  if (c.gone > 0) {
    unsigned rank = c.gone - 1;
    for (int shift = 24; shift >= 0; shift -= 8) {
      if (tid < 256) hist[tid] = 0;
      __syncthreads();
      const unsigned high = shift == 24 ? 0u : ~0u << (shift + 8);
      auto count = [&](int b0, const float (&w)[kPer]) {
#pragma unroll
        for (int j = 0; j < kPer; ++j) {
          const unsigned k = ordered(w[j]);
          if (b0 + j >= c.begin && b0 + j < c.end && ((k ^ key) & high) == 0)
            atomicAdd(&hist[(k >> shift) & 255u], 1u);
        }
      };
      count(tid * kPer, first);
      for (int b0 = (kThreads + tid) * kPer; b0 < c.end; b0 += kThreads * kPer) {
        float w[kPer];
        load(b0, w);
        count(b0, w);
      }
      __syncthreads();
      if (tid < 64) {
        unsigned h[4], sum = 0;
        for (int d = 0; d < 4; ++d) sum += h[d] = hist[4 * tid + d];
        unsigned at = wave_inclusive_sum(sum) - sum;
        for (int d = 0; d < 4; ++d) {
          if (rank >= at && rank < at + h[d]) {
            picked[0] = key | (unsigned)(4 * tid + d) << shift;
            picked[1] = rank - at;
          }
          at += h[d];
        }
      }
      __syncthreads();
      key = picked[0];
      rank = picked[1];
      __syncthreads();
    }
    equal = rank + 1;
  }

  unsigned base[2] = {0, 0};  // below the key, equal to it: among the blocks so far
  for (int c0 = 0; c0 < c.blocks; c0 += kThreads * kPer) {
    const int b0 = c0 + tid * kPer;
    float w[kPer];
    int32_t held[kPer];
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
      w[j] = first[j];
      held[j] = b0 + j < c.blocks ? slot[b0 + j] : 0;
    }
    if (c0) load(b0, w);
    unsigned v[2] = {0, 0}, total[2];
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
      const bool can = c.gone > 0 && b0 + j >= c.begin && b0 + j < c.end;
      v[0] += can && ordered(w[j]) < key;
      v[1] += can && ordered(w[j]) == key;
    }
    block_exclusive_scan<2, unsigned, kEvictWaves>(v, total, scan);
    unsigned less = base[0] + v[0], same = base[1] + v[1];
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
      const int b = b0 + j;
      const bool can = c.gone > 0 && b >= c.begin && b < c.end;
      const bool below = can && ordered(w[j]) < key, on = can && ordered(w[j]) == key;
      const unsigned gone_before = less + min(same, equal);
      if (b < c.blocks) {
        if (below || (on && same < equal)) {
          const unsigned long long at = before[1] + gone_before;
          if (at < (unsigned long long)a.n_entries) a.freed[at] = held[j];
        } else {
          const unsigned long long at = before[0] + (b - gone_before);
          if (at < (unsigned long long)a.n_entries) {
            a.slots_out[at] = held[j];
            a.weight_out[at] = w[j];
          }
        }
      }
      less += below;
      same += on;
    }
    base[0] += total[0];
    base[1] += total[1];
  }
}

__global__ __launch_bounds__(kThreads) void evict_kernel(cascade_evict_t a,
                                                         const int32_t *row_offsets,
                                                         const int32_t *slots, int32_t *status) {
  __shared__ unsigned hist[256];
  __shared__ unsigned long long sums[kEvictWaves * 2];
  __shared__ unsigned scan[kEvictWaves * 2];
  __shared__ unsigned picked[2];
  const int i = blockIdx.x, tid = threadIdx.x;
  // blocks kept and dropped by the requests before this one
  unsigned long long before[2] = {0, 0};
  for (int j = tid; j < i; j += kThreads) {
    const Counts c = count_blocks(a, row_offsets, j);
    before[0] += c.blocks - c.gone;
    before[1] += c.gone;
  }
  block_sum<2, unsigned long long, kEvictWaves>(before, sums);
  const Counts c = count_blocks(a, row_offsets, i);
  const unsigned long long rows_end = before[0] + (c.blocks - c.gone);
  if (tid == 0) {
    a.kv_len_out[i] = c.ok ? a.kv_len[i] - c.gone * a.block_tokens : 0;
    a.row_offsets_out[i + 1] = (int)min(rows_end, (unsigned long long)a.n_entries);
    if (i == 0) a.row_offsets_out[0] = 0;
    if (i == a.n - 1) *a.n_freed = (int)min(before[1] + c.gone, (unsigned long long)a.n_entries);
    if (!c.ok) kv_report(status);
    if (status && rows_end + before[1] + c.gone > (unsigned long long)a.n_entries)
      *status = CASCADE_ENOSPC;
  }
  if (!c.ok) return;
  const float *weight = a.block_weight + row_offsets[i];
  const int32_t *slot = slots + row_offsets[i];
  if (c.blocks <= kThreads)
    evict_blocks<1>(a, c, weight, slot, before, hist, scan, picked);
  else
    evict_blocks<8>(a, c, weight, slot, before, hist, scan, picked);
}

__global__ void evict_none_kernel(cascade_evict_t a) {
  a.row_offsets_out[0] = 0;
  *a.n_freed = 0;
}

}  // namespace
}  // namespace cascade

using namespace cascade;

extern "C" int cascade_kv_evict(const cascade_block_table_t *table, const cascade_evict_t *args,
                                int32_t *status_dev, void *stream) {
  if (!table || !args || args->n < 0 || args->n > kMaxBatch || args->n_entries < 0 ||
      args->block_tokens < 1 || args->sink < 0 || args->recent < 1)
    return CASCADE_EINVAL;
  if (!args->row_offsets_out || !args->n_freed) return CASCADE_EINVAL;
  const auto s = static_cast<hipStream_t>(stream);
  if (args->n == 0) {
    hipLaunchKernelGGL(evict_none_kernel, dim3(1), dim3(1), 0, s, *args);
    return hipGetLastError() == hipSuccess ? CASCADE_OK : CASCADE_EHIP;
  }
  if (!args->kv_len || !args->keep_blocks || !args->kv_len_out || !table->row_offsets)
    return CASCADE_EINVAL;
  if (args->n_entries > 0 && (!args->block_weight || !args->slots_out || !args->weight_out ||
                              !args->freed || !table->slots))
    return CASCADE_EINVAL;
  hipLaunchKernelGGL(evict_kernel, dim3(args->n), dim3(kThreads), 0, s, *args, table->row_offsets,
                     table->slots, status_dev);
  return hipGetLastError() == hipSuccess ? CASCADE_OK : CASCADE_EHIP;
}
