// cascade_kvevict.hip -- blocks with the least accumulated attention weight
// leave their requests, on gfx950.
//
// One workgroup per request.  How many blocks it drops follows from lengths
// and budgets alone, so every workgroup adds up the earlier requests' counts
// itself and knows where its rows and freed slots go: one launch, no
// hand-over.  Which ones: the count-th least weight by a radix selection, 8
// bits of the weights' ordered form a pass (histogram in LDS), which ends
// when the blocks that share the digits so far all go; then one pass in index
// order that drops what lies below them and the first of the equal ones.
//
// The least it can read and write is small (64 requests of up to 8192 blocks:
// 7 MB, 1 us); the call is bound by the latency of dependent loads and
// barriers.  So a pass has one barrier (each has a histogram of its own, and
// every wave finds the digit itself), weights and slots stay in registers
// (one block to a thread, or 8 in a request of more than 1024), and places in
// index order come from ballots.  64 requests of up to 8192 blocks: 13 us,
// with three barriers a pass, weights of neighbours in a thread and a scan of
// the block 21 us, with one block to a thread read again in each pass 24 us;
// 128 requests of 130 to 2048 blocks: 9 us; one request of 512: 7 us.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "cascade.h"
#include "device_util.h"
#include "kv_format.h"

namespace cascade {
namespace {

constexpr int kThreads = 1024;
constexpr int kEvictWaves = kThreads / 64;

// Neighbouring blocks often share a digit, and adds to one LDS address take
// turns: each digit is counted in 4 places, by lane.
constexpr int kCopies = 4;

struct Lds {
  uint4 hist[4][256];                 // per pass and digit, kCopies counts
  unsigned marks[2][8 * kEvictWaves];  // per 64 blocks: below the key, equal to it << 16
  unsigned long long sums[kEvictWaves * 2];
};

struct Counts {
  int blocks, begin, end, gone;  // candidates begin .. end, `gone` of them dropped
  bool ok;
};

__device__ __forceinline__ Counts count_blocks(const cascade_evict_t &a, const int32_t *row_offsets,
                                               int i) {
  const int len = a.kv_len[i], keep = a.keep_blocks[i];
  const int row = row_offsets[i], row_end = row_offsets[i + 1];
  Counts c;
  const bool sane = len >= 0 && len <= kMaxKvLen && row >= 0 && row_end >= row && row_end <= a.n_entries;
  c.blocks = sane ? ((unsigned)len + (unsigned)a.block_tokens - 1) / (unsigned)a.block_tokens : 0;
  c.ok = sane && keep >= 0 && c.blocks <= row_end - row;
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

// One request: block t + kThreads j of each kThreads * kPer is thread t's.
template <int kPer>
__device__ __forceinline__ void evict_blocks(const cascade_evict_t &a, const int32_t *row_offsets,
                                             const int32_t *slots, int32_t *status, const Counts &c, int i,
                                             Lds &lds) {
  static_assert(kPer == 1 || kPer == 8, "marks are summed by one wave, one or two to a lane");
  constexpr int kChunk = kThreads * kPer;
  const int tid = threadIdx.x, lane = lane_id();
  const int wave = __builtin_amdgcn_readfirstlane(wave_id());
  const int row = c.ok ? row_offsets[i] : 0;
  const float *weight = a.block_weight + row;
  const int32_t *slot = slots + row;
  // the first chunk's stay in registers, later ones are read again in every pass
  auto load = [&](auto *from, int b0, auto (&to)[kPer]) {
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
      const int b = b0 + j * kThreads + tid;
      to[j] = b < c.blocks ? from[b] : 0;
    }
  };
  float first[kPer];
  int32_t first_held[kPer];
  load(weight, 0, first);
  load(slot, 0, first_held);

  // blocks kept and dropped by the requests before this one
  unsigned long long before[2] = {0, 0};
  for (int j = tid; j < i; j += kThreads) {
    const Counts e = count_blocks(a, row_offsets, j);
    before[0] += e.blocks - e.gone;
    before[1] += e.gone;
  }
  block_sum<2, unsigned long long, kEvictWaves>(before, lds.sums);
  if (tid == 0) {
    const unsigned long long rows_end = before[0] + (c.blocks - c.gone);
    a.kv_len_out[i] = c.ok ? a.kv_len[i] - c.gone * a.block_tokens : 0;
    a.row_offsets_out[i + 1] = (int)min(rows_end, (unsigned long long)a.n_entries);
    if (i == 0) a.row_offsets_out[0] = 0;
    if (i == a.n - 1) *a.n_freed = (int)min(before[1] + c.gone, (unsigned long long)a.n_entries);
    if (!c.ok) kv_report(status);
    if (status && rows_end + before[1] + c.gone > (unsigned long long)a.n_entries)
      *status = CASCADE_ENOSPC;
  }

  // the gone-th least: its digits as far as they are needed, and how many of
  // the blocks with these digits go
  unsigned key = 0, known = 0, equal = 0;
  if (c.gone > 0) {
    unsigned rank = c.gone - 1;
#pragma unroll 1
    for (int pass = 0; pass < 4; ++pass) {
      const int shift = 24 - 8 * pass;
      unsigned *hist = &lds.hist[pass][0].x + (lane & (kCopies - 1));
      auto count = [&](int b0, const float (&w)[kPer]) {
#pragma unroll
        for (int j = 0; j < kPer; ++j) {
          if (j && b0 + j * kThreads >= c.end) break;
          const int b = b0 + j * kThreads + tid;
          const unsigned k = ordered(w[j]);
          if (b >= c.begin && b < c.end && ((k ^ key) & known) == 0)
            atomicAdd(&hist[((k >> shift) & 255u) * kCopies], 1u);
        }
      };
      count(0, first);
      for (int b0 = kChunk; b0 < c.end; b0 += kChunk) {
        float w[kPer];
        load(weight, b0, w);
        count(b0, w);
      }
      __syncthreads();
      // every wave finds the digit, 4 to a lane
      unsigned h[4], sum = 0;
#pragma unroll
      for (int d = 0; d < 4; ++d) {
        const uint4 n = lds.hist[pass][4 * lane + d];
        sum += h[d] = n.x + n.y + n.z + n.w;
      }
      unsigned at = wave_inclusive_sum(sum) - sum;
      const int from = __ffsll((unsigned long long)__ballot(rank >= at && rank < at + sum)) - 1;
      unsigned digit = 4 * lane, size = h[0];
#pragma unroll
      for (int d = 0; d < 3; ++d) {
        const bool later = digit == 4u * lane + d && rank >= at + h[d];
        at += later ? h[d] : 0;
        digit += later;
        size = later ? h[d + 1] : size;
      }
      key |= (unsigned)__builtin_amdgcn_readlane(digit, from) << shift;
      rank -= __builtin_amdgcn_readlane(at, from);
      known |= 255u << shift;
      if (rank + 1 == (unsigned)__builtin_amdgcn_readlane(size, from)) break;  // all of them
    }
    equal = rank + 1;
  }

  unsigned base[2] = {0, 0};  // below the key, equal to it: among the blocks so far
  for (int c0 = 0, turn = 0; c0 < c.blocks; c0 += kChunk, turn ^= 1) {
    float w[kPer];
    int32_t held[kPer];
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
      w[j] = first[j];
      held[j] = first_held[j];
    }
    if (c0) {
      load(weight, c0, w);
      load(slot, c0, held);
    }
    unsigned long long below[kPer], on[kPer];
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
      const int b = c0 + j * kThreads + tid;
      const bool can = c.gone > 0 && b >= c.begin && b < c.end;
      const unsigned k = ordered(w[j]) & known;
      below[j] = __ballot(can && k < key);
      on[j] = __ballot(can && k == key);
      if (lane == 0) lds.marks[turn][j * kEvictWaves + wave] = __popcll(below[j]) | __popcll(on[j]) << 16;
    }
    __syncthreads();
    unsigned mark[2] = {0, 0};
    if constexpr (kPer == 1) {
      if (lane < kEvictWaves) mark[0] = lds.marks[turn][lane];
    } else {
      mark[0] = lds.marks[turn][2 * lane];
      mark[1] = lds.marks[turn][2 * lane + 1];
    }
    const unsigned inc = wave_inclusive_sum(mark[0] + mark[1]);  // halves stay under 2^16
    const unsigned upto = inc - mark[0] - mark[1];
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
      if (j && c0 + j * kThreads >= c.blocks) break;
      unsigned all;
      if constexpr (kPer == 1) {
        all = __builtin_amdgcn_readlane(upto, wave);
      } else {
        const int from = (j * kEvictWaves + wave) >> 1;
        all = __builtin_amdgcn_readlane(upto, from) + (wave & 1 ? __builtin_amdgcn_readlane(mark[0], from) : 0);
      }
      const int b = c0 + j * kThreads + tid;
      const unsigned long long mine = 1ull << lane;
      const unsigned less = base[0] + (all & 0xffffu) + __popcll(below[j] & (mine - 1));
      const unsigned same = base[1] + (all >> 16) + __popcll(on[j] & (mine - 1));
      const unsigned gone_before = less + min(same, equal);
      if (b < c.blocks) {
        if ((below[j] & mine) || ((on[j] & mine) && same < equal)) {
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
    }
    const unsigned all = __builtin_amdgcn_readlane(inc, 63);
    base[0] += all & 0xffffu;
    base[1] += all >> 16;
  }
}

__global__ __launch_bounds__(kThreads) void evict_kernel(cascade_evict_t a,
                                                         const int32_t *row_offsets,
                                                         const int32_t *slots, int32_t *status) {
  __shared__ Lds lds;
  static_assert(sizeof(lds.hist) == 16 * kThreads, "one store a thread clears them");
  const int i = blockIdx.x;
  (&lds.hist[0][0])[threadIdx.x] = uint4{0, 0, 0, 0};
  const Counts c = count_blocks(a, row_offsets, i);
  if (c.blocks <= kThreads)
    evict_blocks<1>(a, row_offsets, slots, status, c, i, lds);
  else
    evict_blocks<8>(a, row_offsets, slots, status, c, i, lds);
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
