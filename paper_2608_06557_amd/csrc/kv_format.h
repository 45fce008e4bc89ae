// kv_format.h -- the 8-bit KV cache's chunk layout, its batch and its host
// checks, shared by the kernels that write and read it.  Internal to the
// library.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "cascade.h"

namespace cascade {

constexpr int kMaxBatch = 2048;
constexpr int kMaxKvLen = 1 << 30;

// Where a chunk's codes and scales lie; passed to kernels by value.
struct KvView {
  const char *base;  // of the layer's K chunks
  int64_t kv_stride, slot_stride;
  int num_slots;
  int block_shift;  // log2(block_tokens)
  int kv_heads, head_dim;
};

inline bool kv_format_ok(const cascade_kv_format_t *f) {
  if (!f || f->kv_heads < 1 || f->kv_heads > 256) return false;
  if (f->head_dim != 64 && f->head_dim != 128 && f->head_dim != 256) return false;
  return f->block_tokens == 16 || f->block_tokens == 32 || f->block_tokens == 64 ||
         f->block_tokens == 128;
}

inline int64_t kv_chunk_bytes(const cascade_kv_format_t *f) {
  const int64_t codes = (int64_t)f->kv_heads * f->block_tokens * f->head_dim;
  return codes + (4 * f->kv_heads + 15) / 16 * 16;
}

inline bool kv_pool_ok(const cascade_kv_pool_t *p, int32_t layer, const cascade_kv_format_t *f) {
  if (!p || !p->base || !kv_format_ok(f)) return false;
  if (p->num_layers < 1 || layer < 0 || layer >= p->num_layers || p->num_slots < 1) return false;
  if (p->chunk_bytes < kv_chunk_bytes(f)) return false;
  if ((p->layer_stride & 15) || (p->kv_stride & 15) || (p->slot_stride & 15)) return false;
  if (p->layer_stride < 0 || p->kv_stride < 0 || p->slot_stride < 0) return false;
  return ((uintptr_t)p->base & 15) == 0;
}

inline bool kv_batch_ok(const cascade_kv_batch_t *b, const cascade_block_table_t *t) {
  if (!b || !t || b->n < 0 || b->n > kMaxBatch || b->n_tokens < 0 || b->max_new < 0 ||
      b->n_entries < 0)
    return false;
  if (b->n == 0) return true;
  return b->token_offsets && b->kv_len && t->row_offsets && (b->n_entries == 0 || t->slots);
}

inline bool kv_rows_ok(const cascade_rows_t *r) {
  return r && r->data && ((uintptr_t)r->data & 15) == 0 && (r->token_stride & 7) == 0 &&
         (r->head_stride & 7) == 0 && r->token_stride >= 0 && r->head_stride >= 0;
}

inline KvView kv_view(const cascade_kv_pool_t *p, int32_t layer, const cascade_kv_format_t *f) {
  KvView v;
  v.base = static_cast<const char *>(p->base) + (int64_t)layer * p->layer_stride;
  v.kv_stride = p->kv_stride;
  v.slot_stride = p->slot_stride;
  v.num_slots = p->num_slots;
  v.block_shift = __builtin_ctz((unsigned)f->block_tokens);
  v.kv_heads = f->kv_heads;
  v.head_dim = f->head_dim;
  return v;
}

// A load from memory that no kernel of the launch writes, at an address that
// is the same in all lanes: through the constant address space it goes to the
// scalar unit, whatever the kernel stores elsewhere.
template <typename T>
__device__ __forceinline__ T uniform_load(const T *p) {
  return *(const __attribute__((address_space(4))) T *)(p);
}

// The same through the vector unit: a register the compiler knows nothing of
// makes the address look different in every lane.
template <typename T>
__device__ __forceinline__ T vector_load(const T *p) {
  int none;
  asm("v_mov_b32 %0, 0" : "=v"(none));
  return p[none];
}

// A request of a batch, checked against the arrays it points into.
struct KvRequest {
  int first, count;  // new tokens: rows first .. first + count
  int len;           // cached tokens, the new ones included
  int row;           // first entry of the table row
  bool ok;
};

template <bool kUniform = false>
__device__ __forceinline__ KvRequest kv_request(const cascade_kv_batch_t &b,
                                                const int32_t *row_offsets, int block_shift,
                                                int i) {
  const auto load = [](const int32_t *p) { return kUniform ? uniform_load(p) : *p; };
  KvRequest r;
  r.first = load(b.token_offsets + i);
  const int end = load(b.token_offsets + i + 1);
  r.len = load(b.kv_len + i);
  r.row = load(row_offsets + i);
  const int row_end = load(row_offsets + i + 1);
  r.count = (int)((unsigned)end - (unsigned)r.first);
  r.ok = r.first >= 0 && end >= r.first && end <= b.n_tokens && r.count <= b.max_new &&
         r.len >= 0 && r.len <= kMaxKvLen && r.row >= 0 && row_end >= r.row &&
         row_end <= b.n_entries &&
         ((long long)r.len + (1 << block_shift) - 1) >> block_shift <= row_end - r.row;
  return r;
}

__device__ __forceinline__ void kv_report(int32_t *status) {
  if (status) *status = CASCADE_EINVAL;
}

}  // namespace cascade
