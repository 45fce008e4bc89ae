// cascade_attention_shared.hip -- attention of a batch whose neighbouring
// requests share their first blocks, on gfx950.
//
// Softmax over a row's tokens splits at any token: with (m, sum, O) of some and
// of the others it is known of all.  So the work is a list of both: each
// group's shared tokens once, for the rows of all its requests (no row is masked), and each
// request's other tokens.  The kernels of attention_tiles.h take the list in one
// go, groups of many rows as row tiles, where the products bound them instead of the
// reads of the cache; every segment says where it left its rows, and a last launch
// joins each row's two.
//
// Groups of few rows are bound by HBM: 32 groups of 4 tokens behind 1 to 32 Ki tokens, 64/8
// heads of 128 dims, 173 us, 851 MB fetched (776 needed), 4.9 TB/s, two waves a SIMD with
// 32 rows and 65 % of their cycles in waits (codes two steps ahead do not fit the
// registers: 204).  Large groups' row tiles: 1024 rows behind 8 Ki tokens 49 us, the matrix units busy
// 25 % of the cycles, in 16 stages a workgroup, its list and its parts.  One launch each for
// groups and requests, with a join each, took 2 to 30 % longer in all than one list.
//
// Against cascade_attention over the same tables: 17.4 us and 19.5 for 4 tokens behind 4 Ki, 181 and 374 for
// those 32 groups, 110 and 278 for 128 tokens behind 8 Ki.  What is shared twice or more pays from
// about 2 Ki tokens on (128 tokens in groups of 2, 4, 16: of 1 Ki 87, 75 and 86 us against 86, 71 and 64; of
// 2 Ki 114, 88 and 91 against 125, 105 and 82; of 4 Ki 168, 116 and 102 against 210, 179 and 140).
#include "attention_shared.h"

namespace cascade {
int shared_attention_bf16(const SharedCall &c) { return attend_shared<CASCADE_BF16>(c); }

namespace {
// The workspace of attention, then what is known of each row.
struct Places {
  Workspace w;
  size_t states, sums, sources, taken, total;
  Places(const cascade_kv_format_t *f, const cascade_kv_batch_t *b, int q_heads) : w(layout(f, b, q_heads, 0)) {
    const size_t rows = 2 * (size_t)b->n_tokens * q_heads;
    states = w.total;
    sums = states + aligned(sizeof(float) * rows * f->head_dim);
    sources = sums + aligned(sizeof(float) * rows * 2);
    taken = sources + aligned(sizeof(Source) * 2 * b->n_tokens * f->kv_heads);
    total = taken + aligned(sizeof(int) * (kMaxBatch + 1));
  }
};
}  // namespace
}  // namespace cascade

using namespace cascade;

extern "C" size_t cascade_attention_shared_workspace_bytes(const cascade_kv_format_t *format,
                                                           const cascade_kv_batch_t *batch, int32_t q_heads) {
  if (!kv_format_ok(format) || !batch || batch->n_tokens < 0 || batch->n_entries < 0 || !heads_ok(format, q_heads))
    return 0;
  return Places(format, batch, q_heads).total;
}

extern "C" int cascade_attention_shared(const cascade_kv_pool_t *pool, int32_t layer,
                                        const cascade_kv_format_t *format, const cascade_kv_batch_t *batch,
                                        const cascade_block_table_t *table, const cascade_attention_t *args,
                                        const cascade_shared_t *shared, void *workspace, size_t workspace_bytes,
                                        int32_t *status_dev, void *stream) {
  if (!kv_pool_ok(pool, layer, format) || !kv_batch_ok(batch, table) || !attention_ok(args, format) || !shared)
    return CASCADE_EINVAL;
  if (args->block_weight || args->weight_window || shared->max_tokens < 0) return CASCADE_EINVAL;
  if (!workspace || ((uintptr_t)workspace & 255)) return CASCADE_EINVAL;
  const Places p(format, batch, args->q_heads);
  if (workspace_bytes < p.total) return CASCADE_ENOSPC;
  if (batch->n == 0 || batch->n_tokens == 0 || batch->max_new == 0) return CASCADE_OK;
  if (!kv_rows_ok(&args->q) || !kv_rows_ok(&args->out) || !shared->leader || !shared->shared_len)
    return CASCADE_EINVAL;
  Cap cap;
  Attention a = attention_of(pool, layer, format, batch, table, args, status_dev, cap);
  char *ws = static_cast<char *>(workspace);
  a.leader = shared->leader;
  a.shared_len = shared->shared_len;
  a.max_tokens = std::min(shared->max_tokens, batch->n_tokens);
  a.states = reinterpret_cast<float *>(ws + p.states);
  a.state_sums = reinterpret_cast<float *>(ws + p.sums);
  a.sources = reinterpret_cast<Source *>(ws + p.sources);
  a.taken = reinterpret_cast<int *>(ws + p.taken);
  if ((int64_t)batch->n_tokens * args->q_heads > INT32_MAX / kBlock) return CASCADE_EINVAL;
  const SharedCall c = {a, ws, p.w, cap, static_cast<hipStream_t>(stream)};
  return args->dtype == CASCADE_BF16 ? shared_attention_bf16(c) : shared_attention_f16(c);
}
