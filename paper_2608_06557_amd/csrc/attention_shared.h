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

template <int kType, int kDim>
void attend_shared(const SharedCall &c) {
  const Attention &a = c.attention;
  attend<Form::kPrefix, kType, kDim>(a, c.workspace, c.places, c.cap, a.max_tokens, c.stream);
  attend<Form::kRest, kType, kDim>(a, c.workspace, c.places, c.cap, a.batch.max_new, c.stream);
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
