// cascade_attention_shared_f16.hip -- the float16 kernels of attention with
// shared prefixes (cascade_attention_shared.hip), apart only so that the two
// types compile side by side.
#include "attention_shared.h"

namespace cascade {
int shared_attention_f16(const SharedCall &c) { return attend_shared<CASCADE_F16>(c); }
}  // namespace cascade
