// Attention over a table for each key head (include/fc.h, fc_paged_attention with a table of rank 3).
#include "attention.hpp"

namespace fc {

template AttentionKernel attention_kernel_of<Form::kHeads>(int32_t, unsigned, bool);

}  // namespace fc
