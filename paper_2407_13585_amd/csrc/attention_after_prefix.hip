// Attention over what requests have behind a prefix that they share (include/fc.h, fc_prefix_attention).
#include "attention.hpp"

namespace fc {

template AttentionKernel attention_kernel_of<Form::kAfterPrefix>(int32_t, unsigned, bool);

}  // namespace fc
