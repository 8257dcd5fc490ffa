// The backward of the masked attention, bf16, heads of 64 (one translation unit per head dimension: they compile side by side).
#include "sbp_lm_attention_bwd.h"

namespace sbp {
template void launch_masked_backward_bf16<64>(const MaskedAttention&, const LmTables&, hipStream_t);
}
