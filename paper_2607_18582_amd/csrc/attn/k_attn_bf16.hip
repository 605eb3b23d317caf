// Attention on bfloat16 tensors.
#include "attn_kernels.hpp"

namespace mure {

hipError_t attn_short_bf16(const AttnArgs& k, hipStream_t s) { return with_head<bf16_t>(k, true, s); }
hipError_t attn_runs_bf16(const AttnArgs& k, hipStream_t s) { return with_head<bf16_t>(k, false, s); }
hipError_t attn_join_bf16(const AttnArgs& k, int keys, hipStream_t s) { return join<bf16_t>(k, keys, s); }

}  // namespace mure
