// Attention on float32 tensors.
#include "attn_kernels.hpp"

namespace mure {

hipError_t attn_short_f32(const AttnArgs& k, hipStream_t s) { return with_head<float>(k, true, s); }
hipError_t attn_runs_f32(const AttnArgs& k, hipStream_t s) { return with_head<float>(k, false, s); }
hipError_t attn_join_f32(const AttnArgs& k, int keys, hipStream_t s) { return join<float>(k, keys, s); }

}  // namespace mure
