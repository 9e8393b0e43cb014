// Attention over 8-bit pages, causal or with a mask among the new tokens, for gfx950 (MI355X): instances of
// attention_kernels.hpp.

#include "attention_kernels.hpp"

namespace kvp {

hipError_t launch_attention_e4m3(const AttentionArgs &a, uint32_t dtype, hipStream_t stream)
{
    return dtype == KVP_BF16 ? by_head_dim<BF16, kEight>(a, stream) : by_head_dim<F16, kEight>(a, stream);
}

}  // namespace kvp
