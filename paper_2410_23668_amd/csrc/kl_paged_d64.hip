// Paged attention instances for head_dim 64.
#include "kl_paged_attn.h"

namespace kl {

hipError_t launch_paged_attention_d64(const AttnParams &p, hipStream_t stream) {
    return launch_attention_for<64>(p, stream);
}

}  // namespace kl
