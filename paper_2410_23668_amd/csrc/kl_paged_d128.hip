// Paged attention instances for head_dim 128.
#include "kl_paged_attn.h"

namespace kl {

hipError_t launch_paged_attention_d128(const AttnParams &p, hipStream_t stream) {
    return launch_attention_for<128>(p, stream);
}

}  // namespace kl
