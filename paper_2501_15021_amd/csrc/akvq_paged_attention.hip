// Attention of a chunk over pages of 2-bit codes (akvq_paged_attention.h).
#include "akvq_paged_attention.h"

namespace akvq {
hipError_t launch_paged_attention(const PagedAttentionArgs &a, int G, hipStream_t stream) { return launch_attention<2>(a, G, stream); }
}  // namespace akvq
