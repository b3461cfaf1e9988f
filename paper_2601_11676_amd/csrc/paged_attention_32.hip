// Paged attention: bf16, up to 32 queries of a cache head at once (paged_attention.hpp).
#include "paged_attention.hpp"

namespace halo {

int launch_attend_bf16_32(const AttendArgs &a, hipStream_t s) { return launch_dim_128<CoreBf16Two>(a, s); }

}  // namespace halo
