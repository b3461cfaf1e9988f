// Paged attention over a cache of codes: bf16 queries, up to 32 of a cache head at once (paged_attention.hpp).
#include "paged_attention.hpp"

namespace halo {

int launch_attend_q8_32(const AttendArgs &a, hipStream_t s) { return launch_dim_128<CoreQ8Two>(a, s); }

}  // namespace halo
