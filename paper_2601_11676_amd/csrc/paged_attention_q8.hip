// Paged attention over a cache of codes: bf16 queries, up to 16 of a cache head at once (paged_attention.hpp).
#include "paged_attention.hpp"

namespace halo {

int launch_attend_q8(const AttendArgs &a, hipStream_t s) { return launch_dim<CoreQ8One>(a, s); }

}  // namespace halo
