// Paged attention over a cache of codes: float queries, up to 16 of a cache head at once (paged_attention.hpp).
#include "paged_attention.hpp"

namespace halo {

int launch_attend_q8_f32(const AttendArgs &a, hipStream_t s) { return launch_dim<CoreQ8Float>(a, s); }

}  // namespace halo
