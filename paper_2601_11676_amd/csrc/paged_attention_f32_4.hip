// Paged attention: float, up to 4 queries of a cache head (paged_attention.hpp).
#include "paged_attention.hpp"

namespace halo {

int launch_attend_f32_4(const AttendArgs &a, hipStream_t s) { return launch_dim<CoreF32Few>(a, s); }

}  // namespace halo
