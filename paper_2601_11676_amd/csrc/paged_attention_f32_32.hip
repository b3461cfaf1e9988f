// Paged attention: float, up to 32 queries of a cache head at once (paged_attention.hpp).
#include "paged_attention.hpp"

namespace halo {

int launch_attend_f32_32(const AttendArgs &a, hipStream_t s) { return launch_dim_128<CoreF32Two>(a, s); }

}  // namespace halo
