// Paged attention: float, up to 16 queries of a cache head at once (paged_attention.hpp).
#include "paged_attention.hpp"

namespace halo {

int launch_attend_f32(const AttendArgs &a, hipStream_t s) { return launch_dim<CoreF32One>(a, s); }

}  // namespace halo
