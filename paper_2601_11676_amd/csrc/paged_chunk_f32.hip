// Attention of chunks over a paged cache: float rows (paged_chunk.hpp).
#include "paged_chunk.hpp"

namespace halo {

int launch_chunk_f32(const ChunkArgs &a, hipStream_t s) { return launch_chunk_dim<KindF32>(a, s); }

}  // namespace halo
