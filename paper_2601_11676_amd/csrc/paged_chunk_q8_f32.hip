// Attention of chunks over a paged cache: a cache of codes, float queries (paged_chunk.hpp).
#include "paged_chunk.hpp"

namespace halo {

int launch_chunk_q8_f32(const ChunkArgs &a, hipStream_t s) { return launch_chunk_dim<KindQ8F32>(a, s); }

}  // namespace halo
