// Attention of chunks over a paged cache: a cache of codes, bf16 queries (paged_chunk.hpp).
#include "paged_chunk.hpp"

namespace halo {

int launch_chunk_q8(const ChunkArgs &a, hipStream_t s) { return launch_chunk_dim<KindQ8>(a, s); }

}  // namespace halo
