// Attention of chunks, bf16 / 64.
#include "chunk_attend.hpp"

namespace roco {
hipError_t launch_chunk_attend_bf16_64(const ChunkArgs& a, hipStream_t s) { return chunk::launch_attend<kBF16, 64>(a, s); }
}  // namespace roco
