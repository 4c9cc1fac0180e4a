// Attention of chunks, bf16 / 128.
#include "chunk_attend.hpp"

namespace roco {
hipError_t launch_chunk_attend_bf16_128(const ChunkArgs& a, hipStream_t s) { return chunk::launch_attend<kBF16, 128>(a, s); }
}  // namespace roco
