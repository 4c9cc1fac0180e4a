// Attention of chunks, f32 / 64.
#include "chunk_attend.hpp"

namespace roco {
hipError_t launch_chunk_attend_f32_64(const ChunkArgs& a, hipStream_t s) { return chunk::launch_attend<kF32, 64>(a, s); }
}  // namespace roco
