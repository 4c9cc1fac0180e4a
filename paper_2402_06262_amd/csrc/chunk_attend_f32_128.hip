// Attention of chunks, f32 / 128.
#include "chunk_attend.hpp"

namespace roco {
hipError_t launch_chunk_attend_f32_128(const ChunkArgs& a, hipStream_t s) { return chunk::launch_attend<kF32, 128>(a, s); }
}  // namespace roco
