// Sums of chunks over their rows, f32 / 64.
#include "chunk_columns.hpp"

namespace roco {
hipError_t launch_chunk_columns_f32_64(const ChunkArgs& a, hipStream_t s) { return chunk::launch_columns<kF32, 64>(a, s); }
}  // namespace roco
