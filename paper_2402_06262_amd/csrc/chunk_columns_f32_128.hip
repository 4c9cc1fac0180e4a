// Sums of chunks over their rows, f32 / 128.
#include "chunk_columns.hpp"

namespace roco {
hipError_t launch_chunk_columns_f32_128(const ChunkArgs& a, hipStream_t s) { return chunk::launch_columns<kF32, 128>(a, s); }
}  // namespace roco
