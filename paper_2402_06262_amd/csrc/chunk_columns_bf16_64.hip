// Sums of chunks over their rows, bf16 / 64.
#include "chunk_columns.hpp"

namespace roco {
hipError_t launch_chunk_columns_bf16_64(const ChunkArgs& a, hipStream_t s) { return chunk::launch_columns<kBF16, 64>(a, s); }
}  // namespace roco
