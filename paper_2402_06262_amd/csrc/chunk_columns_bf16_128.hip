// Sums of chunks over their rows, bf16 / 128.
#include "chunk_columns.hpp"

namespace roco {
hipError_t launch_chunk_columns_bf16_128(const ChunkArgs& a, hipStream_t s) { return chunk::launch_columns<kBF16, 128>(a, s); }
}  // namespace roco
