// tree_attend of bf16 / 128: a file of its own, so that the forms compile side by side.
#include "tree_attend.hpp"

namespace roco {
hipError_t launch_tree_attend_bf16_128(const TreeArgs& a, hipStream_t s) { return tree::launch_attend_rows<kBF16, 128>(a, s); }
}  // namespace roco
