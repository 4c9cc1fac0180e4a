// tree_attend of bf16 / 64: a file of its own, so that the forms compile side by side.
#include "tree_attend.hpp"

namespace roco {
hipError_t launch_tree_attend_bf16_64(const TreeArgs& a, hipStream_t s) { return tree::launch_attend_rows<kBF16, 64>(a, s); }
}  // namespace roco
