// tree_attend of fp32 / 64: a file of its own, so that the forms compile side by side.
#include "tree_attend.hpp"

namespace roco {
hipError_t launch_tree_attend_f32_64(const TreeArgs& a, hipStream_t s) { return tree::launch_attend_rows<kF32, 64>(a, s); }
}  // namespace roco
