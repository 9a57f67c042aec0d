// Paged attention of drafted bfloat16 tokens; the kernels stand in pages_stream.h and pages_tile.h.
#include "pages_tree_launch.h"

namespace sali {

hipError_t launch_pages_attend_tree_bf16(int store, int dim, const PagesAttend& a, hipStream_t s) { return launch_pages_attend_tree<true>(store, dim, a, s); }

}  // namespace sali
