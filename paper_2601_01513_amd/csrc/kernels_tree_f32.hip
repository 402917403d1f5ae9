// Tree attention of fp32 caches (tree_attn.h).
#include "tree_attn.h"

namespace vsr {

hipError_t launch_tree_f32(const TreeAttnArgs &a, void *ws, hipStream_t s) {
  return launch_tree<float>(a, ws, s);
}

}  // namespace vsr
