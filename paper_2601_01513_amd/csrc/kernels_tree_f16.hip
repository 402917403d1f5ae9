// Tree attention of fp16 caches (tree_attn.h).
#include "tree_attn.h"

namespace vsr {

hipError_t launch_tree_f16(const TreeAttnArgs &a, void *ws, hipStream_t s) {
  return launch_tree<f16>(a, ws, s);
}

}  // namespace vsr
