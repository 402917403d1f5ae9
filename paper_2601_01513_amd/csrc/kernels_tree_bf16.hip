// Tree attention of bfloat16 caches (tree_attn.h).
#include "tree_attn.h"

namespace vsr {

hipError_t launch_tree_bf16(const TreeAttnArgs &a, void *ws, hipStream_t s) {
  return launch_tree<bf16>(a, ws, s);
}

}  // namespace vsr
