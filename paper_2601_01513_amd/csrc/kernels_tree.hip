// Drafted rows over a paged key/value cache: their positions, slots and ancestor masks.
// (Their attention: tree_attn.h.)
#include "common.h"
#include "tree_attn.h"

namespace vsr {

namespace {

// ---------------------------------------------------------------- rows of a tree

// One block a sequence, and one more for the rows of none. A row's mask is its path
// to the root, walked up its parents (in LDS): words are met in falling order, each
// stored once.
constexpr int kRowsThreads = 256, kRowsLds = 8192;

__global__ __launch_bounds__(kRowsThreads) void k_tree_rows(TreeRowsArgs a) {
  __shared__ int32_t up[kRowsLds];
  const int s = blockIdx.x, tid = threadIdx.x;
  if (s == a.pages.n_seqs) {
    int b0, e0, b1, e1;
    seq_rows(a.start, a.T, 0, b0, e0);
    seq_rows(a.start, a.T, s - 1, b1, e1);
    for (int i = tid; i < b0 + a.T - e1; i += kRowsThreads) {
      const int r = i < b0 ? i : e1 + i - b0;
      a.pos[r] = 0;
      a.slot[r] = -1;
      for (int w = 0; w < a.mask_words; ++w) a.mask[r * a.mask_stride + w] = 0;
    }
    return;
  }
  int b, e;
  seq_rows(a.start, a.T, s, b, e);
  const int n = e - b;
  const int32_t *parent = a.parent ? a.parent + b : nullptr;
  if (parent) {
    for (int j = tid; j < min(n, kRowsLds); j += kRowsThreads) up[j] = parent[j];
    __syncthreads();
  }
  // A parent that does not come before its row is none.
  const auto above = [&](int j) {
    if (!parent) return j - 1;
    const int u = j < kRowsLds ? up[j] : parent[j];
    return u < j ? max(u, -1) : -1;
  };
  const int len = seq_len(a.pages, s), room = seq_room(a.pages, s);
  const int shift = a.shift ? a.shift[s] : 0;
  const int32_t *table = a.pages.table + s * a.pages.table_stride;
  for (int j = tid; j < n; j += kRowsThreads) {
    uint32_t *row = a.mask ? a.mask + (b + j) * a.mask_stride : nullptr;
    int depth = 0;
    if (!parent && !row) {
      depth = j;
    } else {
      int word = a.mask_words;
      uint32_t bits = 0;
      for (int x = j; x >= 0; x = above(x)) {
        ++depth;
        if (row && x >> 5 < a.mask_words) {
          if (x >> 5 != word) {
            if (word < a.mask_words) row[word] = bits;
            for (--word; word > x >> 5; --word) row[word] = 0;
            bits = 0;
          }
          bits |= 1u << (x & 31);
        }
      }
      --depth;
      if (row) {
        if (word < a.mask_words) row[word] = bits;
        for (--word; word >= 0; --word) row[word] = 0;
      }
    }
    a.pos[b + j] = (int)((uint32_t)len + (uint32_t)shift + (uint32_t)depth);
    int slot = -1;
    const long at = (long)len + j;
    if (at < room) {
      const int page = table[at >> a.pages.page_shift];
      if ((uint32_t)page < (uint32_t)a.pages.n_pages)
        slot = (page << a.pages.page_shift) | (int)(at & ((1 << a.pages.page_shift) - 1));
    }
    a.slot[b + j] = slot;
  }
}

}  // namespace

hipError_t launch_tree_rows(const TreeRowsArgs &a, hipStream_t s) {
  k_tree_rows<<<a.pages.n_seqs + 1, kRowsThreads, 0, s>>>(a);
  return hipGetLastError();
}

size_t tree_attention_workspace_bytes(int hd, int T, int n_seqs, int n_heads, int n_kv) {
  const int HD = hd <= 64 ? 64 : hd <= 128 ? 128 : 256;
  const int rows = std::max(32, tree_block_rows(tree_rows_of(T, n_seqs, n_heads, n_kv)));
  return (size_t)kTreeGroups * (2 * rows * (HD * sizeof(float) + sizeof(float2)) + sizeof(TreeJoin));
}

hipError_t launch_tree_attention(const TreeAttnArgs &given, int dtype, void *ws, hipStream_t s) {
  TreeAttnArgs a = given;
  a.group = a.n_heads / a.n_kv;
  // With 2^b >= group, ceil(2^(31 + b) / group) times r < 2^31 is off by less than 2^(31 + b) / group.
  int b = 0;
  while (1 << b < a.group) ++b;
  a.group_shift = 31 + b;
  a.group_mul = (uint32_t)(((1ull << a.group_shift) + a.group - 1) / a.group);
  if (dtype == 0) return launch_tree_f32(a, ws, s);
  if (dtype == 1) return launch_tree_bf16(a, ws, s);
  return launch_tree_f16(a, ws, s);
}

}  // namespace vsr
