// Drafted rows over a paged key/value cache: their positions, slots and ancestor masks.
// (Their attention: tree_attn.h.)
#include "common.h"
#include "tree_attn.h"

namespace vsr {

namespace {

// ---------------------------------------------------------------- rows of a tree

// One block a sequence, and one more for the rows of none. A row's mask is its path to the
// root. The block takes 256 rows at a time: a row walks up its parents in LDS until the
// path leaves these rows, words met in falling order and each stored once, and goes on with
// the depth and the mask of the row it has come to, which are there already. So a chain of n
// rows costs 256 steps for each 256 of them, not n. (3 x 21 rows 2.9 us, 256 x 100 rows of
// random trees 6.4: the start of a launch, the walk, and two trips to memory.)
constexpr int kRowsThreads = 256;
static_assert(kRowsThreads % 32 == 0, "a group of rows begins a word");

__global__ __launch_bounds__(kRowsThreads) void k_tree_rows(TreeRowsArgs a) {
  __shared__ int32_t up[kRowsThreads];
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
  const int len = seq_len(a.pages, s), room = seq_room(a.pages, s);
  const uint32_t base = (uint32_t)len + (uint32_t)(a.shift ? a.shift[s] : 0);
  const int32_t *table = a.pages.table + s * a.pages.table_stride;
  for (int j0 = 0; j0 < n; j0 += kRowsThreads) {
    const int j = j0 + tid;
    if (parent) {
      __syncthreads();  // (the rows before are stored, their parents no longer read)
      // A parent that does not come before its row is none.
      if (j < n) up[tid] = parent[j] < j ? max(parent[j], -1) : -1;
      __syncthreads();
    }
    if (j >= n) continue;
    uint32_t *row = a.mask ? a.mask + (b + j) * a.mask_stride : nullptr;
    uint32_t depth = j;
    if (parent) {
      depth = 0;
      int word = a.mask_words, x = j;  // words from `word` up are stored
      uint32_t bits = 0;
      for (; x >= j0; x = up[x - j0]) {
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
      depth = x < 0 ? depth - 1 : depth + ((uint32_t)a.pos[b + x] - base);
      if (row) {
        if (word < a.mask_words) row[word] = bits;
        const int own = min(j0 >> 5, word);
        for (--word; word >= own; --word) row[word] = 0;
        const uint32_t *above = a.mask + (b + max(x, 0)) * a.mask_stride;
        for (; word >= 0; --word) row[word] = x < 0 ? 0 : above[word];
      }
    } else if (row) {
      for (int w = 0; w < a.mask_words; ++w)
        row[w] = w < j >> 5 ? ~0u : w > j >> 5 ? 0 : ~0u >> (31 - (j & 31));
    }
    a.pos[b + j] = (int)(base + depth);
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
  const size_t rows = tree_all_rows(tree_block_rows(tree_rows_of(T, n_seqs, n_heads, n_kv)), HD);
  return 2 * rows * (HD * sizeof(float) + sizeof(float2)) + kTreeGroups * sizeof(TreeJoin);
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
