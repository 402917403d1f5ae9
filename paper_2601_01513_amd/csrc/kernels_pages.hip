// Pages of a shared key/value cache: sequences forked from others, room for more
// positions, and the kept rows of a draft moved together.
//
// refs[p] counts the sequences that hold page p; a page is free at 0, and new pages are
// the free ones of lowest number, in the order of sequences. That keeps no list of free
// pages, and no order of atomics shows in any result.
#include <algorithm>

#include "common.h"

namespace vsr {

namespace {

constexpr int kMaxSeqs = 4096;

__device__ __forceinline__ int held_of(const PageTables &p, int s) {
  return max(0, min(p.held[s], p.max_pages));
}
__device__ __forceinline__ int len_of(const PageTables &p, int s, int held) {
  return max(0, min(p.len[s], held << p.page_shift));
}
__device__ __forceinline__ int pages_for(long positions, int shift) {
  return (int)((positions + (1 << shift) - 1) >> shift);
}
// Where sequence d's state comes from (-1: nowhere, it becomes empty).
__device__ __forceinline__ int source_of(const int32_t *source, int n_seqs, int d) {
  if (!source) return d;
  const int s = source[d];
  return s == -1 ? -1 : (uint32_t)s < (uint32_t)n_seqs ? s : d;
}
__device__ __forceinline__ bool is_page(const PageTables &p, int page) {
  return (uint32_t)page < (uint32_t)p.n_pages;
}

// heir[s]: who goes on with source s's own last page: s if it stays, else the
// lowest-numbered sequence that becomes s (INT32_MAX: nobody). In LDS.
template <int NT>
__device__ __forceinline__ void find_heirs(const PagesUpdateArgs &a, int *heir) {
  const int n = a.pages.n_seqs;
  for (int s = threadIdx.x; s < n; s += NT)
    heir[s] = source_of(a.source, n, s) == s ? s : INT32_MAX;
  __syncthreads();
  for (int d = threadIdx.x; d < n; d += NT) {
    const int s = source_of(a.source, n, d);
    if (s >= 0 && s != d && source_of(a.source, n, s) != s) atomicMin(&heir[s], d);
  }
  __syncthreads();
}

// Tables and counts of the sequences that change. A block takes a run of 2^shift columns
// of the table for every sequence: it reads them all before it writes any, so that
// sequences may change places. A page that stays partly filled is counted for its heir
// alone; the entry of another names the page that is copied into its own below.
constexpr int kForkThreads = 256, kForkEntries = 8192;

__global__ __launch_bounds__(kForkThreads) void k_fork_tables(PagesUpdateArgs a, int shift) {
  __shared__ int heir[kMaxSeqs];
  __shared__ int32_t fresh[kForkEntries];
  const PageTables &p = a.pages;
  const int n = p.n_seqs, c0 = blockIdx.x << shift, part = (1 << p.page_shift) - 1;
  find_heirs<kForkThreads>(a, heir);
  for (int i = threadIdx.x; i < n << shift; i += kForkThreads) {
    const int d = i >> shift, c = c0 + (i & ((1 << shift) - 1)), s = source_of(a.source, n, d);
    int page = -1;
    if (s >= 0 && s != d && c < p.max_pages &&
        c < pages_for(len_of(p, s, held_of(p, s)), p.page_shift))
      page = p.table[s * p.table_stride + c];
    fresh[i] = page;
  }
  __syncthreads();
  for (int i = threadIdx.x; i < n << shift; i += kForkThreads) {
    const int d = i >> shift, c = c0 + (i & ((1 << shift) - 1)), s = source_of(a.source, n, d);
    if (s == d || c >= p.max_pages) continue;
    int32_t *at = p.table + d * p.table_stride + c;
    if (c < held_of(p, d)) {
      const int old = *at;
      if (is_page(p, old)) atomicSub(&p.refs[old], 1);
    }
    if (s < 0) continue;
    const int len = len_of(p, s, held_of(p, s));
    if (c >= pages_for(len, p.page_shift)) continue;
    *at = fresh[i];
    const bool full = c < len >> p.page_shift || !(len & part);
    if ((full || heir[s] == d) && is_page(p, fresh[i])) atomicAdd(&p.refs[fresh[i]], 1);
  }
}

// The first `rows` rows of page `from` go to the page at column `col` of sequence `seq`.
struct PageCopy {
  int seq, col, from, rows;
};
struct PageCopies {
  int n, pad[3];
  PageCopy at[kMaxSeqs];
};

// Exclusive prefix sum over the threads of a block, and the total.
template <int NT>
__device__ __forceinline__ long block_rank(long mine, long *sums, long &total) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  long v = mine;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const long o = __shfl_up(v, d);
    if (lane >= d) v += o;
  }
  __syncthreads();
  if (lane == 63) sums[w] = v;
  __syncthreads();
  long before = 0;
  total = 0;
#pragma unroll
  for (int i = 0; i < NT / 64; ++i) {
    if (i < w) before += sums[i];
    total += sums[i];
  }
  return before + v - mine;
}

// The sequences' new sizes and their new pages. One block: a prefix sum of what each
// sequence needs, then walks over the counts, one to count free pages as far as they are
// needed, one to hand them out in order.
constexpr int kRoomThreads = 1024, kRoomSeqs = kMaxSeqs / kRoomThreads, kRoomPages = 16;

// Bit i: page first + i is free.
__device__ __forceinline__ uint32_t free_pages(const PageTables &p, int first) {
  typedef Pack<int32_t, 4> I4;
  uint32_t bits = 0;
  if (first + kRoomPages <= p.n_pages) {
#pragma unroll
    for (int i = 0; i < kRoomPages; i += 4) {
      const I4 r = *reinterpret_cast<const I4 *>(p.refs + first + i);
#pragma unroll
      for (int j = 0; j < 4; ++j) bits |= (uint32_t)(r.v[j] == 0) << (i + j);
    }
  } else {
    for (int i = 0; first + i < p.n_pages; ++i) bits |= (uint32_t)(p.refs[first + i] == 0) << i;
  }
  return bits;
}

__global__ __launch_bounds__(kRoomThreads) void k_room(PagesUpdateArgs a, PageCopies *copies) {
  __shared__ int heir[kMaxSeqs];
  __shared__ long first[kMaxSeqs + 1];  // rank of each sequence's first new page
  __shared__ int kept[kMaxSeqs];        // pages it goes on with
  __shared__ long sums[kRoomThreads / 64];
  __shared__ int n_copies;
  constexpr int STEP = kRoomThreads * kRoomPages;
  const PageTables &p = a.pages;
  const int n = p.n_seqs, tid = threadIdx.x, part = (1 << p.page_shift) - 1;
  if (a.source) find_heirs<kRoomThreads>(a, heir);
  if (tid == 0) n_copies = 0;
  const int per = (n + kRoomThreads - 1) / kRoomThreads;
  int need[kRoomSeqs], copy[kRoomSeqs], lens[kRoomSeqs];
  bool fits[kRoomSeqs];
  long mine = 0;
#pragma unroll
  for (int i = 0; i < kRoomSeqs; ++i) {
    const int d = tid * per + i;
    need[i] = copy[i] = lens[i] = 0;
    fits[i] = true;
    if (i >= per || d >= n) continue;
    const int s = source_of(a.source, n, d);
    int have = 0;
    if (s >= 0) {
      const int held = held_of(p, s);
      lens[i] = len_of(p, s, held);
      have = s == d ? held : pages_for(lens[i], p.page_shift);
      copy[i] = s != d && (lens[i] & part) && heir[s] != d;
    }
    const long want = (long)lens[i] + (a.room ? max(a.room[d], 0) : 0);
    const long pages = (want + part) >> p.page_shift;
    fits[i] = pages <= p.max_pages;
    need[i] = copy[i] + (fits[i] ? max(0, (int)pages - have) : 0);
    kept[d] = have - copy[i];
    mine += need[i];
  }
  long total, found = 0, rank = block_rank<kRoomThreads>(mine, sums, total);
  for (long at = 0; at < p.n_pages && found < total; at += STEP) {
    long all;
    const long from = at + tid * kRoomPages;
    block_rank<kRoomThreads>(from < p.n_pages ? __popc(free_pages(p, (int)from)) : 0, sums, all);
    found += all;
  }
  // Served: all whose needs, with those before them, are met. Of a copy that is not, the
  // full pages stay.
#pragma unroll
  for (int i = 0; i < kRoomSeqs; ++i) {
    const int d = tid * per + i;
    if (i >= per || d >= n) continue;
    first[d] = rank;
    rank += need[i];
    const bool served = need[i] == 0 || rank <= found;
    p.held[d] = kept[d] + (served ? need[i] : 0);
    p.len[d] = copy[i] && !served ? lens[i] & ~part : lens[i];
    if (a.ok) a.ok[d] = served && fits[i];
    if (copy[i] && served) {  // (in any order: the copies are independent)
      const int from = p.table[d * p.table_stride + kept[d]];
      copies->at[atomicAdd(&n_copies, 1)] = {d, kept[d], from, lens[i] & part};
    }
  }
  if (tid == 0) first[n] = total;
  __syncthreads();
  if (copies && tid == 0) copies->n = n_copies;
  const long most = min(total, found);
  for (long at = 0, before = 0; at < p.n_pages && before < most; at += STEP) {
    long all;
    const long from = at + tid * kRoomPages;
    uint32_t bits = from < p.n_pages ? free_pages(p, (int)from) : 0;
    long k = before + block_rank<kRoomThreads>(__popc(bits), sums, all);
    for (; bits && k < most; ++k, bits &= bits - 1) {
      // The k-th free page is the last sequence's whose first rank is not above k.
      int lo = 0, hi = n;
      while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if (first[mid] <= k)
          lo = mid;
        else
          hi = mid;
      }
      if (first[lo + 1] > found) continue;  // not served
      const int page = (int)from + __builtin_ctz(bits);
      p.refs[page] = 1;
      p.table[lo * p.table_stride + kept[lo] + (k - first[lo])] = page;
    }
    before += all;
  }
}

// Bytes [at, at + sizeof(U)) of row `slot` of one head.
template <typename U>
__device__ __forceinline__ U *row_at(char *base, long slot_stride, long slot, long at) {
  return reinterpret_cast<U *>(base + slot * slot_stride + at);
}

// The copied rows in every layer: units (copy, layer, matrix, head) in turn.
template <typename U>
__global__ __launch_bounds__(256) void k_copy_pages(PageTables p, CacheRows c,
                                                    const PageCopies *copies) {
  const long per = 2L * c.n_layers * c.n_heads, units = copies->n * per;
  const int pieces = (int)(c.row / sizeof(U));
  for (long u = blockIdx.x; u < units; u += gridDim.x) {
    const PageCopy x = copies->at[u / per];
    const int i = (int)(u % per), head = i % c.n_heads, layer = i / (2 * c.n_heads);
    const int to = p.table[x.seq * p.table_stride + x.col];
    if (!is_page(p, x.from) || !is_page(p, to)) continue;
    char *base = (i / c.n_heads & 1 ? c.v : c.k) + layer * c.layer_stride + head * c.head_stride;
    const long a = (long)x.from << p.page_shift, b = (long)to << p.page_shift;
    for (int k = threadIdx.x; k < x.rows * pieces; k += 256) {
      const int r = k / pieces, at = (k % pieces) * (int)sizeof(U);
      *row_at<U>(base, c.slot_stride, b + r, at) = *row_at<U>(base, c.slot_stride, a + r, at);
    }
  }
}

// ---------------------------------------------------------------- kept rows

// How many entries of sequence s's list are moved: they rise, and lie in its room.
__device__ __forceinline__ int kept_of(const PagesKeepArgs &a, int s, int len, int room) {
  const int lane = threadIdx.x & 63;
  const int32_t *kept = a.kept + s * a.kept_stride;
  const int n = a.n_kept ? max(0, min(a.n_kept[s], a.most)) : a.most;
  int last = -1;
  for (int k0 = 0; k0 < n; k0 += 64) {
    const int k = k0 + lane, x = k < n ? kept[k] : 0;
    int before = __shfl_up(x, 1);
    if (lane == 0) before = last;
    const uint64_t bad = __ballot(k < n && (x <= before || x >= room - len));
    if (bad) return k0 + __builtin_ctzll(bad);
    last = __shfl(x, 63);
  }
  return n;
}

__device__ __forceinline__ void bounds_of(const PageTables &p, int s, int &len, int &room) {
  const int held = held_of(p, s);
  room = held << p.page_shift;
  len = len_of(p, s, held);
}

// A wave moves a slice of 64 pieces of the rows of one (sequence, layer, matrix, head).
// Rows move to lower places only, and rise: eight are read, then written, then the next,
// and no row is written that a later one is read from.
template <typename U>
__global__ __launch_bounds__(256) void k_keep_rows(PagesKeepArgs a, int slices, long units) {
  const PageTables &p = a.pages;
  const CacheRows &c = a.cache;
  const int lane = threadIdx.x & 63;
  const long u = (long)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (u >= units) return;
  const int slice = (int)(u % slices);
  const long v = u / slices;
  const int head = (int)(v % c.n_heads), kv = (int)(v / c.n_heads % 2);
  const int layer = (int)(v / c.n_heads / 2 % c.n_layers);
  const int s = (int)(v / c.n_heads / 2 / c.n_layers);
  int len, room;
  bounds_of(p, s, len, room);
  const int n = kept_of(a, s, len, room);
  if (a.len_out != p.len && !a.release && v == (long)s * c.n_layers * 2 * c.n_heads &&
      slice == 0 && lane == 0)
    a.len_out[s] = len + n;
  const int32_t *kept = a.kept + s * a.kept_stride, *table = p.table + s * p.table_stride;
  char *base = (kv ? c.v : c.k) + layer * c.layer_stride + head * c.head_stride;
  const long piece = ((long)slice * 64 + lane) * sizeof(U);
  const bool in = piece < c.row;
  for (int k0 = 0; k0 < n; k0 += 64) {
    // Lane k: where row k0 + k comes from and goes to (-1: it stays).
    const int k = k0 + lane;
    int from = -1, to = -1;
    if (k < n && kept[k] != k) {
      const int x = len + kept[k], y = len + k, part = (1 << p.page_shift) - 1;
      const int px = table[x >> p.page_shift], py = table[y >> p.page_shift];
      if (is_page(p, px) && is_page(p, py)) {
        from = (px << p.page_shift) | (x & part);
        to = (py << p.page_shift) | (y & part);
      }
    }
    for (int r0 = 0; r0 < min(64, n - k0); r0 += 8) {
      U x[8];
#pragma unroll
      for (int r = 0; r < 8; ++r) {
        const int f = __builtin_amdgcn_readlane(from, r0 + r);
        if (f >= 0 && in) x[r] = *row_at<U>(base, c.slot_stride, f, piece);
      }
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
#pragma unroll
      for (int r = 0; r < 8; ++r) {
        const int t = __builtin_amdgcn_readlane(to, r0 + r);
        if (t >= 0 && in) *row_at<U>(base, c.slot_stride, t, piece) = x[r];
      }
    }
  }
}

// The new lengths, and the pages past them given back. A wave a sequence.
__global__ __launch_bounds__(64) void k_keep_done(PagesKeepArgs a) {
  const PageTables &p = a.pages;
  const int s = blockIdx.x;
  int len, room;
  bounds_of(p, s, len, room);
  const int n = kept_of(a, s, len, room), held = room >> p.page_shift;
  if (a.release) {
    const int left = pages_for((long)len + n, p.page_shift);
    for (int c = left + (int)threadIdx.x; c < held; c += 64) {
      const int page = p.table[s * p.table_stride + c];
      if (is_page(p, page)) atomicSub(&p.refs[page], 1);
    }
    if (threadIdx.x == 0) p.held[s] = left;
  }
  if (threadIdx.x == 0) a.len_out[s] = len + n;
}

// The widest piece (16, 4 or 2 bytes) that every row consists of.
int piece_bytes(const CacheRows &c) {
  const uintptr_t any = reinterpret_cast<uintptr_t>(c.k) | reinterpret_cast<uintptr_t>(c.v) |
                        (uintptr_t)(c.row | c.layer_stride | c.slot_stride | c.head_stride);
  return any % 16 == 0 ? 16 : any % 4 == 0 ? 4 : 2;
}

// Heads side by side make one row.
CacheRows merged(CacheRows c) {
  if (c.n_heads == 1 || c.head_stride == c.row) {
    c.row *= c.n_heads;
    c.n_heads = 1;
    c.head_stride = 0;
  }
  return c;
}

template <typename U>
hipError_t launch_keep_rows(const PagesKeepArgs &a, hipStream_t s) {
  const int slices = (int)((a.cache.row / (long)sizeof(U) + 63) / 64);
  const long units = 2L * a.pages.n_seqs * a.cache.n_layers * a.cache.n_heads * slices;
  k_keep_rows<U><<<(int)((units + 3) / 4), 256, 0, s>>>(a, slices, units);
  return hipGetLastError();
}

}  // namespace

size_t pages_update_workspace_bytes(int n_seqs) {
  return sizeof(PageCopies) - sizeof(PageCopy) * (kMaxSeqs - n_seqs);
}

hipError_t launch_pages_update(const PagesUpdateArgs &a, void *ws, hipStream_t s) {
  PageCopies *copies = a.source ? static_cast<PageCopies *>(ws) : nullptr;
  if (a.source) {
    int shift = 0;
    while (shift < 4 && a.pages.n_seqs << (shift + 1) <= kForkEntries) ++shift;
    k_fork_tables<<<((a.pages.max_pages - 1) >> shift) + 1, kForkThreads, 0, s>>>(a, shift);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  k_room<<<1, kRoomThreads, 0, s>>>(a, copies);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || !a.source) return e;
  const CacheRows c = merged(a.cache);
  const long units = 2L * a.pages.n_seqs * c.n_layers * c.n_heads;
  const int grid = (int)std::min(units, 2048L);
  switch (piece_bytes(c)) {
    case 16:
      k_copy_pages<u32x4><<<grid, 256, 0, s>>>(a.pages, c, copies);
      break;
    case 4:
      k_copy_pages<uint32_t><<<grid, 256, 0, s>>>(a.pages, c, copies);
      break;
    default:
      k_copy_pages<uint16_t><<<grid, 256, 0, s>>>(a.pages, c, copies);
  }
  return hipGetLastError();
}

hipError_t launch_pages_keep(const PagesKeepArgs &given, hipStream_t s) {
  PagesKeepArgs a = given;
  a.cache = merged(a.cache);
  hipError_t e;
  switch (piece_bytes(a.cache)) {
    case 16:
      e = launch_keep_rows<u32x4>(a, s);
      break;
    case 4:
      e = launch_keep_rows<uint32_t>(a, s);
      break;
    default:
      e = launch_keep_rows<uint16_t>(a, s);
  }
  if (e != hipSuccess || (a.len_out != a.pages.len && !a.release)) return e;
  k_keep_done<<<a.pages.n_seqs, 64, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace vsr
