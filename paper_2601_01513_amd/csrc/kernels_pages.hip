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

// What a block knows of the sequences, in LDS. heir[s]: who goes on with source s's own
// last page: s if it stays, else the lowest-numbered sequence that becomes s (INT32_MAX:
// nobody).
struct Seqs {
  int src[kMaxSeqs], held[kMaxSeqs], len[kMaxSeqs], heir[kMaxSeqs];
};

template <int NT>
__device__ __forceinline__ void load_seqs(const PagesUpdateArgs &a, Seqs &q) {
  const int n = a.pages.n_seqs;
  for (int d = threadIdx.x; d < n; d += NT) {
    const int s = source_of(a.source, n, d), held = held_of(a.pages, d);
    q.src[d] = s;
    q.held[d] = held;
    q.len[d] = len_of(a.pages, d, held);
    q.heir[d] = s == d ? d : INT32_MAX;
  }
  __syncthreads();
  if (!a.source) return;
  for (int d = threadIdx.x; d < n; d += NT) {
    const int s = q.src[d];
    if (s >= 0 && s != d && q.src[s] != s) atomicMin(&q.heir[s], d);
  }
  __syncthreads();
}

// Tables and counts of the sequences that change, columns [c0, c0 + 2^shift) of all: all
// are read before any is written, so that sequences may change places. A page that stays
// partly filled is counted for its heir alone; the entry of another names the page that is
// copied into its own below.
constexpr int kForkThreads = 1024, kForkEntries = 8192;

__device__ __forceinline__ void fork_tables(const PagesUpdateArgs &a, const Seqs &q, int32_t *fresh,
                                            int c0, int shift) {
  const PageTables &p = a.pages;
  const int n = p.n_seqs << shift, part = (1 << p.page_shift) - 1;
#pragma unroll 1
  for (int i = threadIdx.x; i < n; i += kForkThreads) {
    const int d = i >> shift, c = c0 + (i & ((1 << shift) - 1)), s = q.src[d];
    int page = -1;
    if (s >= 0 && s != d && c < p.max_pages && c < pages_for(q.len[s], p.page_shift))
      page = p.table[s * p.table_stride + c];
    fresh[i] = page;
  }
  __syncthreads();
#pragma unroll 1
  for (int i = threadIdx.x; i < n; i += kForkThreads) {
    const int d = i >> shift, c = c0 + (i & ((1 << shift) - 1)), s = q.src[d];
    if (s == d || c >= p.max_pages) continue;
    int32_t *at = p.table + d * p.table_stride + c;
    if (c < q.held[d]) {
      const int old = *at;
      if (is_page(p, old)) atomicSub(&p.refs[old], 1);
    }
    if (s < 0 || c >= pages_for(q.len[s], p.page_shift)) continue;
    const int page = fresh[i];
    *at = page;
    const bool full = c < q.len[s] >> p.page_shift || !(q.len[s] & part);
    if ((full || q.heir[s] == d) && is_page(p, page)) atomicAdd(&p.refs[page], 1);
  }
}

__global__ __launch_bounds__(kForkThreads) void k_fork_tables(PagesUpdateArgs a, int shift) {
  __shared__ Seqs q;
  __shared__ int32_t fresh[kForkEntries];
  load_seqs<kForkThreads>(a, q);
  for (int c0 = blockIdx.x << shift; c0 < a.pages.max_pages; c0 += gridDim.x << shift) {
    fork_tables(a, q, fresh, c0, shift);
    __syncthreads();  // (fresh is free)
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

__device__ __forceinline__ uint32_t plus(uint32_t a, uint32_t b) {  // (at most 2^32 - 1)
  return __builtin_elementwise_add_sat(a, b);
}

// Inclusive prefix sum over N lanes.
template <int N>
__device__ __forceinline__ uint32_t lane_sums(uint32_t v) {
#pragma unroll 1
  for (int d = 1; d < N; d <<= 1) {
    const uint32_t o = __shfl_up(v, d);
    if ((int)(threadIdx.x & 63) >= d) v = plus(v, o);
  }
  return v;
}

// Exclusive prefix sum over the threads of a block, and the total; more than 2^32 - 1 is
// 2^32 - 1.
template <int NT>
__device__ __forceinline__ uint32_t block_rank(uint32_t mine, uint32_t *sums, uint32_t &total) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const uint32_t v = lane_sums<64>(mine);
  __syncthreads();
  if (lane == 63) sums[w] = v;
  __syncthreads();
  const uint32_t all = lane_sums<NT / 64>(lane < NT / 64 ? sums[lane] : 0);
  total = __shfl(all, NT / 64 - 1);
  const uint32_t before = __shfl(all, max(w - 1, 0)), own = __shfl_up(v, 1);
  return plus(w ? before : 0, lane ? own : 0);
}

// The sequences' new sizes and their new pages. One block: a prefix sum of what each
// sequence needs, then the free pages as far as they are needed, first counted, then
// listed by their ranks and handed out, a thread a page. Small tables are forked by the
// same block (FORK). What takes the time is the way there: seven trips to memory in a row,
// fourteen barriers and 4 KB of code to fetch (7.4 us for 64 sequences).
constexpr int kRoomThreads = 1024, kRoomPages = 16;

// Bit i: page first + i is free.
__device__ __forceinline__ uint32_t free_pages(const PageTables &p, int first) {
  typedef Pack<int32_t, 4> I4;
  uint32_t bits = 0;
  if (first <= p.n_pages - kRoomPages) {  // (first + kRoomPages may pass 2^31)
    I4 r[kRoomPages / 4];
#pragma unroll
    for (int i = 0; i < kRoomPages / 4; ++i)
      r[i] = *reinterpret_cast<const I4 *>(p.refs + first + 4 * i);
#pragma unroll
    for (int i = 0; i < kRoomPages; ++i) bits |= (uint32_t)(r[i / 4].v[i % 4] == 0) << i;
  } else {
#pragma unroll 1
    for (int i = 0; first + i < p.n_pages; ++i) bits |= (uint32_t)(p.refs[first + i] == 0) << i;
  }
  return bits;
}

// What sequence d goes on with.
struct Turn {
  int len, kept, need;  // positions, pages, new pages
  bool copy, fits;      // the last page is copied into the first new one; room is to be had
};
__device__ __forceinline__ Turn turn_of(const PagesUpdateArgs &a, const Seqs &q, int d) {
  const PageTables &p = a.pages;
  const int s = q.src[d], part = (1 << p.page_shift) - 1;
  Turn t;
  t.len = s >= 0 ? q.len[s] : 0;
  const int have = s == d ? q.held[d] : pages_for(t.len, p.page_shift);
  t.copy = s >= 0 && s != d && (t.len & part) && q.heir[s] != d;
  const long pages = ((long)t.len + (a.room ? max(a.room[d], 0) : 0) + part) >> p.page_shift;
  t.fits = pages <= p.max_pages;
  t.need = t.copy + (t.fits ? max(0, (int)pages - have) : 0);
  t.kept = have - t.copy;
  return t;
}

constexpr int kAllMemory = 0x0f70;  // s_waitcnt's word for "no load, store or atomic is on its way"

template <bool FORK>
__global__ __launch_bounds__(kRoomThreads) void k_room(PagesUpdateArgs a, PageCopies *copies,
                                                       int shift) {
  constexpr int STEP = kRoomThreads * kRoomPages;
  __shared__ Seqs q;
  __shared__ uint32_t first[kMaxSeqs + 1];  // rank of each sequence's first new page
  __shared__ int kept[kMaxSeqs];            // pages it goes on with
  __shared__ __attribute__((aligned(4))) uint16_t list[STEP];           // free pages by their ranks
  __shared__ uint32_t sums[kRoomThreads / 64];
  __shared__ int n_copies;
  const PageTables &p = a.pages;
  const int n = p.n_seqs, tid = threadIdx.x;
  if (tid == 0) n_copies = 0;
  load_seqs<kRoomThreads>(a, q);
  if constexpr (FORK) {
    static_assert(sizeof(list) >= sizeof(int32_t) * kForkEntries, "");
    fork_tables(a, q, reinterpret_cast<int32_t *>(list), 0, shift);
    // Every wave's stores and counts lie in the L2 before the others read on (the barrier's
    // own release does not wait for them), and no older line of the L1 is read.
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup");
    __builtin_amdgcn_s_waitcnt(kAllMemory);
    __syncthreads();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "agent");
  }
  const int per = (n + kRoomThreads - 1) / kRoomThreads, d0 = tid * per, d1 = min(n, d0 + per);
  uint32_t mine = 0, total, found, most = 0;
#pragma unroll 1
  for (int d = d0; d < d1; ++d) mine = plus(mine, turn_of(a, q, d).need);
  uint32_t rank = block_rank<kRoomThreads>(mine, sums, total);
  uint32_t bits = 0, k = 0, all = 0;
  int walked = 0;
#pragma unroll 1
  for (int listing = 0; listing < 2; ++listing) {
    uint32_t base = 0;
    const uint32_t until = listing ? most : total;
#pragma unroll 1
    for (long at = 0; at < p.n_pages && base < until; at += STEP) {
      if (!listing || walked > 1) {  // (else what was counted is held here)
        const long from = at + tid * kRoomPages;
        bits = from < p.n_pages ? free_pages(p, (int)from) : 0;
        k = block_rank<kRoomThreads>(__popc(bits), sums, all);
        walked += !listing;
      }
      if (listing) {
#pragma unroll 1
        for (uint32_t i = k; bits && base + i < most; ++i, bits &= bits - 1)
          list[i] = (uint16_t)(tid * kRoomPages + __builtin_ctz(bits));
        __syncthreads();
#pragma unroll 1
        for (uint32_t i = tid; i < min(all, most - base); i += kRoomThreads) {
          // The free page of that rank is the last sequence's whose first is not above it.
          int lo = 0, hi = n;
          while (hi - lo > 1) {
            const int mid = (lo + hi) / 2;
            if (first[mid] <= base + i)
              lo = mid;
            else
              hi = mid;
          }
          if (first[lo + 1] > found) continue;  // not served
          const int page = (int)at + list[i];
          p.refs[page] = 1;
          p.table[lo * p.table_stride + kept[lo] + (base + i - first[lo])] = page;
        }
        __syncthreads();
      }
      base += all;
    }
    if (listing) break;
    // Served: all whose needs, with those before them, are met. Of a copy that is not, the
    // full pages stay.
    found = base;
    most = min(total, found);
#pragma unroll 1
    for (int d = d0; d < d1; ++d) {
      const Turn t = turn_of(a, q, d);
      first[d] = rank;
      kept[d] = t.kept;
      rank = plus(rank, t.need);
      const bool served = t.need == 0 || rank <= found;
      const int part = t.len & ((1 << p.page_shift) - 1);
      p.held[d] = t.kept + (served ? t.need : 0);
      p.len[d] = t.copy && !served ? t.len - part : t.len;
      if (a.ok) a.ok[d] = served && t.fits;
      if (t.copy && served) {  // (in any order: the copies are independent)
        const int from = p.table[d * p.table_stride + t.kept];
        copies->at[atomicAdd(&n_copies, 1)] = {d, t.kept, from, part};
      }
    }
    if (tid == 0) first[n] = total;
    __syncthreads();
  }
  if (copies && tid == 0) copies->n = n_copies;
}

// Bytes [at, at + sizeof(U)) of row `slot` of one head.
template <typename U>
__device__ __forceinline__ U *row_at(char *base, long slot_stride, long slot, long at) {
  return reinterpret_cast<U *>(base + slot * slot_stride + at);
}

// The copied rows in every layer (16 x 4 beams of 36 layers: 17 MB in 5.9 us). Grid (layers, matrices and heads in turn; copies).
template <typename U>
__global__ __launch_bounds__(256) void k_copy_pages(PageTables p, CacheRows c,
                                                    const PageCopies *copies) {
  const int per = 2 * c.n_layers * c.n_heads, n = copies->n;
  // A row's pieces by `across` threads, as many rows at once as the block has room for.
  const int pieces = (int)(c.row / sizeof(U)), across = min(pieces, 256), rows = 256 / across;
  const int r0 = threadIdx.x / across, k0 = threadIdx.x - r0 * across;
  for (int u = blockIdx.y; u < n; u += gridDim.y) {
    const PageCopy x = copies->at[u];
    const int to = p.table[x.seq * p.table_stride + x.col];
    if (!is_page(p, x.from) || !is_page(p, to)) continue;
    const long a = (long)x.from << p.page_shift, b = (long)to << p.page_shift;
    for (int i = blockIdx.x; i < per; i += gridDim.x) {
      const int head = i % c.n_heads, layer = i / (2 * c.n_heads);
      char *base = (i / c.n_heads & 1 ? c.v : c.k) + layer * c.layer_stride + head * c.head_stride;
      for (int r = r0; r0 < rows && r < x.rows; r += rows)
        for (int k = k0; k < pieces; k += across)
          *row_at<U>(base, c.slot_stride, b + r, (long)k * sizeof(U)) =
              *row_at<U>(base, c.slot_stride, a + r, (long)k * sizeof(U));
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

// Grid ((layer, matrix, head, slice) / 4, sequence): a wave moves a slice of 64 pieces of
// the rows (64 sequences of 28 layers, 33 MB read and written: 10.2 us, 3.2 TB/s; the list
// and the table come before each wave's first load).
// Rows move to lower places only, and rise: eight are read, then written, then the next,
// and no row is written that a later one is read from.
template <typename U>
__global__ __launch_bounds__(256) void k_keep_rows(PagesKeepArgs a, int slices, int units) {
  const PageTables &p = a.pages;
  const CacheRows &c = a.cache;
  const int lane = threadIdx.x & 63;
  const int u = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (threadIdx.x >> 6)), s = blockIdx.y;
  if (u >= units) return;
  const int v = u / slices, slice = u - v * slices, vh = v / c.n_heads, head = v - vh * c.n_heads;
  const int kv = vh & 1, layer = vh >> 1;
  int len, room;
  bounds_of(p, s, len, room);
  const int n = kept_of(a, s, len, room);
  if (a.len_out != p.len && !a.release && u == 0 && lane == 0) a.len_out[s] = len + n;
  const int32_t *kept = a.kept + s * a.kept_stride, *table = p.table + s * p.table_stride;
  char *base = (kv ? c.v : c.k) + layer * c.layer_stride + head * c.head_stride;
  const int piece = (slice * 64 + lane) * (int)sizeof(U);
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
  const int units = 2 * a.cache.n_layers * a.cache.n_heads * slices;
  k_keep_rows<U><<<dim3((units + 3) / 4, a.pages.n_seqs), 256, 0, s>>>(a, slices, units);
  return hipGetLastError();
}

}  // namespace

size_t pages_update_workspace_bytes(int n_seqs) {
  return sizeof(PageCopies) - sizeof(PageCopy) * (kMaxSeqs - n_seqs);
}

hipError_t launch_pages_update(const PagesUpdateArgs &a, void *ws, hipStream_t s) {
  PageCopies *copies = a.source ? static_cast<PageCopies *>(ws) : nullptr;
  const int n = a.pages.n_seqs;
  int shift = 0;
  if (a.source)
    while (1 << shift < a.pages.max_pages && n << (shift + 1) <= kForkEntries) ++shift;
  // One block is as fast as a launch more while it passes over the table twice at most: 9.0
  // us against 4.1 + 7.0 for 3 sequences of 128 entries, 13.4 against 4.9 + 7.4 for 64 of 64.
  if (a.source && 1 << shift >= a.pages.max_pages && n << shift <= 2 * kForkThreads) {
    k_room<true><<<1, kRoomThreads, 0, s>>>(a, copies, shift);
  } else {
    if (a.source) {
      shift = std::min(shift, 4);  // (16 columns are a line of the table.)
      // (A launch has below 2^32 threads: wider tables in turns.)
      const int blocks = std::min(((a.pages.max_pages - 1) >> shift) + 1, 1 << 16);
      k_fork_tables<<<blocks, kForkThreads, 0, s>>>(a, shift);
      const hipError_t e = hipGetLastError();
      if (e != hipSuccess) return e;
    }
    k_room<false><<<1, kRoomThreads, 0, s>>>(a, copies, 0);
  }
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || !a.source) return e;
  const CacheRows c = merged(a.cache);
  const int across = std::min(2 * c.n_layers * c.n_heads, 1024);
  const dim3 grid(across, std::min(n, std::max(1, 2048 / across)));
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
