// Attention of drafted rows over their sequences' pages (kernels_tree_*.hip, a file a
// type).
//
// Sequence s has len[s] positions in its pages; row j of its draft sits at position
// len + j. For query row j and head h, over the positions p it sees (p < len, or bit
// p - len of its mask; without masks p - len <= j):
//   x_p = scale q[j, h] . k[p, h / G],  out = sum_p e^(x_p - lse) v[p, h / G],
//   lse = log sum_p e^x_p;  nothing seen: out 0, lse -inf.
//
// One pass over the keys with a running reference and sum. The work of all sequences is cut
// into equal parts, one a block, and the partial results joined. Few rows a sequence are
// bound by memory (64 x 1 rows of 16 heads on 2 behind 4096 positions, bf16: 46.9 + 6.0 us,
// 4.3 TB/s); many by the turns that eight waves pass together at a key tile's barrier,
// products, softmax, products (660 TFLOP/s in full tiles; 16 x 48 rows of 40 heads on 8
// behind 16384, f16: 268 + 16 us).
#pragma once

#include <algorithm>
#include <type_traits>

#include "common.h"

namespace vsr {

// A join of partial results: those of item (b, n, kvh, tile) from blocks first .. last
// (last < 0: none).
struct TreeJoin {
  int b, n, kvh, tile, step, last;
};

hipError_t launch_tree_f32(const TreeAttnArgs &a, void *ws, hipStream_t s);
hipError_t launch_tree_bf16(const TreeAttnArgs &a, void *ws, hipStream_t s);
hipError_t launch_tree_f16(const TreeAttnArgs &a, void *ws, hipStream_t s);

namespace {

__device__ __forceinline__ int seq_held(const PageTables &p, int s) {
  return max(0, min(p.held[s], p.max_pages));
}
// Positions that sequence s's pages have room for.
__device__ __forceinline__ int seq_room(const PageTables &p, int s) {
  return (int)min((long)seq_held(p, s) << p.page_shift, (long)INT32_MAX);
}
__device__ __forceinline__ int seq_len(const PageTables &p, int s) {
  return max(0, min(p.len[s], seq_room(p, s)));
}
// Rows [b, e) of sequence s among T.
__device__ __forceinline__ void seq_rows(const int32_t *start, int T, int s, int &b, int &e) {
  b = start ? max(0, min(start[s], T)) : min(s, T);
  e = start ? max(b, min(start[s + 1], T)) : min(s + 1, T);
}

// ---------------------------------------------------------------- attention

__device__ const u32x4 g_zeros = {0, 0, 0, 0};

template <typename T>
struct Mat;  // a type's matrix products, 16 keys (rows) by 16 queries (columns)
template <>
struct Mat<bf16> {
  typedef bf16x8 x8;
  typedef bf16x4 x4;
  static __device__ __forceinline__ f32x4 mul(x8 a, x8 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
  }
  static __device__ __forceinline__ f32x4 mul(x4 a, x4 b, f32x4 c) {
    typedef short s16x4 __attribute__((ext_vector_type(4)));
    return __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(__builtin_bit_cast(s16x4, a),
                                                     __builtin_bit_cast(s16x4, b), c, 0, 0, 0);
  }
};
template <>
struct Mat<f16> {
  typedef f16x8 x8;
  typedef f16x4 x4;
  static __device__ __forceinline__ f32x4 mul(x8 a, x8 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
  }
  static __device__ __forceinline__ f32x4 mul(x4 a, x4 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x16f16(a, b, c, 0, 0, 0);
  }
};
template <>
struct Mat<float> {
  static __device__ __forceinline__ f32x4 mul(float a, float b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0);
  }
};

constexpr int kAllLoads = 0x0f70;  // s_waitcnt's word for "no load is on its way"

// Shape of a block: NW waves, WM along the rows (each RT tiles of 16) and WK along the
// keys of a tile of BK; LDS rows of CH 16-byte chunks.
template <typename T_, int HD_, int NW_, int RT_, int WM_>
struct TreeShape {
  typedef T_ T;
  static constexpr int HD = HD_, NW = NW_, RT = RT_, WM = WM_, WK = NW / WM;
  static constexpr int NT = NW * 64;
  static constexpr bool F32 = sizeof(T) == 4;
  static constexpr int BK = F32 && HD == 256 ? 32 : 64;
  static constexpr int BM = WM * RT * 16;
  static constexpr int KW = BK / 16 / WK;    // 16-key tiles of a wave
  static constexpr int EC = 16 / sizeof(T);  // elements a chunk
  static constexpr int CH = HD / EC;
  // Threads that load: of eight waves the last four, which have fewer rows if any do. While
  // these wait for the load unit (32 loads of 1 KB a tile: 1250 cycles of 4900), the other
  // wave of their SIMD has it to itself. (All eight: 2 % slower.)
  static constexpr int LT = NW == 8 ? NT / 2 : NT;
  static constexpr int NL = BK * CH / LT;    // chunks of K each of them loads
  static constexpr int TILE = BK * CH;       // chunks of a K or V tile
  // Blocks a CU: by LDS, and two waves a SIMD.
  static constexpr int PER_CU = NW == 4 && 4 * TILE * 16 <= 72 << 10 ? 2 : 1;
  // Probabilities are held 2^LIFT times as large: at most 2^(8 + LIFT), which fits an fp16,
  // whose smallest numbers then reach 2^-31 of the likeliest key and full digits 2^-21. (At
  // 2^0 a key below 2^-25 counted for nothing, and long contexts behind one strong key
  // lost all their other keys.)
  static constexpr float LIFT = std::is_same<T, f16>::value ? 7.f : 0.f;
  static constexpr float DROP = LIFT > 0.f ? 0x1p-7f : 1.f;  // 2^-LIFT
  static_assert(KW >= 1 && NL >= 1, "each wave has keys, each thread a load");
  static_assert(NW * 16 * HD * 4 <= 4 * TILE * 16, "a row group of each wave fits the ring");
};

// LDS gives 256 bytes to 16 lanes at once: chunk c of row r lies where 16 rows' chunks
// c fall on different banks.
template <int CH>
__device__ __forceinline__ int swz(int r) {
  return CH >= 16 ? r & 15 : (r >> 1) & 7;
}

// The walk of all blocks over all work. An item is (sequence, key head, tile of rows),
// tiles innermost, the sequence's rows shared evenly by its tiles, a tile's 16-row groups
// by the waves. Its key tiles cost 6 + the row groups that take them: 16 x 48 rows behind
// 16384 positions took 284 us so and at 9 +, 286 at 4 +, 290 at 2 +, 294 with the groups
// rounded up to four. Block g takes the key tiles that begin in [g per, (g + 1) per) of
// the summed costs.
struct Work {
  int s, b, n;      // a sequence and its rows
  int len, keys;    // positions before the draft, and with it
  int tiles, step;  // row tiles, rows of each
  int nb, cost;     // key tiles of an item, cost of each
  long base;        // cost of the items before the sequence's
};

template <class S>
__device__ __forceinline__ void work_of(const TreeAttnArgs &a, int s, Work &w) {
  int e;
  seq_rows(a.start, a.T, s, w.b, e);
  w.s = s;
  w.n = e - w.b;
  w.len = seq_len(a.pages, s);
  w.keys = min(w.len + w.n, seq_room(a.pages, s));
  const int rows = w.n * a.group;
  w.tiles = (rows + S::BM - 1) / S::BM;
  // (The least multiple of 16 that `tiles` of cover the rows.)
  w.step = w.tiles <= 1 ? max(16, (rows + 15) / 16 * 16)
                        : ((rows + w.tiles - 1) / w.tiles + 15) / 16 * 16;
  w.nb = max(1, (w.keys + S::BK - 1) / S::BK);
  w.cost = 6 + w.step / 16 * S::WK;
}

__device__ __forceinline__ long work_cost(const TreeAttnArgs &a, const Work &w) {
  return (long)a.n_kv * w.tiles * (w.nb * w.cost);
}

// What a block takes of a call's cost. It passes 2^31 where a chain of 2^22 rows of 64 heads
// meets all its keys.
__host__ __device__ __forceinline__ long share_of(long total, int blocks) {
  return std::max(1L, (total + blocks - 1) / blocks);
}

// a / b, 0 <= a < 2^57, 0 < b < 2^31, where that is below 2^31: by a reciprocal put right (a
// 64-bit division is 1 KB of code, and a kernel's steps from item to item wait for their
// code as well).
__device__ __forceinline__ int quotient(long a, int b) {
  long q = (long)((double)a * __builtin_amdgcn_rcp((double)b));
  long r = a - q * b;
  while (r < 0) {
    --q;
    r += b;
  }
  while (r >= b) {
    ++q;
    r -= b;
  }
  return (int)q;
}
// r / group.
__device__ __forceinline__ int token_of(const TreeAttnArgs &a, int r) {
  return (int)(((uint64_t)(uint32_t)r * a.group_mul) >> a.group_shift);
}

// Exclusive prefix sum over a block's NT threads, and the total.
template <int NT>
__device__ __forceinline__ long block_scan(long mine, long *sums, long &total) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  long v = mine;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const long o = __shfl_up(v, d);
    if (lane >= d) v += o;
  }
  if (lane == 63) sums[w] = v;
  __syncthreads();
  long before = 0;
  total = 0;
#pragma unroll
  for (int i = 0; i < NT / 64; ++i) {
    if (i < w) before += sums[i];
    total += sums[i];
  }
  __syncthreads();
  return before + v - mine;
}

__device__ __forceinline__ long lane_value(long v, int lane) {
  const uint32_t lo = __builtin_amdgcn_readlane((int)v, lane);
  const uint32_t hi = __builtin_amdgcn_readlane((int)(v >> 32), lane);
  return (long)((uint64_t)hi << 32 | lo);
}

// Inclusive prefix sum over the lanes of a wave (wave_scan's steps).
template <int CTRL, int ROWS>
__device__ __forceinline__ long scan_step(long v) {
  const uint32_t lo = __builtin_amdgcn_update_dpp(0, (int)v, CTRL, ROWS, 0xF, false);
  const uint32_t hi = __builtin_amdgcn_update_dpp(0, (int)(v >> 32), CTRL, ROWS, 0xF, false);
  return v + (long)((uint64_t)hi << 32 | lo);
}
__device__ __forceinline__ long wave_scan_long(long v) {
  v = scan_step<0x111, 0xF>(v);
  v = scan_step<0x112, 0xF>(v);
  v = scan_step<0x114, 0xF>(v);
  v = scan_step<0x118, 0xF>(v);
  v = scan_step<0x142, 0xA>(v);
  return scan_step<0x143, 0xC>(v);
}

// The sequences' costs in order. Up to 64 sequences every wave holds them all, one a lane;
// more are held by the block, runs of them a thread, and read again where they are needed.
template <class S>
struct Plan {
  Work mine;   // a lane's sequence
  long cost, upto;
  long total, first;
  bool few;

  __device__ __forceinline__ Plan(const TreeAttnArgs &a, long *sums) {
    few = a.pages.n_seqs <= 64;
    if (few) {
      const int lane = threadIdx.x & 63;
      cost = 0;
      if (lane < a.pages.n_seqs) {
        work_of<S>(a, lane, mine);
        cost = work_cost(a, mine);
      }
      upto = wave_scan_long(cost);
      total = lane_value(upto, 63);
    } else {
      const int per = (a.pages.n_seqs + S::NT - 1) / S::NT;
      cost = 0;
      for (int i = 0; i < per; ++i) {
        const int s = threadIdx.x * per + i;
        if (s >= a.pages.n_seqs) break;
        work_of<S>(a, s, mine);
        cost += work_cost(a, mine);
      }
      first = block_scan<S::NT>(cost, sums, total);
      total = lane_value(total, 0);
    }
  }

  // The sequence in whose cost `at` lies.
  __device__ __forceinline__ void find(const TreeAttnArgs &a, long at, long *found, Work &w) {
    if (few) {
      const int s = __builtin_ctzll(__ballot(at < upto && at >= upto - cost));
      const auto of = [&](int v) { return __builtin_amdgcn_readlane(v, s); };
      w = {s, of(mine.b), of(mine.n), of(mine.len), of(mine.keys), of(mine.tiles), of(mine.step),
           of(mine.nb), of(mine.cost), lane_value(upto - cost, s)};
      return;
    }
    const int per = (a.pages.n_seqs + S::NT - 1) / S::NT;
    const int s0 = threadIdx.x * per;
    long base = first;
    if (at >= first && at < first + cost) {
      for (int i = 0; i < per && s0 + i < a.pages.n_seqs; ++i) {
        Work x;
        work_of<S>(a, s0 + i, x);
        const long u = work_cost(a, x);
        if (at >= base && at < base + u) {
          found[0] = s0 + i;
          found[1] = base;
        }
        base += u;
      }
    }
    __syncthreads();
    const int s = __builtin_amdgcn_readfirstlane((int)found[0]);
    work_of<S>(a, s, w);
    w.base = lane_value(found[1], 0);
    __syncthreads();
  }

  // From a sequence's end, `at`, to the next that has rows.
  __device__ __forceinline__ void next(const TreeAttnArgs &a, long at, Work &w) {
    if (few) {
      find(a, at, nullptr, w);
      return;
    }
    while (at >= w.base + work_cost(a, w)) {
      const long base = w.base + work_cost(a, w);
      work_of<S>(a, w.s + 1, w);
      w.base = base;
    }
  }
};

// A block takes two of the dearest key tiles at least (one that lies between an item's
// first and last block then has one of its tiles).
template <class S>
__device__ __forceinline__ int blocks_used(long total, int groups) {
  constexpr int least = 2 * (6 + S::RT * S::NW);
  return (int)max(1L, min(total / least, (long)groups));
}
// Blocks of one XCD take neighbouring ranges (tiles that share keys), unless there are
// fewer of them than the grid has.
__device__ __forceinline__ int logical_block(int b, int eff, int groups) {
  return eff < groups ? b : b % 8 * (groups / 8) + b / 8;
}

__device__ __forceinline__ float over_groups_max(float x) {
  auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
  r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float over_groups_sum(float x) {
  auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = __uint_as_float(r[0]) + __uint_as_float(r[1]);
  r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// A lane's rows: query column lane % 16 of each of RT tiles.
template <class S>
struct Rows {
  static constexpr int QN = S::F32 ? S::HD / 4 : S::HD / 32;
  typedef typename std::conditional<S::F32, float, u32x4>::type Q;
  Q q[S::RT][QN];
  int j[S::RT];         // row of the draft
  float m[S::RT], l[S::RT];
  int n;                // of the wave's row groups, those that have rows
  f32x4 o[S::RT][S::HD / 16];
};

template <typename T>
__device__ __forceinline__ T load_part(const T *p, int i, int hd) {
  return i < hd ? p[i] : T(0.f);
}

// Row groups of 16 of the item's `rows` that wave wm of S::WM has: n of them from first on.
struct Groups {
  int first, n;
};
template <class S>
__device__ __forceinline__ Groups groups_of(int rows, int wm) {
  const int all = (rows + 15) / 16, each = all / S::WM, more = all % S::WM;
  return {wm * each + min(wm, more), each + (wm < more)};
}

__device__ __forceinline__ int item_rows(const TreeAttnArgs &a, const Work &w, int tile) {
  return min(w.step, w.n * a.group - tile * w.step);
}

template <class S>
__device__ __forceinline__ void load_rows(const TreeAttnArgs &a, const Work &w, int kvh, int tile,
                                          Rows<S> &R) {
  typedef typename S::T T;
  constexpr int V = 16 / sizeof(T);  // elements a load
  typedef Pack<T, V> P;
  const int lane = threadIdx.x & 63, g4 = lane >> 4, wm = (threadIdx.x >> 6) % S::WM;
  const int rows = item_rows(a, w, tile);
  const Groups mine = groups_of<S>(rows, wm);
  R.n = __builtin_amdgcn_readfirstlane(mine.n);
#pragma unroll
  for (int rt = 0; rt < S::RT; ++rt) {
    const int r = (mine.first + rt) * 16 + (lane & 15);
    const int rc = tile * w.step + (rt < mine.n && r < rows ? r : 0);
    R.j[rt] = token_of(a, rc);
    R.m[rt] = -INFINITY;
    R.l[rt] = 0.f;
    const T *q = static_cast<const T *>(a.q) + (w.b + R.j[rt]) * a.q_ts +
                 (long)(kvh * a.group + rc - R.j[rt] * a.group) * a.q_hs;
    P x[S::CH / 4];
    if (a.hd == S::HD) {
#pragma unroll
      for (int c = 0; c < S::CH / 4; ++c)
        x[c] = *reinterpret_cast<const P *>(q + (4 * c + g4) * V);
    } else {
#pragma unroll
      for (int c = 0; c < S::CH / 4; ++c)
#pragma unroll
        for (int i = 0; i < V; ++i) x[c].v[i] = load_part(q, (4 * c + g4) * V + i, a.hd);
    }
#pragma unroll
    for (int c = 0; c < S::CH / 4; ++c) {
      u32x4 bits = __builtin_bit_cast(u32x4, x[c]);
      if (a.negate) bits ^= S::F32 ? 0x80000000u : 0x80008000u;
      if constexpr (S::F32) {
#pragma unroll
        for (int i = 0; i < 4; ++i) R.q[rt][c * 4 + i] = __uint_as_float(bits[i]);
      } else {
        R.q[rt][c] = bits;
      }
    }
#pragma unroll
    for (int d = 0; d < S::HD / 16; ++d) R.o[rt][d] = f32x4{};
  }
}

// The thread's number, of which the compiler knows nothing: what follows from it is worked
// out again for each tile. Kept in registers over the loops it was spilled, and the
// reloads stood ahead of the loads.
__device__ __forceinline__ int thread_again() {
  int tid = threadIdx.x;
  asm volatile("" : "+v"(tid));
  return tid;
}

// Pages of the keys that a thread loads, of the tile at kb (past the keys: the last one's).
template <class S>
__device__ __forceinline__ void load_pages(const TreeAttnArgs &a, const Work &w, int kb,
                                           int32_t *page) {
  const int32_t *table = a.pages.table + w.s * a.pages.table_stride;
  const int tid = thread_again() - (S::NT - S::LT);
#pragma unroll
  for (int i = 0; i < S::NL; ++i) {
    const int p = kb + i * (S::LT / S::CH) + tid / S::CH;
    page[i] = table[min(p, w.keys - 1) >> a.pages.page_shift];
  }
}

// Chunk of the row that a thread's load i brings (it lands in chunk tid % CH of the row).
template <class S>
__device__ __forceinline__ int load_chunk(int tid, int i) {
  constexpr int STEP = S::LT / S::CH;  // rows from load to load
  const int c = (tid % S::CH) ^ swz<S::CH>(tid / S::CH);
  return S::CH >= 16 ? c ^ (i * STEP & 15) : c;
}

// Key tile kb of both matrices on its way into an LDS stage: rows past the sequence's
// keys and columns past hd are zeros. VEC: 16-byte loads straight into LDS (strides below
// 2^32 bytes); else through registers.
template <class S, bool VEC>
__device__ __forceinline__ void load_tile(const TreeAttnArgs &a, const Work &w, int kvh, int kb,
                                          const int32_t *page, u32x4 *stage) {
  typedef typename S::T T;
  const int tid = thread_again() - (S::NT - S::LT), wave = tid & ~63, shift = a.pages.page_shift;
  const T *k = static_cast<const T *>(a.k) + kvh * a.k_hs;
  const T *v = static_cast<const T *>(a.v) + kvh * a.v_hs;
  const bool all = kb + S::BK <= w.keys && a.hd == S::HD;
  if (VEC && all) {
    // (Without the checks below: 268 us against 274, 16 x 48 rows behind 16384 positions.)
    const uint32_t kt = (uint32_t)(a.k_ts * sizeof(T)), vt = (uint32_t)(a.v_ts * sizeof(T));
    const int c0 = load_chunk<S>(tid, 0) * 16, p0 = kb + tid / S::CH;
    u32x4 *to = stage + __builtin_amdgcn_readfirstlane(wave);
#pragma unroll
    for (int i = 0; i < S::NL; ++i) {
      const uint32_t pg = (uint32_t)page[i] < (uint32_t)a.pages.n_pages ? page[i] : 0;
      const uint32_t p = p0 + i * (S::LT / S::CH), slot = pg << shift | (p & ((1u << shift) - 1));
      const int c = S::CH >= 16 && S::LT / S::CH < 16 ? load_chunk<S>(tid, i) * 16 : c0;
      __builtin_amdgcn_global_load_lds(reinterpret_cast<const char *>(k) + c + (uint64_t)slot * kt,
                                       to + i * S::LT, 16, 0, 0);
      __builtin_amdgcn_global_load_lds(reinterpret_cast<const char *>(v) + c + (uint64_t)slot * vt,
                                       to + i * S::LT + S::TILE, 16, 0, 0);
    }
    return;
  }
#pragma unroll
  for (int i = 0; i < S::NL; ++i) {
    const int r = i * (S::LT / S::CH) + tid / S::CH, p = kb + r, c = load_chunk<S>(tid, i);
    const uint32_t pg = (uint32_t)page[i] < (uint32_t)a.pages.n_pages ? page[i] : 0;
    const uint32_t slot = pg << shift | ((uint32_t)p & ((1u << shift) - 1));
    if constexpr (VEC) {
      const uint32_t kt = (uint32_t)(a.k_ts * sizeof(T)), vt = (uint32_t)(a.v_ts * sizeof(T));
      const char *kp = reinterpret_cast<const char *>(k) + c * 16 + (uint64_t)slot * kt;
      const char *vp = reinterpret_cast<const char *>(v) + c * 16 + (uint64_t)slot * vt;
      if (p >= w.keys || c * S::EC >= a.hd)
        kp = vp = reinterpret_cast<const char *>(&g_zeros);
      u32x4 *to = stage + i * S::LT + __builtin_amdgcn_readfirstlane(wave);
      __builtin_amdgcn_global_load_lds(kp, to, 16, 0, 0);
      __builtin_amdgcn_global_load_lds(vp, to + S::TILE, 16, 0, 0);
    } else {
      const int at = i * S::LT + tid;
      const T *kp = k + slot * a.k_ts + c * S::EC, *vp = v + slot * a.v_ts + c * S::EC;
      const bool real = p < w.keys && c * S::EC < a.hd;
      Pack<T, S::EC> x{}, y{};
      if (real && (c + 1) * S::EC <= a.hd) {
        x = *reinterpret_cast<const Pack<T, S::EC> *>(kp);
        y = *reinterpret_cast<const Pack<T, S::EC> *>(vp);
      } else if (real) {
#pragma unroll
        for (int e = 0; e < S::EC; ++e) {
          x.v[e] = load_part(kp, e, a.hd - c * S::EC);
          y.v[e] = load_part(vp, e, a.hd - c * S::EC);
        }
      }
      stage[at] = __builtin_bit_cast(u32x4, x);
      stage[S::TILE + at] = __builtin_bit_cast(u32x4, y);
    }
  }
}

// Byte offsets in a tile of what a lane reads of its first 16 keys, for chunk 0 (keys) and
// column tile 0 (values). Others differ by an exclusive or (a swizzled row's chunks c and
// c0 ^ c) and by whole rows. The compiler is kept from working them out ahead of the
// loops: it took a register for each, spilled them, and waited for the reloads.
template <class S>
__device__ __forceinline__ int key_offset() {
  const int l = threadIdx.x & 15, g4 = (threadIdx.x & 63) >> 4;
  int at = l * S::CH * 16 + ((g4 ^ swz<S::CH>(l)) << 4);
  asm volatile("" : "+v"(at));
  return at;
}
template <class S>
__device__ __forceinline__ int value_offset() {
  const int l = threadIdx.x & 15, g4 = (threadIdx.x & 63) >> 4;
  int at;
  if constexpr (S::F32) {
    at = 4 * g4 * S::CH * 16 + ((l >> 2 ^ swz<S::CH>(4 * g4)) << 4) + (l & 3) * 4;
  } else {
    const int r = 4 * g4 + (l >> 2);
    at = r * S::CH * 16 + (((l & 3) >> 1 ^ swz<S::CH>(r)) << 4) + (l & 1) * 8;
  }
  asm volatile("" : "+v"(at));
  return at;
}

// Four V elements of column d 16 + lane % 16, keys 4 (lane / 16) .. + 3 of the 16 from
// row k0 on: a transposing read of four rows by 16 lanes.
template <class S>
__device__ __forceinline__ typename Mat<typename S::T>::x4 v_frag(const u32x4 *vs, int at, int k0,
                                                                  int d) {
  typedef short s16x4 __attribute__((ext_vector_type(4)));
  const char *p = reinterpret_cast<const char *>(vs) + (at ^ d * 32) + k0 * S::CH * 16;
  return __builtin_bit_cast(
      typename Mat<typename S::T>::x4,
      __builtin_amdgcn_ds_read_tr16_b64_v4i16(
          (__attribute__((address_space(3))) s16x4 *)const_cast<char *>(p)));
}

// The V operands of VG columns of 16 from column tile d0 on, for a wave's keys.
template <class S, int VG>
struct VFrag {
  typename Mat<typename S::T>::x4 v[VG][S::KW];
  __device__ __forceinline__ void read(const u32x4 *vs, int at, int key0, int d0) {
#pragma unroll
    for (int n = 0; n < VG; ++n)
#pragma unroll
      for (int t = 0; t < S::KW; ++t) v[n][t] = v_frag<S>(vs, at, key0 + t * 16, d0 + n);
  }
};

template <typename T>
__device__ __forceinline__ bool not_finite(T x) {
  return !(__builtin_fabsf(to_f32(x)) < INFINITY);
}

// Values that are no numbers, in the rows of a draft, must reach the rows that see them and
// no others, but 0 times them is no number either. They are set to 0 in the tile here
// (returns whether a thread met one; the tile's first rows are context), and put where they
// belong when the rows are stored (odd_values).
template <class S>
__device__ __forceinline__ bool clear_odd(u32x4 *vs, int context) {
  typedef typename S::T T;
  // (An exponent of ones carries into the sign's place.)
  constexpr uint32_t MASK = S::F32 ? 0x7f800000u : std::is_same<T, bf16>::value ? 0x7f807f80u : 0x7c007c00u;
  constexpr uint32_t ONE = S::F32 ? 0x00800000u : std::is_same<T, bf16>::value ? 0x00800080u : 0x04000400u;
  constexpr uint32_t TOP = S::F32 ? 0x80000000u : 0x80008000u;
  uint32_t any = 0;
#pragma unroll
  for (int i = 0; i < S::BK * S::CH / S::NT; ++i) {
    const int n = i * S::NT + threadIdx.x;
    const u32x4 x = vs[n];
    uint32_t odd = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) odd |= ((x[e] & MASK) + ONE) & TOP;
    any |= n / S::CH < context ? 0 : odd;
  }
  if (!__any(any != 0)) return false;
#pragma unroll 1
  for (int i = 0; i < S::BK * S::CH / S::NT; ++i) {
    const int n = i * S::NT + threadIdx.x;
    if (n / S::CH < context) continue;
    Pack<T, S::EC> x = __builtin_bit_cast(Pack<T, S::EC>, vs[n]);
#pragma unroll
    for (int e = 0; e < S::EC; ++e)
      if (not_finite(x.v[e])) x.v[e] = from_f32<T>(0.f);
    vs[n] = __builtin_bit_cast(u32x4, x);
  }
  return any != 0;
}

// Keeps the compiler from moving anything across: groups of LDS reads stay a group of
// products ahead of their use (left to itself it puts each read right before its
// product, and a tile waits for 28 of them).
__device__ __forceinline__ void in_order() { __builtin_amdgcn_sched_barrier(0); }

// Bit 4 t + i: whether row j of the draft sees position p0 + 16 t + i, t < KW, i < 4.
template <class S>
__device__ __forceinline__ uint32_t seen_bits(const TreeAttnArgs &a, const Work &w, int j, int p0) {
  uint32_t seen = 0;
  const uint32_t *row = a.mask ? a.mask + (w.b + j) * a.mask_stride : nullptr;
#pragma unroll
  for (int t = 0; t < S::KW; ++t) {
    const int p = p0 + 16 * t, d = p - w.len;  // (d < 0: the context)
    uint32_t bits;
    if (row) {
      // Bits d .. d + 3 of the row's mask; past its words they are clear.
      const int wd = max(d, 0) >> 5;
      uint64_t v = wd < a.mask_words && p < w.keys ? row[wd] : 0;
      if (wd + 1 < a.mask_words && p < w.keys) v |= (uint64_t)row[wd + 1] << 32;
      bits = d >= 0 ? (uint32_t)(v >> (d & 31)) : d > -4 ? (uint32_t)(v << -d) : 0;
    } else {
      const int n = j - d + 1;  // positions d .. j
      bits = n >= 4 ? 15 : n > 0 ? (1u << n) - 1 : 0;
    }
    const int room = w.keys - p;
    if (room < 4) bits &= room > 0 ? (1u << room) - 1 : 0;
    if (d < 0) bits |= d > -4 ? (1u << -d) - 1 : 15;
    seen |= (bits & 15) << (4 * t);
  }
  return seen;
}

// One key tile against NR groups of a wave's rows. DRAFT: the tile has keys that not all
// rows see.
template <class S, bool DRAFT, int NR>
__device__ __forceinline__ void tile_step(const TreeAttnArgs &a, const Work &w, int kb,
                                          const u32x4 *st, Rows<S> &R) {
  typedef typename S::T T;
  typedef Mat<T> M;
  const int lane = threadIdx.x & 63, g4 = lane >> 4, wk = (threadIdx.x >> 6) / S::WM;
  const u32x4 *ks = st, *vs = st + S::TILE;
  const int key0 = wk * S::KW * 16;
  // What a lane's rows see of its keys, bit 4 t + i (worked out before the products, which
  // need the registers).
  [[maybe_unused]] uint32_t seen[NR];
  if constexpr (DRAFT) {
#pragma unroll
    for (int rt = 0; rt < NR; ++rt) {
      in_order();
      seen[rt] = seen_bits<S>(a, w, R.j[rt], kb + key0 + 4 * g4);
    }
    in_order();
  }
  f32x4 x[NR][S::KW];
  constexpr int KC = S::CH / 4;  // 16-byte chunks a lane reads of a key tile
  const int k_at = key_offset<S>(), v_at = value_offset<S>();
  const auto read_keys = [&](int t, u32x4 *kf) {
    const char *p = reinterpret_cast<const char *>(ks) + (key0 + t * 16) * S::CH * 16;
#pragma unroll
    for (int c = 0; c < KC; ++c) kf[c] = *reinterpret_cast<const u32x4 *>(p + (k_at ^ c * 64));
  };
  u32x4 kf[2][KC];
  read_keys(0, kf[0]);
#pragma unroll
  for (int t = 0; t < S::KW; ++t) {
    in_order();
    if (t + 1 < S::KW) read_keys(t + 1, kf[(t + 1) & 1]);
    in_order();
#pragma unroll
    for (int rt = 0; rt < NR; ++rt) x[rt][t] = f32x4{};
#pragma unroll
    for (int c = 0; c < KC; ++c)
#pragma unroll
      for (int rt = 0; rt < NR; ++rt) {
        if constexpr (S::F32) {
          const f32x4 kv = __builtin_bit_cast(f32x4, kf[t & 1][c]);
#pragma unroll
          for (int i = 0; i < 4; ++i) x[rt][t] = M::mul(kv[i], R.q[rt][c * 4 + i], x[rt][t]);
        } else {
          x[rt][t] = M::mul(__builtin_bit_cast(typename M::x8, kf[t & 1][c]),
                            __builtin_bit_cast(typename M::x8, R.q[rt][c]), x[rt][t]);
        }
      }
  }
  in_order();
  // The first values are on their way during the softmax.
  constexpr int VG = S::F32 ? 1 : 2;  // columns of 16 a group of value reads
  struct None {};
  typename std::conditional<S::F32, None, VFrag<S, VG>>::type vf[2];
  if constexpr (!S::F32) vf[0].read(vs, v_at, key0, 0);
  if constexpr (DRAFT) {
#pragma unroll
    for (int rt = 0; rt < NR; ++rt)
#pragma unroll
      for (int t = 0; t < S::KW; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          x[rt][t][i] = seen[rt] >> (4 * t + i) & 1 ? x[rt][t][i] : -INFINITY;
  }
  const float c = a.scale_log2;
#pragma unroll
  for (int rt = 0; rt < NR; ++rt) {
    float top = -INFINITY;
#pragma unroll
    for (int t = 0; t < S::KW; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) top = fmaxf(top, x[rt][t][i]);
    top = over_groups_max(top) * c;
    // The reference of the exponents moves only where a score passes it by 2^8. (A difference:
    // 8 above a reference past 2^27 is rounded to 16, and fp16's probabilities overflowed.)
    if (__any(top - R.m[rt] > 8.f)) {
      const float m = fmaxf(R.m[rt], top);
      const float f = m == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(R.m[rt] - m);
      R.m[rt] = m;
      R.l[rt] *= f;
#pragma unroll
      for (int d = 0; d < S::HD / 16; ++d) R.o[rt][d] *= f;
    }
    const float ref = R.m[rt] == -INFINITY ? 0.f : R.m[rt];
    // One fused step a score; where references are so large that their own rounding would
    // show, scores are rounded like them first.
    const bool large = __any(fabsf(ref) > 65536.f);
    if (large) {
#pragma clang fp contract(off)
#pragma unroll
      for (int t = 0; t < S::KW; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float y = x[rt][t][i] * c;
          x[rt][t][i] = (y - ref) + S::LIFT;
        }
      asm volatile("");  // (or the products are taken out of the branch)
    } else {
      const float low = ref - S::LIFT;
#pragma unroll
      for (int t = 0; t < S::KW; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) x[rt][t][i] = __builtin_fmaf(x[rt][t][i], c, -low);
    }
    // (The sum is of probabilities before their rounding to 16 bits: of the rounded ones, lse
    // was off by 7e-4 in bf16.)
    float sum = 0.f;
#pragma unroll
    for (int t = 0; t < S::KW; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float p = __builtin_amdgcn_exp2f(x[rt][t][i]);
        x[rt][t][i] = p;
        sum += p;
      }
    R.l[rt] += sum;
  }
  if constexpr (S::F32) {
#pragma unroll
    for (int t = 0; t < S::KW; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const char *row = reinterpret_cast<const char *>(vs) + (key0 + t * 16 + i) * S::CH * 16;
#pragma unroll
        for (int d = 0; d < S::HD / 16; ++d) {
          const float v = *reinterpret_cast<const float *>(row + (v_at ^ (d * 64 ^ i * 16)));
#pragma unroll
          for (int rt = 0; rt < NR; ++rt) R.o[rt][d] = M::mul(v, x[rt][t][i], R.o[rt][d]);
        }
      }
  } else {
    typedef typename M::x4 x4;
    typedef typename M::x8 x8;
    // Rounded to the values' type, as the matrix units take them: results are 2.3e-3 off for
    // bf16, where their own rounding alone makes 1.7e-3, 2.9e-4 and 2.1e-4 for fp16. (A second
    // product with what the rounding leaves would double the work with values.)
    x4 p[NR][S::KW];
#pragma unroll
    for (int rt = 0; rt < NR; ++rt)
#pragma unroll
      for (int t = 0; t < S::KW; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) p[rt][t][i] = from_f32<T>(x[rt][t][i]);
    constexpr int NG = S::HD / 16 / VG;
#pragma unroll
    for (int g = 0; g < NG; ++g) {
      in_order();
      if (g + 1 < NG) vf[(g + 1) & 1].read(vs, v_at, key0, (g + 1) * VG);
      in_order();
#pragma unroll
      for (int n = 0; n < VG; ++n) {
        const x4 *v = vf[g & 1].v[n];
        const int d = g * VG + n;
#pragma unroll
        for (int t = 0; t < S::KW; t += 2)
#pragma unroll
          for (int rt = 0; rt < NR; ++rt) {
            if constexpr (S::KW == 1) {
              R.o[rt][d] = M::mul(v[0], p[rt][0], R.o[rt][d]);
            } else {
              // The 32 keys of two tiles: a lane's first four k are tile t's, the others
              // t + 1's, in both operands.
              const x8 vv = __builtin_shufflevector(v[t], v[t + 1], 0, 1, 2, 3, 4, 5, 6, 7);
              const x8 pp = __builtin_shufflevector(p[rt][t], p[rt][t + 1], 0, 1, 2, 3, 4, 5, 6, 7);
              R.o[rt][d] = M::mul(vv, pp, R.o[rt][d]);
            }
          }
      }
    }
  }
}

// Whether row j sees position len + d of its draft.
__device__ __forceinline__ bool sees(const TreeAttnArgs &a, const Work &w, int j, int d) {
  if (!a.mask) return d <= j;
  return d >> 5 < a.mask_words &&
         (a.mask[(w.b + j) * a.mask_stride + (d >> 5)] >> (d & 31) & 1);
}

// What row j sees of values that are no numbers, in columns 4 c .. + 3 of the draft's
// positions from <= position < to.
template <class S>
__device__ __forceinline__ f32x4 odd_values(const TreeAttnArgs &a, const Work &w, int kvh, int j,
                                         int c, int from, int to) {
  typedef typename S::T T;
  f32x4 y{};
#pragma unroll 1
  for (int p = max(from, w.len); p < to; ++p) {
    if (!sees(a, w, j, p - w.len)) continue;
    int page = a.pages.table[w.s * a.pages.table_stride + (p >> a.pages.page_shift)];
    if ((uint32_t)page >= (uint32_t)a.pages.n_pages) page = 0;
    const long slot = ((long)page << a.pages.page_shift) | (p & ((1 << a.pages.page_shift) - 1));
    const T *v = static_cast<const T *>(a.v) + kvh * a.v_hs + slot * a.v_ts + 4 * c;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float f = 4 * c + e < a.hd ? to_f32(v[e]) : 0.f;
      y[e] += not_finite(f) ? f : 0.f;
    }
  }
  return y;
}

// Columns 4 c .. + 3 of a row of the item: its sum y over a sum of probabilities l, scores
// relative to `top`; into out and lse, or (which >= 0) partial result `which`.
template <class S>
__device__ __forceinline__ void put_row(const TreeAttnArgs &a, const Work &w, int kvh, int tile,
                                        int r, int c, f32x4 y, float l, float top, long which) {
  typedef typename S::T T;
  if (which >= 0) {
    reinterpret_cast<f32x4 *>(a.part)[(which * S::BM + r) * (S::HD / 4) + c] = y;
    if (c == 0) a.part_ml[which * S::BM + r] = make_float2(top, l);
    return;
  }
  const int gr = tile * w.step + r, j = token_of(a, gr), h = kvh * a.group + gr - j * a.group;
  // (A row that saw nothing has l = 0 and y = 0; NaN stays.)
  const float inv = l == 0.f ? 1.f : 1.f / l;
  T *out = static_cast<T *>(a.out) + (w.b + j) * a.o_ts + h * a.o_hs + 4 * c;
  Pack<T, 4> t;
#pragma unroll
  for (int e = 0; e < 4; ++e) t.v[e] = from_f32<T>(y[e] * inv);
  if (4 * c + 4 <= a.hd) {
    *reinterpret_cast<Pack<T, 4> *>(out) = t;
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (4 * c + e < a.hd) out[e] = t.v[e];
  }
  if (c == 0 && a.lse)
    a.lse[(long)(w.b + j) * a.n_heads + h] =
        l == 0.f ? -INFINITY
                 : (top + __builtin_log2f(l * S::DROP)) * 0.69314718055994531f;
}

// An item's rows stored (put_row), a group of each wave after the other, through the ring's
// two stages: there the waves along the keys join their shares, and a loop stores whole
// rows (unrolled from registers, the stores were 60 KB of code, met once a block).
template <class S>
__device__ __forceinline__ void store_rows(const TreeAttnArgs &a, const Work &w, int kvh, int tile,
                                           Rows<S> &R, u32x4 *lds0, u32x4 *lds1, float2 *ml,
                                           long which, const int *met_odd, int from, int to) {
  constexpr int CF = S::HD / 4, LR = S::WM * 16;  // float chunks of a row, rows a pass
  const int tid = threadIdx.x, lane = tid & 63, g4 = lane >> 4, l = lane & 15;
  const int wm = (tid >> 6) % S::WM, wk = (tid >> 6) / S::WM;
  const int rows = item_rows(a, w, tile), last = min(to, w.keys);
  // Float chunk c of row r of the pass, wave k along the keys.
  const auto at = [&](int k, int r, int c) -> f32x4 & {
    const int i = (k * LR + r) * CF + (c ^ (r & 15));
    u32x4 *p = i < 2 * S::TILE ? lds0 + i : lds1 + (i - 2 * S::TILE);
    return *reinterpret_cast<f32x4 *>(p);
  };
#pragma unroll
  for (int rt = 0; rt < S::RT; ++rt) {
    __syncthreads();  // the ring is free, and met_odd what it will be
    const float sum = over_groups_sum(R.l[rt]);
    if (g4 == 0) ml[wk * LR + wm * 16 + l] = make_float2(R.m[rt], sum);
    float f = 1.f;
    if constexpr (S::WK > 1) {
      __syncthreads();
      float top = -INFINITY;
#pragma unroll
      for (int k = 0; k < S::WK; ++k) top = fmaxf(top, ml[k * LR + wm * 16 + l].x);
      f = R.m[rt] == -INFINITY ? (top == -INFINITY ? 1.f : 0.f)
                               : __builtin_amdgcn_exp2f(R.m[rt] - top);
    }
#pragma unroll
    for (int d = 0; d < S::HD / 16; ++d) at(wk, wm * 16 + l, d * 4 + g4) = R.o[rt][d] * f;
    __syncthreads();
#pragma unroll 1
    for (int i = tid; i < LR * CF; i += S::NT) {
      const int p = i / CF, c = i % CF;
      const Groups g = groups_of<S>(rows, p / 16);
      const int r = (g.first + rt) * 16 + p % 16;
      if (rt >= g.n || r >= rows) continue;
      float top = -INFINITY, sum = 0.f;
#pragma unroll
      for (int k = 0; k < S::WK; ++k) top = fmaxf(top, ml[k * LR + p].x);
      f32x4 y{};
#pragma unroll
      for (int k = 0; k < S::WK; ++k) {
        const float2 x = ml[k * LR + p];
        sum += S::WK == 1 || x.x == -INFINITY ? x.y : x.y * __builtin_amdgcn_exp2f(x.x - top);
        y += at(k, p, c);
      }
      if (*met_odd) y += odd_values<S>(a, w, kvh, token_of(a, tile * w.step + r), c, from, last);
      put_row<S>(a, w, kvh, tile, r, c, y, sum, top, which);
    }
  }
  __syncthreads();  // LDS may be filled again
}

template <class S, bool VEC>
__global__ __launch_bounds__(S::NT, S::PER_CU) void k_tree_attn(TreeAttnArgs a) {
  __shared__ u32x4 ring0[2 * S::TILE], ring1[2 * S::TILE];
  __shared__ float2 ml[S::NW * 16];
  __shared__ long sums[S::NT / 64], found[2];
  __shared__ int met_odd;
  if (threadIdx.x == 0) met_odd = 0;
  Plan<S> plan(a, sums);
  const long total = plan.total;
  const int eff = blocks_used<S>(total, a.groups);
  const int g = logical_block(blockIdx.x, eff, a.groups);
  const long per = share_of(total, eff);
  long at = g * per;
  const long end = min(total, at + per);
  if (at >= end) {
    if (threadIdx.x == 0) a.joins[g].last = -1;
    return;
  }
  Work w;
  plan.find(a, at, found, w);
  Rows<S> R;
  for (;;) {
    const long local = at - w.base;
    const int each = w.nb * w.cost;
    const int item = __builtin_amdgcn_readfirstlane(quotient(local, each));
    const int off = __builtin_amdgcn_readfirstlane((int)(local - (long)item * each));
    const int off_end = __builtin_amdgcn_readfirstlane((int)min((long)each, off + (end - at)));
    const int b0 = __builtin_amdgcn_readfirstlane(quotient(off + w.cost - 1, w.cost));
    const int b1 = __builtin_amdgcn_readfirstlane(quotient(off_end + w.cost - 1, w.cost));
    const int kvh = __builtin_amdgcn_readfirstlane(quotient(item, w.tiles));
    const int tile = item - kvh * w.tiles;
    // Without masks, key tiles past the last row's own position are seen by none.
    const int last = min(w.n * a.group, (tile + 1) * w.step) - 1;
    const int upto = a.mask ? w.keys : min(w.keys, w.len + token_of(a, last) + 1);
    const int b2 = min(b1, (upto + S::BK - 1) / S::BK);
    // Tiles before `plain` are seen whole by every row.
    const int all = a.mask ? w.len : min(w.keys, w.len + token_of(a, tile * w.step) + 1);
    const int plain = min(b2, all / S::BK);
    int32_t page[S::NL];
    const bool loads = __builtin_amdgcn_readfirstlane(threadIdx.x >= S::NT - S::LT);
    if (loads && b0 < b2) load_pages<S>(a, w, b0 * S::BK, page);
    if (b0 < b1) load_rows<S>(a, w, kvh, tile, R);
    if (b0 < b2) {
      if (loads) {
        load_tile<S, VEC>(a, w, kvh, b0 * S::BK, page, ring0);
        load_pages<S>(a, w, (b0 + 1) * S::BK, page);
      }
      // Tile b, in `cur`, against NR row groups, while tile b + 1 is on its way into `nxt`.
      // The stages are arrays of their own so that the compiler knows that reads of one
      // need not wait for loads into the other.
      const auto step = [&](auto nr, auto draft, int b, u32x4 *cur,
                            u32x4 *nxt) __attribute__((always_inline)) {
        __builtin_amdgcn_s_waitcnt(kAllLoads);
        __syncthreads();  // tile b is there for every wave, the other stage is free
        if (loads && b + 1 < b2) {
          load_tile<S, VEC>(a, w, kvh, (b + 1) * S::BK, page, nxt);
          load_pages<S>(a, w, (b + 2) * S::BK, page);
        }
        if constexpr (draft.value) {
          if (clear_odd<S>(cur + S::TILE, w.len - b * S::BK)) met_odd = 1;
          __syncthreads();
        }
        if constexpr (nr.value > 0)
          tile_step<S, draft.value, nr.value>(a, w, b * S::BK, cur, R);
      };
      // Tiles that all rows see first, in a loop of their own, and waves by their number
      // of row groups in loops of their own (they meet at the same barriers): with
      // one loop around several kinds the kernel spilled registers inside it, and a reload
      // from scratch waits for every load before it, the next tile's among them.
      const auto walk = [&](auto nr) __attribute__((always_inline)) {
        const std::integral_constant<bool, false> context;
        const std::integral_constant<bool, true> draft;
        int b = b0;
        bool second = false;
        for (; b < plain; ++b) {
          step(nr, context, b, ring0, ring1);
          if (++b >= plain) {
            second = true;
            break;
          }
          step(nr, context, b, ring1, ring0);
        }
        for (; b < b2; ++b, second = !second)
          step(nr, draft, b, second ? ring1 : ring0, second ? ring0 : ring1);
      };
      if (R.n == S::RT)
        walk(std::integral_constant<int, S::RT>());
      else if (S::RT > 1 && R.n == 1)
        walk(std::integral_constant<int, 1>());
      else
        walk(std::integral_constant<int, 0>());
    }
    if (b0 < b1) {
      const bool whole = b0 == 0 && b1 == w.nb;
      store_rows<S>(a, w, kvh, tile, R, ring0, ring1, ml, whole ? -1 : 2L * g + (b0 == 0),
                    &met_odd, max(b0, plain) * S::BK, b2 * S::BK);
      if (threadIdx.x == 0) met_odd = 0;
    }
    at += off_end - off;
    if (at >= end) {
      // An item that begins here and ends in another block is joined afterwards, with the
      // blocks up to that in which its last key tile begins.
      if (threadIdx.x == 0) {
        int last = -1;
        if (b0 == 0 && b1 > 0 && b1 < w.nb) {
          const long begins = w.base + (item + 1L) * each - w.cost;
          for (last = g + 1; (last + 1) * per <= begins;) ++last;
        }
        a.joins[g] = {w.b, w.n, kvh, tile, w.step, last};
      }
      return;
    }
    if (at >= w.base + work_cost(a, w)) plan.next(a, at, w);
  }
}

constexpr int kTreeGroups = 512;  // the most blocks
constexpr int kJoinThreads = 256, kJoinGrid = 2048;

// Joins the items that more than one block has walked: block g's list entry names the item
// that it begins and another ends (each has one at most). Blocks take groups of rows of all
// items in turn (a grid over items and rows was mostly blocks with nothing to do: 8192
// of them took 11 us). Few partial results a row are read by one thread a column at once;
// many by SL threads in turn, whose sums are added in one order.
template <class S>
__global__ __launch_bounds__(kJoinThreads) void k_tree_join(TreeAttnArgs a) {
  constexpr int CF = S::HD / 4, SL = 4, RB = kJoinThreads / (CF * SL), RF = RB * SL;
  constexpr int FEW = 8;
  static_assert(RB >= 1 && kTreeGroups <= 2 * kJoinThreads, "a block has a row, a thread two blocks");
  __shared__ float2 ml[RB][kTreeGroups];  // of each partial result: reference, sum
  __shared__ f32x4 part[SL][RB][CF];
  __shared__ int first[kTreeGroups + 1], owner[kTreeGroups], sums[kJoinThreads / 64];
  const int tid = threadIdx.x, lane = tid & 63;
  // The items that have rows to join, and the first unit of each.
  int units[2], n_items = 0;
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const int g = 2 * tid + k;
    units[k] = 0;
    if (g < a.groups) {
      const TreeJoin i = a.joins[g];
      const int rows = min(i.step, i.n * a.group - i.tile * i.step);
      if (i.last >= 0)
        units[k] = i.last - g < FEW ? (rows + RF - 1) / RF : (rows + RB - 1) / RB;
    }
    n_items += units[k] > 0;
  }
  // (Units are below 2^16 in all, items too: one scan counts both.)
  int both = n_items << 20 | (units[0] + units[1]);
  int upto = wave_scan(both);
  if (lane == 63) sums[tid >> 6] = upto;
  __syncthreads();
  int total = 0;
#pragma unroll
  for (int i = 0; i < kJoinThreads / 64; ++i) {
    if (i < tid >> 6) upto += sums[i];
    total += sums[i];
  }
  int before = upto - both;
#pragma unroll
  for (int k = 0; k < 2; ++k)
    if (units[k]) {
      first[before >> 20] = before & 0xfffff;
      owner[before >> 20] = 2 * tid + k;
      before += 1 << 20 | units[k];
    }
  const int items = total >> 20, all = total & 0xfffff;
  const int c = tid % CF, r = tid / CF % RB, sl = tid / (CF * RB);
  __syncthreads();
  for (int u = blockIdx.x; u < all; u += kJoinGrid) {
    int lo = 0, hi = items;
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (first[mid] <= u)
        lo = mid;
      else
        hi = mid;
    }
    const int g = owner[lo];
    const TreeJoin i = a.joins[g];
    const int rows = min(i.step, i.n * a.group - i.tile * i.step), n = i.last - g + 1;
    const int r0 = (u - first[lo]) * (n <= FEW ? RF : RB);
    Work w;
    w.b = i.b;
    w.step = i.step;
    const auto at = [&](int b, int r) { return (2L * (g + b) + (b == 0)) * S::BM + r0 + r; };
    if (n <= FEW) {
      const int r = tid / CF;
      if (r0 + r >= rows) continue;
      float2 x[FEW];
      f32x4 o[FEW];
#pragma unroll
      for (int b = 0; b < FEW; ++b) {
        const long from = at(min(b, n - 1), r);
        x[b] = a.part_ml[from];
        o[b] = reinterpret_cast<const f32x4 *>(a.part)[from * CF + c];
      }
      float top = -INFINITY, l = 0.f;
#pragma unroll
      for (int b = 0; b < FEW; ++b) top = fmaxf(top, x[b].x);
      f32x4 y{};
#pragma unroll
      for (int b = 0; b < FEW; ++b) {
        if (b >= n) break;
        const float f = x[b].x == -INFINITY ? (top == -INFINITY ? 1.f : 0.f)
                                            : __builtin_amdgcn_exp2f(x[b].x - top);
        l += x[b].y * f;
        y += o[b] * f;
      }
      put_row<S>(a, w, i.kvh, i.tile, r0 + r, c, y, l, top, -1);
      continue;
    }
    __syncthreads();  // LDS is free
    for (int k = tid; k < n * RB; k += kJoinThreads)
      ml[k % RB][k / RB] = a.part_ml[at(k / RB, min(k % RB, rows - 1 - r0))];
    const int rr = min(r, rows - 1 - r0);
    f32x4 some[4];  // (on their way before the weights are known)
#pragma unroll
    for (int k = 0; k < 4; ++k)
      some[k] = reinterpret_cast<const f32x4 *>(a.part)[at(min(sl + k * SL, n - 1), rr) * CF + c];
    __syncthreads();
    float top = -INFINITY;
    for (int b = 0; b < n; ++b) top = fmaxf(top, ml[r][b].x);
    const auto weight = [&](int b) {
      const float x = ml[r][b].x;
      return x == -INFINITY ? (top == -INFINITY ? 1.f : 0.f) : __builtin_amdgcn_exp2f(x - top);
    };
    f32x4 y{};
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (sl + k * SL < n) y += some[k] * weight(sl + k * SL);
#pragma unroll 4
    for (int b = sl + 4 * SL; b < n; b += SL)
      y += reinterpret_cast<const f32x4 *>(a.part)[at(b, rr) * CF + c] * weight(b);
    part[sl][r][c] = y;
    __syncthreads();
    if (sl == 0 && r0 + r < rows) {
#pragma unroll
      for (int k = 1; k < SL; ++k) y += part[k][r][c];
      float l = 0.f;
      for (int b = 0; b < n; ++b) l += ml[r][b].y * weight(b);
      put_row<S>(a, w, i.kvh, i.tile, r0 + r, c, y, l, top, -1);
    }
  }
}

// Whether keys and values can go straight into LDS, 16 bytes at a time.
template <typename T>
bool tree_aligned(const TreeAttnArgs &a) {
  const auto even = [](const void *p, long ts, long hs) {
    return (reinterpret_cast<uintptr_t>(p) | (uintptr_t)(ts * sizeof(T)) |
            (uintptr_t)(hs * sizeof(T))) % 16 == 0 && (uint64_t)ts * sizeof(T) <= UINT32_MAX;
  };
  return a.hd * sizeof(T) % 16 == 0 && even(a.k, a.k_ts, a.k_hs) && even(a.v, a.v_ts, a.v_hs);
}

// Rows of all blocks together, by the rows of one (tree_block_rows) and head_dim's shape.
constexpr int tree_all_rows(int block_rows, int HD) {
  return block_rows <= 32 ? kTreeGroups * 32 : HD == 256 ? 256 * 128 : 256 * 256;
}

template <class S, bool VEC>
hipError_t launch_tree_shape(TreeAttnArgs a, void *ws, hipStream_t s) {
  a.groups = 256 * S::PER_CU;
  // (Four waves also run in the place of eight, where rows do not lie on 16 bytes.)
  static_assert(256 * S::PER_CU <= kTreeGroups &&
                    256 * S::PER_CU * S::BM <= tree_all_rows(S::NW == 8 ? 256 : 32, S::HD) &&
                    tree_all_rows(32, S::HD) <= tree_all_rows(256, S::HD),
                "the workspace has room for each block");
  a.part = static_cast<float *>(ws);
  a.part_ml = reinterpret_cast<float2 *>(a.part + (size_t)2 * a.groups * S::BM * S::HD);
  a.joins = reinterpret_cast<TreeJoin *>(a.part_ml + (size_t)2 * a.groups * S::BM);
  k_tree_attn<S, VEC><<<a.groups, S::NT, 0, s>>>(a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  k_tree_join<S><<<kJoinGrid, kJoinThreads, 0, s>>>(a);
  return hipGetLastError();
}

inline int tree_rows_of(int T, int n_seqs, int n_heads, int n_kv) {
  return (int)std::min<long>(((long)T * (n_heads / n_kv) + n_seqs - 1) / n_seqs, 1 << 20);
}

// Rows of a block by the rows that a mean sequence has for a key head: four waves along
// the keys, two blocks a CU, where 16 or 32 rows are enough; else eight waves along the
// rows. (32 sequences of 8192 keys, 8 key heads: 64 rows 261 us on four waves, 247 on eight,
// 128 rows 298 and 260; 16 rows 217 on four waves of 16 rows, 32 rows 236 and 247.)
inline int tree_block_rows(int rows) { return rows <= 16 ? 16 : rows <= 32 ? 32 : 256; }

template <typename T, int HD>
hipError_t launch_tree_type(const TreeAttnArgs &a, void *ws, hipStream_t s) {
  constexpr bool wide = sizeof(T) == 4 && HD == 256;  // (its tiles of 32 keys feed two waves)
  typedef TreeShape<T, HD, 4, wide ? 1 : 2, wide ? 2 : 1> Small;
  if (!tree_aligned<T>(a)) return launch_tree_shape<Small, false>(a, ws, s);
  const int rows = tree_block_rows(tree_rows_of(a.T, a.pages.n_seqs, a.n_heads, a.n_kv));
  if (rows == 256)
    return launch_tree_shape<TreeShape<T, HD, 8, HD == 256 ? 1 : 2, 8>, true>(a, ws, s);
  if constexpr (!wide)
    if (rows == 16) return launch_tree_shape<TreeShape<T, HD, 4, 1, 1>, true>(a, ws, s);
  return launch_tree_shape<Small, true>(a, ws, s);
}

template <typename T>
hipError_t launch_tree(const TreeAttnArgs &a, void *ws, hipStream_t s) {
  if (a.hd <= 64) return launch_tree_type<T, 64>(a, ws, s);
  if (a.hd <= 128) return launch_tree_type<T, 128>(a, ws, s);
  return launch_tree_type<T, 256>(a, ws, s);
}

}  // namespace
}  // namespace vsr
