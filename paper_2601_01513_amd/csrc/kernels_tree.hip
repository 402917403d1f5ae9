// Drafted trees over a paged key/value cache: their rows' positions, slots and ancestor
// masks, and their attention.
//
// Sequence s has len[s] positions in its pages; row j of its draft sits at position
// len + j. For query row j and head h, over the positions p it sees (p < len, or bit
// p - len of its mask; without masks p - len <= j):
//   x_p = scale q[j, h] . k[p, h / G],  out = sum_p e^(x_p - lse) v[p, h / G],
//   lse = log sum_p e^x_p;  nothing seen: out 0, lse -inf.
#include <algorithm>

#include "common.h"

namespace vsr {

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

constexpr int kTreeThreads = 256;

// Shape of a block: 4 waves, WM along the rows (each RT tiles of 16) and WK along the
// keys of a tile of BK; LDS rows of CH 16-byte chunks.
template <typename T_, int HD_, int RT_, int WM_>
struct TreeShape {
  typedef T_ T;
  static constexpr int HD = HD_, RT = RT_, WM = WM_, WK = 4 / WM_;
  static constexpr bool F32 = sizeof(T) == 4;
  static constexpr int BK = F32 && HD == 256 ? 32 : 64;
  static constexpr int BM = WM * RT * 16;
  static constexpr int KW = BK / 16 / WK;   // 16-key tiles of a wave
  static constexpr int EC = 16 / sizeof(T);  // elements a chunk
  static constexpr int CH = HD / EC;
  static constexpr int NL = BK * CH / kTreeThreads;  // chunks of K a thread loads
  static constexpr int TILE = BK * CH;               // chunks of a K or V tile
  static_assert(KW >= 1 && NL >= 1, "each wave has keys");
  static_assert((size_t)WK * BM * HD * 4 <= (size_t)4 * TILE * 16, "the join fits the ring");
};

// LDS gives 256 bytes to 16 lanes at once: chunk c of row r lies where 16 rows' chunks
// c fall on different banks.
template <int CH>
__device__ __forceinline__ int swz(int r) {
  return CH >= 16 ? r & 15 : (r >> 1) & 7;
}

// The walk of all blocks over all work: item (sequence, key head, tile of rows, tiles
// innermost) has as many units as its sequence has key tiles; block g of `eff` takes
// units [total g / eff, total (g + 1) / eff).
struct Work {
  int s, b, n;       // a sequence and its rows
  int len, keys;     // positions before the draft, and with it
  int tiles, nb;     // row tiles, key tiles
  long base;         // units before it
};

template <class S>
__device__ __forceinline__ void work_of(const TreeAttnArgs &a, int s, Work &w) {
  int e;
  seq_rows(a.start, a.T, s, w.b, e);
  w.s = s;
  w.n = e - w.b;
  w.len = seq_len(a.pages, s);
  w.keys = (int)min((long)w.len + w.n, (long)seq_room(a.pages, s));
  const int G = a.n_heads / a.n_kv;
  w.tiles = (int)(((long)w.n * G + S::BM - 1) / S::BM);
  w.nb = max(1, (int)(((long)w.keys + S::BK - 1) / S::BK));
}

__device__ __forceinline__ long work_units(const TreeAttnArgs &a, const Work &w) {
  return (long)a.n_kv * w.tiles * w.nb;
}

struct Plan {
  long total;
  int eff;
  int n_pref;
};

// Units before each thread's run of sequences, and their total, in LDS.
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
  for (int i = 0; i < kTreeThreads / 64; ++i) {
    if (i < w) before += sums[i];
    total += sums[i];
  }
  __syncthreads();
  return before + v - mine;
}

constexpr int kMinUnits = 2;  // the least units worth a block

__device__ __forceinline__ int blocks_used(long total, int groups) {
  return (int)max(1L, min((total + kMinUnits - 1) / kMinUnits, (long)groups));
}
// Blocks of one XCD take neighbouring ranges (tiles that share keys), unless there are
// fewer of them than the grid has.
__device__ __forceinline__ int logical_block(int b, int eff, int groups) {
  return eff < groups ? b : b % 8 * (groups / 8) + b / 8;
}

// Finds the sequence that holds unit `at` (and its Work): every thread gets it.
template <class S>
__device__ __forceinline__ void find_unit(const TreeAttnArgs &a, long first, long at, long *found,
                                          Work &w) {
  const int per = (a.pages.n_seqs + kTreeThreads - 1) / kTreeThreads;
  const int s0 = threadIdx.x * per;
  long base = first;
  for (int i = 0; i < per && s0 + i < a.pages.n_seqs; ++i) {
    Work x;
    work_of<S>(a, s0 + i, x);
    const long u = work_units(a, x);
    if (at >= base && at < base + u) {
      found[0] = s0 + i;
      found[1] = base;
    }
    base += u;
  }
  __syncthreads();
  const int s = __builtin_amdgcn_readfirstlane((int)found[0]);
  work_of<S>(a, s, w);
  w.base = found[1];
  __syncthreads();
}

template <class S>
__device__ __forceinline__ long my_units(const TreeAttnArgs &a) {
  const int per = (a.pages.n_seqs + kTreeThreads - 1) / kTreeThreads;
  long u = 0;
  for (int i = 0; i < per; ++i) {
    const int s = threadIdx.x * per + i;
    if (s >= a.pages.n_seqs) break;
    Work x;
    work_of<S>(a, s, x);
    u += work_units(a, x);
  }
  return u;
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
  f32x4 o[S::RT][S::HD / 16];
};

template <typename T>
__device__ __forceinline__ T load_part(const T *p, int i, int hd) {
  return i < hd ? p[i] : T(0.f);
}

template <class S>
__device__ __forceinline__ void load_rows(const TreeAttnArgs &a, const Work &w, int kvh, int tile,
                                          Rows<S> &R) {
  typedef typename S::T T;
  const int lane = threadIdx.x & 63, g4 = lane >> 4, wm = (threadIdx.x >> 6) % S::WM;
  const int G = a.n_heads / a.n_kv;
#pragma unroll
  for (int rt = 0; rt < S::RT; ++rt) {
    const long r = (long)tile * S::BM + (wm * S::RT + rt) * 16 + (lane & 15);
    const bool real = r < (long)w.n * G;
    const int rc = real ? (int)r : 0;
    R.j[rt] = rc / G;
    R.m[rt] = -INFINITY;
    R.l[rt] = 0.f;
    const T *q = static_cast<const T *>(a.q) + (w.b + R.j[rt]) * a.q_ts +
                 (long)(kvh * G + rc % G) * a.q_hs;
    constexpr int V = S::F32 ? 4 : 8;
#pragma unroll
    for (int c = 0; c < Rows<S>::QN / (S::F32 ? 4 : 1); ++c) {
      const int at = c * 4 * V + g4 * V;
      Pack<T, V> x;
      if (at + V <= a.hd) {
        x = *reinterpret_cast<const Pack<T, V> *>(q + at);
      } else {
#pragma unroll
        for (int i = 0; i < V; ++i) x.v[i] = load_part(q, at + i, a.hd);
      }
      if constexpr (S::F32) {
#pragma unroll
        for (int i = 0; i < 4; ++i) R.q[rt][c * 4 + i] = x.v[i];
      } else {
        R.q[rt][c] = __builtin_bit_cast(u32x4, x);
      }
    }
#pragma unroll
    for (int d = 0; d < S::HD / 16; ++d) R.o[rt][d] = f32x4{};
  }
}

// Pages of the keys that a thread loads, of the tile at kb.
template <class S>
__device__ __forceinline__ void load_pages(const TreeAttnArgs &a, const Work &w, int kb,
                                           int32_t *page) {
  const int32_t *table = a.pages.table + w.s * a.pages.table_stride;
#pragma unroll
  for (int i = 0; i < S::NL; ++i) {
    const int p = kb + (i * kTreeThreads + (int)threadIdx.x) / S::CH;
    page[i] = p < w.keys ? table[p >> a.pages.page_shift] : -1;
  }
}

// Key tile kb of both matrices on its way into an LDS stage: rows past the sequence's
// keys are zeros. VEC: 16-byte loads straight into LDS; else through registers.
template <class S, bool VEC>
__device__ __forceinline__ void load_tile(const TreeAttnArgs &a, const Work &w, int kvh, int kb,
                                          const int32_t *page, u32x4 *stage) {
  typedef typename S::T T;
  const int tid = threadIdx.x;
  const T *k = static_cast<const T *>(a.k) + kvh * a.k_hs;
  const T *v = static_cast<const T *>(a.v) + kvh * a.v_hs;
#pragma unroll
  for (int i = 0; i < S::NL; ++i) {
    const int at = i * kTreeThreads + tid, r = at / S::CH, c = (at % S::CH) ^ swz<S::CH>(r);
    const int p = kb + r;
    const bool real = p < w.keys && c * S::EC < a.hd;
    const int pg = (uint32_t)page[i] < (uint32_t)a.pages.n_pages ? page[i] : 0;
    const long slot = ((long)pg << a.pages.page_shift) | (p & ((1 << a.pages.page_shift) - 1));
    const T *kp = k + slot * a.k_ts + c * S::EC, *vp = v + slot * a.v_ts + c * S::EC;
    if constexpr (VEC) {
      const void *kz = real ? static_cast<const void *>(kp) : static_cast<const void *>(&g_zeros);
      const void *vz = real ? static_cast<const void *>(vp) : static_cast<const void *>(&g_zeros);
      u32x4 *to = stage + i * kTreeThreads + (tid & ~63);
      __builtin_amdgcn_global_load_lds(kz, to, 16, 0, 0);
      __builtin_amdgcn_global_load_lds(vz, to + S::TILE, 16, 0, 0);
    } else {
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

// Four V elements of column (dt 16 + lane % 16), keys 4 (lane / 16) .. + 3 of the 16
// from row k0 on.
template <class S>
__device__ __forceinline__ typename Mat<typename S::T>::x4 v_frag(const u32x4 *vs, int k0, int dt) {
  typedef short s16x4 __attribute__((ext_vector_type(4)));
  const int lane = threadIdx.x & 63, i = lane & 15;
  const int r = k0 + 4 * (lane >> 4) + (i >> 2);
  const int c = (dt * 2 + ((i & 3) >> 1)) ^ swz<S::CH>(r);
  const char *p = reinterpret_cast<const char *>(vs + r * S::CH + c) + (i & 1) * 8;
  return __builtin_bit_cast(
      typename Mat<typename S::T>::x4,
      __builtin_amdgcn_ds_read_tr16_b64_v4i16(
          (__attribute__((address_space(3))) s16x4 *)const_cast<char *>(p)));
}

// Values that are no numbers, in the rows of a draft, reach the rows that see them and no
// others (0 times them is no number either): x is the value itself and 0 otherwise, seen 1
// or 0; counts of +inf, -inf and NaN, each added as such where it is not 0.
__device__ __forceinline__ float odd_sum(float pos, float neg, float nan) {
  return (pos > 0.f ? INFINITY : 0.f) + (neg > 0.f ? -INFINITY : 0.f) + (nan > 0.f ? NAN : 0.f);
}

template <typename X>
__device__ __forceinline__ bool not_finite(X x) {
  return !(__builtin_fabsf(to_f32(x)) < INFINITY);
}

// One key tile against a wave's rows. DRAFT: the tile has keys past len.
template <class S, bool DRAFT>
__device__ __forceinline__ void tile_step(const TreeAttnArgs &a, const Work &w, int kb,
                                          const u32x4 *st, Rows<S> &R) {
  typedef typename S::T T;
  typedef Mat<T> M;
  const int lane = threadIdx.x & 63, g4 = lane >> 4, wk = (threadIdx.x >> 6) / S::WM;
  const u32x4 *ks = st, *vs = st + S::TILE;
  const int key0 = wk * S::KW * 16;
  f32x4 x[S::RT][S::KW];
#pragma unroll
  for (int t = 0; t < S::KW; ++t) {
#pragma unroll
    for (int rt = 0; rt < S::RT; ++rt) x[rt][t] = f32x4{};
    const int r = key0 + t * 16 + (lane & 15);
#pragma unroll
    for (int c = 0; c < S::CH / 4; ++c) {
      const u32x4 kf = ks[r * S::CH + ((4 * c + g4) ^ swz<S::CH>(r))];
#pragma unroll
      for (int rt = 0; rt < S::RT; ++rt) {
        if constexpr (S::F32) {
          const f32x4 kv = __builtin_bit_cast(f32x4, kf);
#pragma unroll
          for (int i = 0; i < 4; ++i) x[rt][t] = M::mul(kv[i], R.q[rt][c * 4 + i], x[rt][t]);
        } else {
          x[rt][t] = M::mul(__builtin_bit_cast(typename M::x8, kf),
                            __builtin_bit_cast(typename M::x8, R.q[rt][c]), x[rt][t]);
        }
      }
    }
  }
  uint32_t seen[S::RT];  // bit 4 t + i (DRAFT)
#pragma unroll
  for (int rt = 0; rt < S::RT; ++rt) {
    seen[rt] = 0;
    float top = -INFINITY;
#pragma unroll
    for (int t = 0; t < S::KW; ++t) {
      [[maybe_unused]] const int p0 = kb + key0 + t * 16 + 4 * g4;
      if constexpr (DRAFT) {
        uint32_t bits = 0;
        const int d0 = p0 - w.len;
        if (a.mask) {
          // (Bits past the words are clear; d0 may be up to 3 below the first.)
          const uint32_t *row = a.mask + (w.b + R.j[rt]) * a.mask_stride;
          const int wd = max(d0, 0) >> 5;
          uint64_t v = wd < a.mask_words && p0 < w.keys ? row[wd] : 0;
          if (wd + 1 < a.mask_words && p0 < w.keys) v |= (uint64_t)row[wd + 1] << 32;
          bits = d0 >= 0 ? (uint32_t)(v >> (d0 & 31)) : d0 > -4 ? (uint32_t)(v << -d0) : 0;
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int d = d0 + i;
          const bool drafted = a.mask ? (bits >> i) & 1 : d <= R.j[rt];
          const bool vis = d < 0 || (drafted && p0 + i < w.keys);
          seen[rt] |= (uint32_t)vis << (4 * t + i);
        }
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float y = x[rt][t][i] * a.scale_log2;
        if constexpr (DRAFT) y = (seen[rt] >> (4 * t + i)) & 1 ? y : -INFINITY;
        x[rt][t][i] = y;
        top = fmaxf(top, y);
      }
    }
    top = over_groups_max(top);
    if (__any(top > R.m[rt])) {
      const float m = fmaxf(R.m[rt], top);
      const float f = m == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(R.m[rt] - m);
      R.m[rt] = m;
      R.l[rt] *= f;
#pragma unroll
      for (int d = 0; d < S::HD / 16; ++d) R.o[rt][d] *= f;
    }
    const float ref = R.m[rt] == -INFINITY ? 0.f : R.m[rt];
#pragma unroll
    for (int t = 0; t < S::KW; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float p = __builtin_amdgcn_exp2f(x[rt][t][i] - ref);
        x[rt][t][i] = p;
        R.l[rt] += p;
      }
  }
  if constexpr (S::F32) {
#pragma unroll
    for (int t = 0; t < S::KW; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int r = key0 + t * 16 + 4 * g4 + i;
#pragma unroll
        for (int d = 0; d < S::HD / 16; ++d) {
          const int col = d * 16 + (lane & 15);
          float v = reinterpret_cast<const float *>(vs + r * S::CH + ((col >> 2) ^ swz<S::CH>(r)))[col & 3];
          if constexpr (DRAFT) {
            const bool odd = not_finite(v);
            if (__any(odd)) {
              const float one = odd ? 1.f : 0.f;
              const float p1 = v > 0.f ? one : 0.f, n1 = v < 0.f ? one : 0.f,
                          z1 = v != v ? 1.f : 0.f;
#pragma unroll
              for (int rt = 0; rt < S::RT; ++rt) {
                const float vis = (float)((seen[rt] >> (4 * t + i)) & 1);
                const f32x4 np = M::mul(p1, vis, f32x4{}), nn = M::mul(n1, vis, f32x4{}),
                            nz = M::mul(z1, vis, f32x4{});
#pragma unroll
                for (int e = 0; e < 4; ++e) R.o[rt][d][e] += odd_sum(np[e], nn[e], nz[e]);
              }
              v = odd ? 0.f : v;
            }
          }
#pragma unroll
          for (int rt = 0; rt < S::RT; ++rt) R.o[rt][d] = M::mul(v, x[rt][t][i], R.o[rt][d]);
        }
      }
  } else {
    typedef typename M::x4 x4;
    typedef typename M::x8 x8;
    x4 p[S::RT][S::KW];
#pragma unroll
    for (int rt = 0; rt < S::RT; ++rt)
#pragma unroll
      for (int t = 0; t < S::KW; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) p[rt][t][i] = from_f32<T>(x[rt][t][i]);
#pragma unroll
    for (int d = 0; d < S::HD / 16; ++d) {
      x4 v[S::KW];
#pragma unroll
      for (int t = 0; t < S::KW; ++t) {
        v[t] = v_frag<S>(vs, key0 + t * 16, d);
        if constexpr (DRAFT) {
          bool odd = false;
#pragma unroll
          for (int i = 0; i < 4; ++i) odd |= not_finite(v[t][i]);
          if (__any(odd)) {
            x4 p1, n1, z1;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const float f = to_f32(v[t][i]);
              const bool is = not_finite(f);
              p1[i] = from_f32<T>(is && f > 0.f ? 1.f : 0.f);
              n1[i] = from_f32<T>(is && f < 0.f ? 1.f : 0.f);
              z1[i] = from_f32<T>(f != f ? 1.f : 0.f);
              if (is) v[t][i] = from_f32<T>(0.f);
            }
#pragma unroll
            for (int rt = 0; rt < S::RT; ++rt) {
              x4 vis;
#pragma unroll
              for (int i = 0; i < 4; ++i)
                vis[i] = from_f32<T>((float)((seen[rt] >> (4 * t + i)) & 1));
              const f32x4 np = M::mul(p1, vis, f32x4{}), nn = M::mul(n1, vis, f32x4{}),
                          nz = M::mul(z1, vis, f32x4{});
#pragma unroll
              for (int e = 0; e < 4; ++e) R.o[rt][d][e] += odd_sum(np[e], nn[e], nz[e]);
            }
          }
        }
      }
#pragma unroll
      for (int rt = 0; rt < S::RT; ++rt) {
        if constexpr (S::KW == 1) {
          R.o[rt][d] = M::mul(v[0], p[rt][0], R.o[rt][d]);
        } else {
          // The 32 keys of two tiles: a lane's first four k are tile t's, the others t + 1's,
          // in both operands.
#pragma unroll
          for (int t = 0; t < S::KW; t += 2) {
            const x8 vv = __builtin_shufflevector(v[t], v[t + 1], 0, 1, 2, 3, 4, 5, 6, 7);
            const x8 pp = __builtin_shufflevector(p[rt][t], p[rt][t + 1], 0, 1, 2, 3, 4, 5, 6, 7);
            R.o[rt][d] = M::mul(vv, pp, R.o[rt][d]);
          }
        }
      }
    }
  }
}

// Float chunk c (of HD / 4) of row r in the join's LDS area.
template <class S>
__device__ __forceinline__ int join_at(int wk, int r, int c) {
  return (wk * S::BM + r) * (S::HD / 4) + (c ^ (r & 15));
}

// The waves' shares of an item joined and stored: out and lse, or (which >= 0) partial
// result `which` of block g.
template <class S>
__device__ __forceinline__ void store_rows(const TreeAttnArgs &a, const Work &w, int kvh, int tile,
                                           Rows<S> &R, u32x4 *lds, float2 *ml, long which) {
  typedef typename S::T T;
  const int tid = threadIdx.x, lane = tid & 63, g4 = lane >> 4;
  const int wm = (tid >> 6) % S::WM, wk = (tid >> 6) / S::WM;
  const int G = a.n_heads / a.n_kv;
  __syncthreads();  // the ring is free
#pragma unroll
  for (int rt = 0; rt < S::RT; ++rt) {
    R.l[rt] = over_groups_sum(R.l[rt]);
    if (g4 == 0)
      ml[wk * S::BM + (wm * S::RT + rt) * 16 + lane] = make_float2(R.m[rt], R.l[rt]);
  }
  __syncthreads();
  f32x4 *o = reinterpret_cast<f32x4 *>(lds);
#pragma unroll
  for (int rt = 0; rt < S::RT; ++rt) {
    const int r = (wm * S::RT + rt) * 16 + (lane & 15);
    float top = -INFINITY;
#pragma unroll
    for (int i = 0; i < S::WK; ++i) top = fmaxf(top, ml[i * S::BM + r].x);
    const float f = R.m[rt] == -INFINITY ? (top == -INFINITY ? 1.f : 0.f)
                                         : __builtin_amdgcn_exp2f(R.m[rt] - top);
#pragma unroll
    for (int d = 0; d < S::HD / 16; ++d) o[join_at<S>(wk, r, d * 4 + g4)] = R.o[rt][d] * f;
  }
  __syncthreads();
  for (int i = tid; i < S::BM * (S::HD / 4); i += kTreeThreads) {
    const int r = i / (S::HD / 4), c = i % (S::HD / 4);
    const long gr = (long)tile * S::BM + r;
    if (gr >= (long)w.n * G) break;
    float top = -INFINITY, l = 0.f;
#pragma unroll
    for (int k = 0; k < S::WK; ++k) top = fmaxf(top, ml[k * S::BM + r].x);
    f32x4 y{};
#pragma unroll
    for (int k = 0; k < S::WK; ++k) {
      const float2 x = ml[k * S::BM + r];
      l += x.x == -INFINITY ? x.y : x.y * __builtin_amdgcn_exp2f(x.x - top);
      y += o[join_at<S>(k, r, c)];
    }
    if (which >= 0) {
      reinterpret_cast<f32x4 *>(a.part)[(which * S::BM + r) * (S::HD / 4) + c] = y;
      if (c == 0) a.part_ml[which * S::BM + r] = make_float2(top, l);
      continue;
    }
    const int j = (int)gr / G, h = kvh * G + (int)gr % G;
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
          l == 0.f ? -INFINITY : (top + __builtin_log2f(l)) * 0.69314718055994531f;
  }
  __syncthreads();  // LDS may be filled again
}

template <class S, bool VEC>
__global__ __launch_bounds__(kTreeThreads) void k_tree_attn(TreeAttnArgs a) {
  __shared__ u32x4 ring[4 * S::TILE];
  __shared__ float2 ml[S::WK * S::BM];
  __shared__ long sums[kTreeThreads / 64], found[2];
  long total;
  const long first = block_scan(my_units<S>(a), sums, total);
  if (total == 0) return;
  const int eff = blocks_used(total, a.groups);
  const int g = logical_block(blockIdx.x, eff, a.groups);
  if (g >= eff) return;
  long at = total * g / eff;
  const long end = total * (g + 1) / eff;
  Work w;
  find_unit<S>(a, first, at, found, w);
  const int G = a.n_heads / a.n_kv;
  Rows<S> R;
  for (;;) {
    const long local = at - w.base;
    const int item = (int)(local / w.nb), b0 = (int)(local % w.nb);
    const int kvh = item / w.tiles, tile = item % w.tiles;
    const int b1 = (int)min((long)w.nb, b0 + (end - at));
    // Without masks, key tiles past the last row's own position are seen by none.
    const int last = min(w.n - 1, (int)min((long)INT32_MAX, ((long)(tile + 1) * S::BM - 1) / G));
    const long upto = a.mask ? w.keys : min((long)w.keys, (long)w.len + last + 1);
    const int b2 = min(b1, (int)((upto + S::BK - 1) / S::BK));
    load_rows<S>(a, w, kvh, tile, R);
    int32_t page[S::NL];
    if (b0 < b2) {
      load_pages<S>(a, w, b0 * S::BK, page);
      load_tile<S, VEC>(a, w, kvh, b0 * S::BK, page, ring);
      if (b0 + 1 < b2) load_pages<S>(a, w, (b0 + 1) * S::BK, page);
      int stage = 0;
      for (int b = b0; b < b2; ++b) {
        __syncthreads();  // tile b is there, the other stage is free
        if (b + 1 < b2) {
          load_tile<S, VEC>(a, w, kvh, (b + 1) * S::BK, page, ring + (stage ^ 1) * 2 * S::TILE);
          if (b + 2 < b2) load_pages<S>(a, w, (b + 2) * S::BK, page);
        }
        const u32x4 *st = ring + stage * 2 * S::TILE;
        if ((long)(b + 1) * S::BK <= w.len)
          tile_step<S, false>(a, w, b * S::BK, st, R);
        else
          tile_step<S, true>(a, w, b * S::BK, st, R);
        stage ^= 1;
      }
    }
    const bool whole = b0 == 0 && b1 == w.nb;
    store_rows<S>(a, w, kvh, tile, R, ring, ml, whole ? -1 : 2L * g + (b0 == 0));
    at += b1 - b0;
    if (at >= end) return;
    while (at >= w.base + work_units(a, w)) {
      const long base = w.base + work_units(a, w);
      work_of<S>(a, w.s + 1, w);
      w.base = base;
    }
  }
}

// Joins the items that more than one block has walked. Block (x, y): the item that
// attention block x begins and another ends (each has one at most), rows y RB .. + RB.
template <class S>
__global__ __launch_bounds__(kTreeThreads) void k_tree_join(TreeAttnArgs a) {
  typedef typename S::T T;
  constexpr int CF = S::HD / 4, RB = kTreeThreads / CF;
  __shared__ long sums[kTreeThreads / 64], found[2];
  long total;
  const long first = block_scan(my_units<S>(a), sums, total);
  if (total == 0) return;
  const int eff = blocks_used(total, a.groups), g = blockIdx.x;
  if (g >= eff) return;
  const long beg = total * g / eff, end = total * (g + 1) / eff;
  Work w;
  find_unit<S>(a, first, end - 1, found, w);
  const int item = (int)((end - 1 - w.base) / w.nb);
  const long ibeg = w.base + (long)item * w.nb, iend = ibeg + w.nb;
  if (ibeg < beg || iend <= end) return;
  const int kvh = item / w.tiles, tile = item % w.tiles, G = a.n_heads / a.n_kv;
  const int r = blockIdx.y * RB + threadIdx.x / CF, c = threadIdx.x % CF;
  const long gr = (long)tile * S::BM + r;
  if (r >= S::BM || gr >= (long)w.n * G) return;
  int last = g + 1;
  while (total * (last + 1) / eff < iend) ++last;
  const auto at = [&](int b) { return (2L * b + (b == g)) * S::BM + r; };
  float top = -INFINITY, l = 0.f;
  for (int b = g; b <= last; ++b) top = fmaxf(top, a.part_ml[at(b)].x);
  f32x4 y{};
  for (int b = g; b <= last; ++b) {
    const float2 x = a.part_ml[at(b)];
    const float f = x.x == -INFINITY ? (top == -INFINITY ? 1.f : 0.f)
                                     : __builtin_amdgcn_exp2f(x.x - top);
    l += x.y * f;
    y += reinterpret_cast<const f32x4 *>(a.part)[at(b) * CF + c] * f;
  }
  const int j = (int)gr / G, h = kvh * G + (int)gr % G;
  const float inv = l == 0.f ? 1.f : 1.f / l;
  T *out = static_cast<T *>(a.out) + (w.b + j) * a.o_ts + h * a.o_hs + 4 * c;
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (4 * c + e < a.hd) out[e] = from_f32<T>(y[e] * inv);
  if (c == 0 && a.lse)
    a.lse[(long)(w.b + j) * a.n_heads + h] =
        l == 0.f ? -INFINITY : (top + __builtin_log2f(l)) * 0.69314718055994531f;
}

constexpr int kTreeGroups = 512;

template <class S>
hipError_t launch_tree_shape(TreeAttnArgs a, void *ws, hipStream_t s) {
  a.groups = kTreeGroups;
  a.part = static_cast<float *>(ws);
  a.part_ml = reinterpret_cast<float2 *>(a.part + (size_t)2 * kTreeGroups * S::BM * S::HD);
  const auto even = [&](const void *p, long ts, long hs) {
    const uintptr_t low = reinterpret_cast<uintptr_t>(p) | (uintptr_t)(ts * sizeof(typename S::T)) |
                          (uintptr_t)(hs * sizeof(typename S::T));
    return low % 16 == 0;
  };
  const bool vec = a.hd % S::EC == 0 && even(a.k, a.k_ts, a.k_hs) && even(a.v, a.v_ts, a.v_hs);
  if (vec)
    k_tree_attn<S, true><<<a.groups, kTreeThreads, 0, s>>>(a);
  else
    k_tree_attn<S, false><<<a.groups, kTreeThreads, 0, s>>>(a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  constexpr int RB = kTreeThreads / (S::HD / 4);
  k_tree_join<S><<<dim3(a.groups, (S::BM + RB - 1) / RB), kTreeThreads, 0, s>>>(a);
  return hipGetLastError();
}

int tree_rows_of(int T, int n_seqs, int n_heads, int n_kv) {
  return (int)std::min<long>(((long)T * (n_heads / n_kv) + n_seqs - 1) / n_seqs, 1 << 20);
}

// Rows of a block by the rows that a mean sequence has for a key head.
int tree_block_rows(int rows) { return rows <= 16 ? 16 : rows <= 32 ? 32 : rows <= 64 ? 64 : 128; }

template <typename T, int HD>
hipError_t launch_tree_type(const TreeAttnArgs &a, void *ws, hipStream_t s) {
  constexpr bool wide = sizeof(T) == 4 && HD == 256;  // (its tiles of 32 keys feed two waves)
  switch (tree_block_rows(tree_rows_of(a.T, a.pages.n_seqs, a.n_heads, a.n_kv))) {
    case 16:
      if constexpr (!wide) return launch_tree_shape<TreeShape<T, HD, 1, 1>>(a, ws, s);
    case 32:
      if constexpr (!wide) return launch_tree_shape<TreeShape<T, HD, 2, 1>>(a, ws, s);
      return launch_tree_shape<TreeShape<T, HD, 1, 2>>(a, ws, s);
    case 64:
      return launch_tree_shape<TreeShape<T, HD, 2, 2>>(a, ws, s);
    default:
      return launch_tree_shape<TreeShape<T, HD, 2, 4>>(a, ws, s);
  }
}

template <typename T>
hipError_t launch_tree_hd(const TreeAttnArgs &a, void *ws, hipStream_t s) {
  if (a.hd <= 64) return launch_tree_type<T, 64>(a, ws, s);
  if (a.hd <= 128) return launch_tree_type<T, 128>(a, ws, s);
  return launch_tree_type<T, 256>(a, ws, s);
}

}  // namespace

hipError_t launch_tree_rows(const TreeRowsArgs &a, hipStream_t s) {
  k_tree_rows<<<a.pages.n_seqs + 1, kRowsThreads, 0, s>>>(a);
  return hipGetLastError();
}

size_t tree_attention_workspace_bytes(int dtype, int hd, int T, int n_seqs, int n_heads, int n_kv) {
  (void)dtype;
  const int HD = hd <= 64 ? 64 : hd <= 128 ? 128 : 256;
  const int rows = std::max(32, tree_block_rows(tree_rows_of(T, n_seqs, n_heads, n_kv)));
  return (size_t)2 * kTreeGroups * rows * (HD * sizeof(float) + sizeof(float2));
}

hipError_t launch_tree_attention(TreeAttnArgs a, int dtype, void *ws, hipStream_t s) {
  if (dtype == 0) return launch_tree_hd<float>(a, ws, s);
  if (dtype == 1) return launch_tree_hd<bf16>(a, ws, s);
  return launch_tree_hd<f16>(a, ws, s);
}

}  // namespace vsr
