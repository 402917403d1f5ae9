// Log-probabilities of given tokens, with their ranks, the distribution's entropy and
// the most likely alternatives, in one read of the logits.
//
// For a row x with largest value m and d = x - m:
//   S' = sum over all but one largest of e^d,  W = sum of d e^d,
//   logprob[t] = x[t] - m - log1p(S'),  entropy = log1p(S') - W / (1 + S').
// The largest is left out of S' so that log1p keeps its relative accuracy where one token
// has nearly all the mass.
//
// A block takes a segment of a row, each of its waves 1024 entries of every 4096. Lanes
// keep (m, S', W) online and count the entries ahead of the token. For the alternatives a
// wave keeps a list of candidates in LDS and a bound below which no entry can be one of
// its best: at first the top-th largest of the tile's 64 lane maxima, later the top-th
// largest of the list; tiles without an entry above it pass by one comparison of the lane
// maxima. Segments are merged by a second kernel.
#include <algorithm>
#include <type_traits>

#include "common.h"

namespace vsr {

namespace {

constexpr int kLpThreads = 256, kLpWaves = kLpThreads / 64;
constexpr int kLpLane = 16;                  // entries a lane and tile
constexpr int kLpTile = kLpLane * 64;        // entries a wave and tile
constexpr int kMaxTop = 64;
constexpr int kList = kLpTile + kMaxTop;     // a full tile behind the best ones so far
static_assert(kLpWaves * kList >= 64 * kMaxTop, "the lists hold 64 segments' best");

// An order of floats as unsigned numbers; 0: nothing (and NaN).
__device__ __forceinline__ uint32_t order_of(float x) {
  const uint32_t b = __float_as_uint(x + 0.f);  // (-0 is 0)
  return x != x ? 0u : b ^ (b & 0x80000000u ? 0xffffffffu : 0x80000000u);
}
__device__ __forceinline__ float value_of(uint32_t o) {
  return __uint_as_float(o ^ (o & 0x80000000u ? 0x80000000u : 0xffffffffu));
}
constexpr uint32_t kNothing = 0x007fffffu;  // order_of(-inf): no candidate is as low

struct Stats {
  float m, s, w;
  int ahead;
};

__device__ __forceinline__ Stats joined(const Stats &a, const Stats &b) {
  const bool up = b.m > a.m;
  const float m = up ? b.m : a.m, lm = up ? a.m : b.m;
  const float ls = up ? a.s : b.s, lw = up ? a.w : b.w;
  Stats r{m, up ? b.s : a.s, up ? b.w : a.w, a.ahead + b.ahead};
  if (lm == -INFINITY) {
    r.s += ls;  // (0, or NaN)
  } else {
    const float d = lm - m, f = __expf(d), one = 1.f + ls;
    r.s += f * one;
    r.w += f == 0.f ? 0.f : f * (lw + one * d);
  }
  return r;
}

__device__ __forceinline__ Stats over_wave(Stats a) {
#pragma unroll
  for (int d = 1; d < 64; d <<= 1)
    a = joined(a, {__shfl_xor(a.m, d), __shfl_xor(a.s, d), __shfl_xor(a.w, d), __shfl_xor(a.ahead, d)});
  return a;
}

struct Entry {
  uint32_t order;
  int id;
};

__device__ __forceinline__ int set_lanes(bool in) { return __popcll(__ballot(in)); }

// The largest bound that at least `want` of the values reach which count(b) counts (the
// same in every lane); the lowest candidate if there are fewer. The lowest LOW bits of an
// order follow from the others (those of a 16-bit type's values).
template <int LOW, class Count>
__device__ __forceinline__ uint32_t wave_bound(int want, Count count) {
  uint32_t b = 0;
#pragma unroll 1
  for (int bit = 31; bit >= LOW; --bit) {
    const uint32_t t = b | 1u << bit;
    if (count(t) >= want) b = t;
  }
  if (LOW && b < 0x80000000u) b |= (1u << LOW) - 1;
  return max(b, kNothing + 1);
}

// Leaves the `top` best of a wave's list of n (ties: the lowest ids), in the order they
// were in; returns their number, and in `bound` the lowest order among them if they are
// `top`.
template <int LOW>
__device__ __forceinline__ int wave_cut(Entry *list, int n, int top, uint32_t &bound) {
  const int lane = threadIdx.x & 63;
  if (n < top) return n;
  uint32_t b;
  if (n <= 256) {
    uint32_t o[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] = i * 64 + lane < n ? list[i * 64 + lane].order : 0;
    b = wave_bound<LOW>(top, [&](uint32_t t) {
      int c = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) c += set_lanes(o[i] >= t);
      return c;
    });
  } else {
    b = wave_bound<LOW>(top, [&](uint32_t t) {
      int c = 0;
      for (int i = 0; i < n; i += 64) c += set_lanes(i + lane < n && list[i + lane].order >= t);
      return c;
    });
  }
  bound = max(bound, b);
  int above = 0, ties = 0;
  for (int i = 0; i < n; i += 64) {
    const uint32_t o = i + lane < n ? list[i + lane].order : 0;
    above += set_lanes(o > b);
    ties += set_lanes(o == b);
  }
  int upto = INT32_MAX;  // the largest id of a tie that stays
  if (ties > top - above) {
    ties = top - above;
    upto = 0;
#pragma unroll 1
    for (int bit = 24; bit >= 0; --bit) {
      const int t = upto | 1 << bit;
      int c = 0;
      for (int i = 0; i < n; i += 64) {
        const Entry e = i + lane < n ? list[i + lane] : Entry{0, 0};
        c += set_lanes(e.order == b && e.id < t);
      }
      if (c < ties) upto = t;
    }
  }
  int out = 0;
  for (int i = 0; i < n; i += 64) {
    const Entry e = i + lane < n ? list[i + lane] : Entry{0, 0};
    const bool in = e.order > b || (e.order == b && e.id <= upto);
    const uint64_t who = __ballot(in);
    if (in) list[out + __popcll(who & ((1ull << lane) - 1))] = e;
    out += __popcll(who);
  }
  return out;
}

// The entries of the block's lists (n[w] of wave w) in order: put(rank, entry) for the
// best `top`, Entry{0, -1} for ranks past their number.
template <class Put>
__device__ __forceinline__ void block_order(Entry (*lists)[kList], const int *n, int top, Put put) {
  int all = 0;
  for (int w = 0; w < kLpWaves; ++w) all += n[w];
  for (int i = threadIdx.x; i < all; i += kLpThreads) {
    int w = 0, j = i;
    while (j >= n[w]) j -= n[w++];
    const Entry e = lists[w][j];
    int rank = 0;
    for (int v = 0; v < kLpWaves; ++v)
      for (int k = 0; k < n[v]; ++k) {
        const Entry o = lists[v][k];
        rank += o.order > e.order || (o.order == e.order && o.id < e.id);
      }
    if (rank < top) put(rank, e);
  }
  for (int r = all + threadIdx.x; r < top; r += kLpThreads) put(r, Entry{0, -1});
}

// A row's token and its logit.
template <typename T>
struct Given {
  int id;       // -1: none, or outside the vocabulary
  float x;
  __device__ __forceinline__ Given(const LogprobArgs &a, int r) {
    id = a.tokens ? a.tokens[r] : -1;
    if ((uint32_t)id >= (uint32_t)a.vocab) id = -1;
    x = id < 0 ? NAN : to_f32(static_cast<const T *>(a.logits)[r * a.stride + id]);
  }
};

// A row's outputs, by one thread.
template <typename T>
__device__ __forceinline__ void store_row(const LogprobArgs &a, int r, const Given<T> &t,
                                          const Stats &s) {
  const bool none = s.m == -INFINITY;  // (s.s is then 0, or NaN)
  const float lse = log1pf(s.s);
  if (a.entropy) a.entropy[r] = none ? s.s : lse - s.w / (1.f + s.s);
  if (a.logprob)
    a.logprob[r] = s.s != s.s ? s.s : none || t.id < 0 ? -INFINITY : (t.x - s.m) - lse;
  if (a.rank) a.rank[r] = t.id < 0 || t.x != t.x ? -1 : s.ahead;
}
__device__ __forceinline__ void store_top(const LogprobArgs &a, int r, int rank, Entry e,
                                          const Stats &s) {
  const long at = (long)r * a.top + rank;
  if (a.top_id) a.top_id[at] = e.id;
  if (a.top_logprob)
    a.top_logprob[at] = s.s != s.s ? s.s : e.id < 0 ? -INFINITY : (value_of(e.order) - s.m) - log1pf(s.s);
}

// The next float up (NaN past infinity).
__device__ __forceinline__ float next_up(float x) {
  if (x == 0.f) return __uint_as_float(1);
  const uint32_t b = __float_as_uint(x);
  return x == INFINITY ? NAN : __uint_as_float(x > 0.f ? b + 1 : b - 1);
}

// Grid (segments, rows): `tiles` tiles of kLpWaves waves a segment.
template <typename T, bool TOP>
__global__ __launch_bounds__(kLpThreads) void k_logprobs(LogprobArgs a, int tiles, Stats *part,
                                                         Entry *best) {
  constexpr int VEC = 16 / sizeof(T), NP = kLpLane / VEC, STEP = kLpWaves * kLpTile;
  constexpr int LOW = sizeof(T) == 4 ? 0 : std::is_same<T, bf16>::value ? 16 : 13;
  typedef Pack<T, VEC> P;
  __shared__ Entry lists[TOP ? kLpWaves : 1][TOP ? kList : 1];
  __shared__ Stats stats[kLpWaves];
  __shared__ int sizes[kLpWaves];
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, r = blockIdx.y;
  const T *row = static_cast<const T *>(a.logits) + r * a.stride;
  const int beg = blockIdx.x * tiles * STEP + w * kLpTile;
  const int end = (int)min((long)a.vocab, (long)(blockIdx.x + 1) * tiles * STEP);
  const auto load = [&](int v0, P *p) {
    if (v0 + kLpTile <= a.vocab) {
#pragma unroll
      for (int k = 0; k < NP; ++k)
        p[k] = *reinterpret_cast<const P *>(row + v0 + (k * 64 + lane) * VEC);
    } else {
#pragma unroll
      for (int k = 0; k < NP; ++k)
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
          const int v = v0 + (k * 64 + lane) * VEC + j;
          p[k].v[j] = v < a.vocab ? row[v] : from_f32<T>(-INFINITY);
        }
    }
  };
  P raw[NP], next[NP];
  if (beg < end) load(beg, raw);
  const Given<T> t(a, r);
  const float after = next_up(t.x);
  Stats s{-INFINITY, 0.f, 0.f, 0};
  uint32_t bound = kNothing;
  int n = 0;
  for (int v0 = beg; v0 < end; v0 += STEP) {
    if (v0 + STEP < end) load(v0 + STEP, next);
    float x[kLpLane], top = -INFINITY;
#pragma unroll
    for (int i = 0; i < kLpLane; ++i) {
      x[i] = to_f32(raw[i / VEC].v[i % VEC]);
      top = fmaxf(top, x[i]);
    }
    float same = 0.f;  // entries that are the lane's largest, but for the one left out
    if (__any(top > s.m)) {
      if (top > s.m) {
        if (s.m > -INFINITY) {
          const float d = s.m - top, f = __expf(d), one = 1.f + s.s;
          s.w = f == 0.f ? 0.f : f * (s.w + one * d);
          s.s = f * one;
        }
        s.m = top;
        same = -1.f;
      }
    }
    const float m = s.m == -INFINITY ? 0.f : s.m;
    const bool here = t.id >= v0 && t.id < v0 + kLpTile;
    const float least = v0 > t.id ? after : t.x;
#pragma unroll
    for (int i = 0; i < kLpLane; ++i) {
      const float d = x[i] - m, e = __expf(d);
      same += d == 0.f ? 1.f : 0.f;
      s.s += d == 0.f ? 0.f : e;
      s.w += e * fmaxf(d, -200.f);  // (e is 0 there, also for -inf)
      s.ahead += x[i] >= least;
    }
    s.s += same;
    if (here) {  // (counted by >= above: those after the token, and itself, only if larger)
#pragma unroll
      for (int i = 0; i < kLpLane; ++i) {
        const int v = v0 + (i / VEC * 64 + lane) * VEC + i % VEC;
        s.ahead -= x[i] == t.x && v >= t.id;
      }
    }
    if constexpr (TOP) {
      const uint32_t o = order_of(top);
      if (__any(o > bound)) {
        const uint32_t b = wave_bound<LOW>(a.top, [&](uint32_t u) { return set_lanes(o >= u); });
        int more = 0;
#pragma unroll
        for (int i = 0; i < kLpLane; ++i) {
          const uint32_t u = order_of(x[i]);
          more += set_lanes(u >= b && u > bound);
        }
        if (n + more > kList) n = wave_cut<LOW>(lists[w], n, a.top, bound);
#pragma unroll
        for (int i = 0; i < kLpLane; ++i) {
          const uint32_t u = order_of(x[i]);
          const bool in = u >= b && u > bound;
          const uint64_t who = __ballot(in);
          if (in)
            lists[w][n + __popcll(who & ((1ull << lane) - 1))] = {
                u, v0 + (i / VEC * 64 + lane) * VEC + i % VEC};
          n += __popcll(who);
        }
        // (The lanes that reach b are `top` at least, unless b is the lowest candidate.)
        if (b > kNothing + 1) bound = max(bound, b);
        if (n >= 2 * a.top + 64) n = wave_cut<LOW>(lists[w], n, a.top, bound);
      }
    }
#pragma unroll
    for (int k = 0; k < NP; ++k) raw[k] = next[k];
  }
  s = over_wave(s);
  if constexpr (TOP) n = wave_cut<LOW>(lists[w], n, a.top, bound);
  if (lane == 0) {
    stats[w] = s;
    sizes[w] = n;
  }
  __syncthreads();
  s = joined(joined(stats[0], stats[1]), joined(stats[2], stats[3]));
  const long at = (long)r * gridDim.x + blockIdx.x;
  if (threadIdx.x == 0) {
    if (gridDim.x == 1)
      store_row(a, r, t, s);
    else
      part[at] = s;
  }
  if constexpr (TOP)
    block_order(lists, sizes, a.top, [&](int rank, Entry e) {
      if (gridDim.x == 1)
        store_top(a, r, rank, e, s);
      else
        best[at * a.top + rank] = e;
    });
}

template <typename T, bool TOP>
__global__ __launch_bounds__(kLpThreads) void k_logprobs_merge(LogprobArgs a, int segments,
                                                               const Stats *part,
                                                               const Entry *best) {
  __shared__ Entry lists[TOP ? kLpWaves : 1][TOP ? kList : 1];
  __shared__ int sizes[kLpWaves];
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, r = blockIdx.x;
  const Given<T> t(a, r);
  const Stats s = over_wave(lane < segments ? part[(long)r * segments + lane]
                                            : Stats{-INFINITY, 0.f, 0.f, 0});
  if (threadIdx.x == 0) store_row(a, r, t, s);
  if constexpr (TOP) {
    int n = 0;
    const Entry *row = best + (long)r * segments * a.top;
    const int all = segments * a.top;
    for (int i = w * 64; i < all; i += kLpThreads) {
      const Entry e = i + lane < all ? row[i + lane] : Entry{0, -1};
      const uint64_t who = __ballot(e.id >= 0);
      if (e.id >= 0) lists[w][n + __popcll(who & ((1ull << lane) - 1))] = e;
      n += __popcll(who);
    }
    uint32_t bound = 0;
    n = wave_cut<0>(lists[w], n, a.top, bound);
    if (lane == 0) sizes[w] = n;
    __syncthreads();
    block_order(lists, sizes, a.top, [&](int rank, Entry e) { store_top(a, r, rank, e, s); });
  }
}

struct Segments {
  int n, tiles;
};
Segments segments_of(int rows, int vocab) {
  const int step = kLpWaves * kLpTile, tiles = (vocab + step - 1) / step;
  const int want = std::max(1, std::min({(1024 + rows - 1) / rows, 64, tiles}));
  const int each = (tiles + want - 1) / want;
  return {(tiles + each - 1) / each, each};
}

template <typename T, bool TOP>
hipError_t launch_logprobs_as(const LogprobArgs &a, void *ws, hipStream_t s) {
  const Segments g = segments_of(a.rows, a.vocab);
  Stats *part = static_cast<Stats *>(ws);
  Entry *best = reinterpret_cast<Entry *>(part + (size_t)a.rows * g.n);
  k_logprobs<T, TOP><<<dim3(g.n, a.rows), kLpThreads, 0, s>>>(a, g.tiles, part, best);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || g.n == 1) return e;
  k_logprobs_merge<T, TOP><<<a.rows, kLpThreads, 0, s>>>(a, g.n, part, best);
  return hipGetLastError();
}

template <typename T>
hipError_t launch_logprobs_type(const LogprobArgs &a, void *ws, hipStream_t s) {
  return a.top ? launch_logprobs_as<T, true>(a, ws, s) : launch_logprobs_as<T, false>(a, ws, s);
}

}  // namespace

size_t logprobs_workspace_bytes(int rows, int vocab, int top) {
  return (size_t)rows * segments_of(rows, vocab).n * (sizeof(Stats) + top * sizeof(Entry));
}

hipError_t launch_logprobs(const LogprobArgs &a, int dtype, void *ws, hipStream_t s) {
  if (dtype == 0) return launch_logprobs_type<float>(a, ws, s);
  if (dtype == 1) return launch_logprobs_type<bf16>(a, ws, s);
  return launch_logprobs_type<f16>(a, ws, s);
}

}  // namespace vsr
