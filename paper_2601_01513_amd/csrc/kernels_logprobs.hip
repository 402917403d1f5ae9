// Log-probabilities of given tokens, with their ranks, the distribution's entropy and
// the most likely alternatives, in one read of the logits.
//
// For a row x with largest value m and d = x - m:
//   S' = sum over all but one largest of e^d,  W = sum of d e^d,
//   logprob[t] = x[t] - m - log1p(S'),  entropy = log1p(S') - W / (1 + S').
// The largest is left out of S' so that log1p keeps its relative accuracy where one token
// has nearly all the mass.
//
// A block takes a segment of a row, each of its waves 1024 entries of every 4096. A wave
// holds the largest value it has met, and a reference near it for the exponentials; most
// tiles have none as large, and pass without a word about the one left out. Lanes keep the
// largest of what they read, and of each span of tiles. The top-th largest of a block's 256
// is a bound that `top` entries reach, and the entries that do are in spans of lanes whose
// largest does (little more than `top` of them): these are read again for the candidates.
// Segments are merged by a second kernel.
//
// 512 rows of 152064 bf16 (156 MB) with 20 alternatives: 46 + 5 us, 39 without (4.0 TB/s:
// memory and the exponentials together); candidates kept inside the loop took 76 + 5. 3
// rows of 151936 fp32: 8 + 7, a launch's way twice.
#include <algorithm>
#include <type_traits>

#include "common.h"

namespace vsr {

namespace {

constexpr int kLpThreads = 256, kLpWaves = kLpThreads / 64;
constexpr int kLpLane = 16;                  // entries a lane and tile
constexpr int kLpTile = kLpLane * 64;        // entries a wave and tile
constexpr int kMaxTop = 64;
constexpr int kPad = 8;                      // keys read at once
constexpr int kMaxSegments = 64;
constexpr int kSpans = 16;                   // spans of tiles in a segment
constexpr int kRoom = kMaxTop + 64;          // candidates of a wave

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

// A candidate: its order above, the complement of its id below, so that the better of two
// is the larger. 0: none.
typedef uint64_t Key;
__device__ __forceinline__ Key key_of(uint32_t order, int id) { return (Key)order << 32 | (uint32_t)~id; }
__device__ __forceinline__ uint32_t order_in(Key k) { return (uint32_t)(k >> 32); }
__device__ __forceinline__ int id_in(Key k) { return k ? (int)~(uint32_t)k : -1; }

__device__ __forceinline__ int set_lanes(bool in) { return __popcll(__ballot(in)); }
__device__ __forceinline__ int lanes_before(uint64_t who) {
  return __builtin_amdgcn_mbcnt_hi((uint32_t)(who >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)who, 0));
}

// The lowest bits of an order that follow from the others, with values of type T.
template <typename T>
constexpr int low_bits() {
  return sizeof(T) == 4 ? 0 : std::is_same<T, bf16>::value ? 16 : 13;
}

// The largest bound that at least `want` of the values reach which count(b) counts (the
// same in every lane); the lowest candidate if there are fewer.
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

// The same of the values of a block's threads, one each.
template <int LOW>
__device__ __forceinline__ uint32_t block_bound(int want, uint32_t mine, uint32_t *all) {
  all[threadIdx.x] = mine;
  __syncthreads();
  uint32_t o[kLpWaves];
#pragma unroll
  for (int i = 0; i < kLpWaves; ++i) o[i] = all[i * 64 + (threadIdx.x & 63)];
  return wave_bound<LOW>(want, [&](uint32_t u) {
    int c = 0;
#pragma unroll
    for (int i = 0; i < kLpWaves; ++i) c += set_lanes(o[i] >= u);
    return c;
  });
}

// Leaves the `top` best of a wave's list of n > top, in the order they were in; returns
// the lowest order among them.
template <int LOW>
__device__ __forceinline__ uint32_t wave_cut(Key *list, int n, int top) {
  const int lane = threadIdx.x & 63;
  uint32_t b;
  if (n <= 128) {
    const uint32_t o0 = order_in(list[lane]), o1 = 64 + lane < n ? order_in(list[64 + lane]) : 0;
    b = wave_bound<LOW>(top, [&](uint32_t t) {
      return set_lanes(o0 >= t && lane < n) + set_lanes(o1 >= t);
    });
  } else {
    b = wave_bound<LOW>(top, [&](uint32_t t) {
      int c = 0;
      for (int i = 0; i < n; i += 64) c += set_lanes(i + lane < n && order_in(list[i + lane]) >= t);
      return c;
    });
  }
  int above = 0, ties = 0;
  for (int i = 0; i < n; i += 64) {
    const uint32_t o = i + lane < n ? order_in(list[i + lane]) : 0;
    above += set_lanes(o > b);
    ties += set_lanes(o == b);
  }
  uint32_t least = 0;  // the lowest complement of an id among the ties that stay
  if (ties > top - above) {
#pragma unroll 1
    for (int bit = 31; bit >= 0; --bit) {
      const uint32_t t = least | 1u << bit;
      int c = 0;
      for (int i = 0; i < n; i += 64) {
        const Key e = i + lane < n ? list[i + lane] : 0;
        c += set_lanes(order_in(e) == b && (uint32_t)e >= t);
      }
      if (c >= top - above) least = t;
    }
  }
  int out = 0;
  for (int i = 0; i < n; i += 64) {
    const Key e = i + lane < n ? list[i + lane] : 0;
    const bool in = e >= ((Key)b << 32 | least);
    const uint64_t who = __ballot(in);
    if (in) list[out + lanes_before(who)] = e;
    out += __popcll(who);
  }
  return b;
}

// The best `top` of the lists of a block's waves in order: put(rank, key), with key 0 for
// ranks past their number. Wave w's list has n[w] <= 64 keys, 0 up to the next multiple of
// kPad. A thread counts the keys above its own.
template <int LIST, class Put>
__device__ __forceinline__ void block_order(const Key (*lists)[LIST], const int *n, int top, Put put) {
  typedef Pack<Key, 2> Two;
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const Key e = lane < n[w] ? lists[w][lane] : 0;
  int rank = 0, all = 0;
#pragma unroll
  for (int v = 0; v < kLpWaves; ++v) {
    const int nv = n[v];
    all += nv;
#pragma unroll 1
    for (int k = 0; k < nv; k += kPad) {
      Two o[kPad / 2];
#pragma unroll
      for (int i = 0; i < kPad / 2; ++i) o[i] = *reinterpret_cast<const Two *>(&lists[v][k + 2 * i]);
#pragma unroll
      for (int i = 0; i < kPad / 2; ++i) rank += (o[i].v[0] > e) + (o[i].v[1] > e);
    }
  }
  if (e && rank < top) put(rank, e);
  if ((int)threadIdx.x >= all && (int)threadIdx.x < top) put(threadIdx.x, 0);
}

// A wave's list of n ready for block_order: its best if there are more than 64, and padded.
template <int LOW>
__device__ __forceinline__ int list_done(Key *list, int n, int top) {
  const int lane = threadIdx.x & 63;
  if (n > 64) {
    wave_cut<LOW>(list, n, top);
    n = top;
  }
  if (lane < kPad) list[n + lane] = 0;
  return n;
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
__device__ __forceinline__ void store_top(const LogprobArgs &a, int r, int rank, Key k,
                                          const Stats &s) {
  const long at = (long)r * a.top + rank;
  if (a.top_id) a.top_id[at] = id_in(k);
  if (a.top_logprob)
    a.top_logprob[at] = s.s != s.s ? s.s : k == 0 ? -INFINITY : (value_of(order_in(k)) - s.m) - log1pf(s.s);
}

// How far a wave's largest value may pass its reference: sums are scaled by less than
// e^-kRefLag at a time, so that the roundings of earlier scalings fade, however often a
// row rises.
constexpr float kRefLag = 4.f;

// The next float up (NaN past infinity).
__device__ __forceinline__ float next_up(float x) {
  if (x == 0.f) return __uint_as_float(1);
  const uint32_t b = __float_as_uint(x);
  return x == INFINITY ? NAN : __uint_as_float(x > 0.f ? b + 1 : b - 1);
}

// Grid (segments, rows): `tiles` tiles of kLpWaves waves a segment.
template <typename T, bool TOP>
__global__ __launch_bounds__(kLpThreads) void k_logprobs(LogprobArgs a, int tiles, Stats *part,
                                                         Key *best) {
  constexpr int VEC = 16 / sizeof(T), NP = kLpLane / VEC, STEP = kLpWaves * kLpTile;
  constexpr int LOW = low_bits<T>();
  typedef Pack<T, VEC> P;
  __shared__ __attribute__((aligned(16))) Key lists[TOP ? kLpWaves : 1][kRoom + kPad];
  __shared__ uint32_t peaks[kLpThreads];
  __shared__ uint16_t tops[TOP ? kSpans : 1][kLpThreads];  // upper half of a span's order
  __shared__ uint16_t found[TOP ? kLpWaves : 1][128];      // spans to read: lane, span
  __shared__ Stats stats[kLpWaves];
  __shared__ int sizes[kLpWaves];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r = blockIdx.y;
  const T *row = static_cast<const T *>(a.logits) + r * a.stride;
  const int beg = blockIdx.x * tiles * STEP + w * kLpTile;
  const int end = (int)min((long)a.vocab, (long)(blockIdx.x + 1) * tiles * STEP);
  const auto load = [&](int v0, P *p) __attribute__((always_inline)) {
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
  float m = -INFINITY;        // the wave's largest value
  float ref = -INFINITY;      // what its exponentials are relative to
  // The lane's share of S' and W relative to ref, a term a tile. (A term a column in 32 bits
  // made chains of 16 roundings a tile: 4096 equal terms were off by 8e-6 of their sum. Here
  // 32 bits take 6 roundings a tile and 64 the rest.)
  double sum = 0., wsum = 0.;
  int ahead = 0;              // the wave's
  float peak = -INFINITY;     // the lane's largest value
  float high = -INFINITY;     // that of the span
  const int span = (tiles + kSpans - 1) / kSpans;
  int turn = 0, at_span = 0;
  const auto tile = [&](int v0, const P *raw) __attribute__((always_inline)) {
    float x[kLpLane], top = -INFINITY;
#pragma unroll
    for (int i = 0; i < kLpLane; ++i) {
      x[i] = to_f32(raw[i / VEC].v[i % VEC]);
      top = fmaxf(top, x[i]);
    }
    const float least = v0 > t.id ? after : t.x;
    float part[4] = {}, wpart[4] = {};
    if (!__any(top >= m)) {
#pragma unroll
      for (int i = 0; i < kLpLane; ++i) {
        const float d = x[i] - ref, e = __expf(d);
        part[i % 4] += e;
        wpart[i % 4] += e * fmaxf(d, -200.f);  // (e is 0 there, also for -inf)
        ahead += set_lanes(x[i] >= least);
      }
    } else {
      float now = top;
#pragma unroll
      for (int d = 1; d < 64; d <<= 1) now = fmaxf(now, __shfl_xor(now, d));
      const bool out = now > m;
      if (out) {
        if (m > -INFINITY) {
          // Lane 0 takes in what was the largest so far.
          const float d = m - ref, e = lane == 0 ? __expf(d) : 0.f;
          sum += e;
          wsum += e * d;
        }
        if (now > ref + kRefLag) {
          // (From a reference of -inf there is nothing to carry over.)
          const float d = ref - now, f = __expf(d);
          wsum = f == 0.f ? 0. : f * (wsum + d * sum);
          sum *= f;
          ref = now;
        }
        m = now;
      }
      const float z = ref == -INFINITY ? 0.f : ref;
      int same = 0;
#pragma unroll
      for (int i = 0; i < kLpLane; ++i) {
        const float d = x[i] - z, e = x[i] == m ? 0.f : __expf(d);
        same += x[i] == m;
        part[i % 4] += e;
        wpart[i % 4] += e * fmaxf(d, -200.f);
        ahead += set_lanes(x[i] >= least);
      }
      const uint64_t who = __ballot(same > 0);
      if (m > -INFINITY) {
        // (NaN where the largest is infinite.)
        const bool left = out && who && lane == __builtin_ctzll(who);
        const float d = m - ref, e = __expf(d) * (float)(same - left);
        part[0] += e;
        wpart[0] += e * d;
      }
    }
    sum += (part[0] + part[1]) + (part[2] + part[3]);
    wsum += (wpart[0] + wpart[1]) + (wpart[2] + wpart[3]);
    if (t.id >= v0 && t.id < v0 + kLpTile) {
      // (Counted by >= above: those after the token, and itself, only if larger.)
#pragma unroll
      for (int i = 0; i < kLpLane; ++i) {
        const int v = v0 + (i / VEC * 64 + lane) * VEC + i % VEC;
        ahead -= set_lanes(x[i] == t.x && v >= t.id);
      }
    }
    if constexpr (TOP) {
      high = fmaxf(high, top);
      if (++turn == span || v0 + STEP >= end) {
        tops[at_span++][threadIdx.x] = (uint16_t)(order_of(high) >> 16);
        peak = fmaxf(peak, high);
        high = -INFINITY;
        turn = 0;
      }
    }
  };
  for (int v0 = beg; v0 < end; v0 += 2 * STEP) {
    if (v0 + STEP < end) load(v0 + STEP, next);
    tile(v0, raw);
    if (v0 + STEP >= end) break;
    if (v0 + 2 * STEP < end) load(v0 + 2 * STEP, raw);
    tile(v0 + STEP, next);
  }
  float S = (float)sum, W = (float)wsum;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    S += __shfl_xor(S, d);
    W += __shfl_xor(W, d);
  }
  if (m > ref) {  // (both finite)
    const float d = ref - m, f = __expf(d);
    W = f * (W + d * S);
    S *= f;
  }
  if (lane == 0) stats[w] = {m, S, W, ahead};
  if constexpr (TOP) {
    const uint32_t bound = block_bound<LOW>(a.top, order_of(peak), peaks);
    float lim = value_of(bound);
    int n = 0;
    uint16_t *mine_found = found[w];
    // Reads spans found[0..many): by lanes, or in the order of ids if all are one span.
    const auto collect = [&](int many) __attribute__((always_inline)) {
      const int per = NP * span, pieces = many * per;
      const bool one = mine_found[0] >> 6 == mine_found[many - 1] >> 6;
      uint32_t cut = 0;
#pragma unroll 1
      for (int u0 = 0; u0 < pieces; u0 += 64) {
        const int u = min(u0 + lane, pieces - 1), q = u / (one ? many : per);
        const int rest = u - q * (one ? many : per), f = mine_found[one ? rest : q];
        const int i = one ? q : rest;
        const int v = beg + ((f >> 6) * span + i / NP) * STEP + (i % NP * 64 + (f & 63)) * VEC;
        float x[VEC];
        if (u0 + lane < pieces && v + VEC <= end) {
          const P p = *reinterpret_cast<const P *>(row + v);
#pragma unroll
          for (int j = 0; j < VEC; ++j) x[j] = to_f32(p.v[j]);
        } else {
#pragma unroll
          for (int j = 0; j < VEC; ++j)
            x[j] = u0 + lane < pieces && v + j < end ? to_f32(row[v + j]) : -INFINITY;
        }
        int more = 0;
#pragma unroll
        for (int j = 0; j < VEC; ++j) more += set_lanes(x[j] >= lim);
        const auto append = [&](float y, int j) __attribute__((always_inline)) {
          const bool is = y >= lim;
          const uint64_t which = __ballot(is);
          if (is) lists[w][n + lanes_before(which)] = key_of(order_of(y), v + j);
          n += __popcll(which);
        };
        if (n + more <= kRoom) {
#pragma unroll
          for (int j = 0; j < VEC; ++j) append(x[j], j);
        } else {
#pragma unroll 1
          for (int j = 0; j < VEC; ++j) {
            if (n > kMaxTop) {
              cut = wave_cut<LOW>(lists[w], n, a.top);
              lim = fmaxf(lim, one && j == 0 ? next_up(value_of(cut)) : value_of(cut));
              n = a.top;
            }
            append(u0 + lane < pieces && v + j < end ? to_f32(row[v + j]) : -INFINITY, j);
          }
        }
      }
      // What comes has higher ids (and within one span, from turn to turn): it has to pass
      // the last of the best.
      if (cut) lim = fmaxf(lim, next_up(value_of(cut)));
    };
    int many = 0;
    for (int k = 0; k < at_span; ++k) {
      // (lim rises when a list was cut)
      const bool in = tops[k][threadIdx.x] >= (order_of(lim) >> 16);
      const uint64_t who = __ballot(in);
      if (in) mine_found[many + lanes_before(who)] = (uint16_t)(k << 6 | lane);
      many += __popcll(who);
      if (many >= 64) {
        collect(many);
        many = 0;
      }
    }
    if (many) collect(many);
    n = list_done<LOW>(lists[w], n, a.top);
    if (lane == 0) sizes[w] = n;
  }
  __syncthreads();
  const Stats s = joined(joined(stats[0], stats[1]), joined(stats[2], stats[3]));
  const long at = (long)r * gridDim.x + blockIdx.x;
  if (threadIdx.x == 0) {
    if (gridDim.x == 1)
      store_row(a, r, t, s);
    else
      part[at] = s;
  }
  if constexpr (TOP)
    block_order(lists, sizes, a.top, [&](int rank, Key k) {
      if (gridDim.x == 1)
        store_top(a, r, rank, k, s);
      else
        best[at * a.top + rank] = k;
    });
}

template <typename T, bool TOP>
__global__ __launch_bounds__(kLpThreads) void k_logprobs_merge(LogprobArgs a, int segments,
                                                               const Stats *part, const Key *best) {
  constexpr int MANY = kMaxTop * kMaxSegments / kLpThreads;
  __shared__ __attribute__((aligned(16))) Key lists[TOP ? kLpWaves : 1][64 * MANY + kPad];
  __shared__ uint32_t peaks[TOP ? kLpThreads : 1];
  __shared__ int sizes[kLpWaves];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r = blockIdx.x;
  const Given<T> t(a, r);
  Stats s{-INFINITY, 0.f, 0.f, 0};
  if (lane < segments) s = part[(long)r * segments + lane];
  if constexpr (TOP) {
    // As above: a thread holds up to MANY keys, of different ranks in their segments, and the
    // top-th largest of the threads' best is a bound.
    const Key *row = best + (long)r * segments * a.top;
    const int all = segments * a.top;
    Key keys[MANY], high = 0;
#pragma unroll
    for (int j = 0; j < MANY; ++j) {
      keys[j] = 0;
      if (j * kLpThreads >= all) continue;
      const int i = j * kLpThreads + ((threadIdx.x + 37 * j) & (kLpThreads - 1));
      if (i < all) keys[j] = row[i];
      high = max(high, keys[j]);
    }
    Key bound = 1;
    if (all > kLpThreads)
      bound = (Key)block_bound<low_bits<T>()>(a.top, order_in(high), peaks) << 32;
    int n = 0;
#pragma unroll
    for (int j = 0; j < MANY; ++j) {
      if (j * kLpThreads >= all) continue;
      const uint64_t who = __ballot(keys[j] >= bound);
      if (keys[j] >= bound) lists[w][n + lanes_before(who)] = keys[j];
      n += __popcll(who);
    }
    n = list_done<low_bits<T>()>(lists[w], n, a.top);
    if (lane == 0) sizes[w] = n;
  }
  for (int d = 1; d < segments; d <<= 1)
    s = joined(s, {__shfl_xor(s.m, d), __shfl_xor(s.s, d), __shfl_xor(s.w, d), __shfl_xor(s.ahead, d)});
  if (threadIdx.x == 0) store_row(a, r, t, s);
  if constexpr (TOP) {
    __syncthreads();
    // (Lane 0 has the statistics; in the others the order of the sum differs.)
    s.m = __shfl(s.m, 0), s.s = __shfl(s.s, 0);
    block_order(lists, sizes, a.top, [&](int rank, Key k) { store_top(a, r, rank, k, s); });
  }
}

// Segments to fill the chip four blocks a CU: for 512, 1024, 1280, 2048 blocks 48, 43, 51,
// 50 us (512 rows of 152064 bf16, 20 alternatives), 117, 117, 127, 128 (1024 rows, fp32).
struct Segments {
  int n, tiles;
};
Segments segments_of(int rows, int vocab) {
  const int step = kLpWaves * kLpTile, tiles = (vocab + step - 1) / step;
  const int want = std::max(1, std::min({(1024 + rows - 1) / rows, kMaxSegments, tiles}));
  const int each = (tiles + want - 1) / want;
  return {(tiles + each - 1) / each, each};
}

template <typename T, bool TOP>
hipError_t launch_logprobs_as(const LogprobArgs &a, void *ws, hipStream_t s) {
  const Segments g = segments_of(a.rows, a.vocab);
  Stats *part = static_cast<Stats *>(ws);
  Key *best = reinterpret_cast<Key *>(part + (size_t)a.rows * g.n);
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
  return (size_t)rows * segments_of(rows, vocab).n * (sizeof(Stats) + top * sizeof(Key));
}

hipError_t launch_logprobs(const LogprobArgs &a, int dtype, void *ws, hipStream_t s) {
  if (dtype == 0) return launch_logprobs_type<float>(a, ws, s);
  if (dtype == 1) return launch_logprobs_type<bf16>(a, ws, s);
  return launch_logprobs_type<f16>(a, ws, s);
}

}  // namespace vsr
