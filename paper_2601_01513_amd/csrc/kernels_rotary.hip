// Rotary positions with several axes and the RMSNorm of query and key heads,
// in one pass over the heads of a QKV projection.
//
// Head x of token t (head_dim values), pair i < rot / 2:
//   y = x / sqrt(mean(x^2) + eps) * gain            (norm form only)
//   angle = pos[axis(i)][t] * base^(-2 i / rot)
//   (out_i, out_{i + rot/2}) = (y_i cos - y_{i+rot/2} sin, y_{i+rot/2} cos + y_i sin)
// and out_d = y_d for d >= rot. Statistics and rotation are fp32; each output
// is rounded once to the tensors' type.
//
// The kernel reads and writes each head once and is bound by that traffic (the
// counters show no byte more written): 16384 tokens of 40 + 8 bf16 heads, 403 MB, take 71 us
// (5.7 TB/s; a bare copy of the same rows takes 71.5), 8192 with the norms 36 us, 4096
// tokens of 28 + 4 heads (in the caches) 12 us, 8192 of them in fp32 47 us (5.7 TB/s).
// Few tokens are bound by one round trip to memory and the launch: 3.1 us for a decode
// step's 8, 3.7 for 3 with norms.
//
// A head is handed to lph consecutive lanes of a wave (8 for head_dim 128 in 16
// bits): a lane holds VEC consecutive pairs, both halves, so that the rotation and
// the 16-byte loads and stores never leave the lane and the norm is a sum over
// lph lanes. An item, a wave's work at a time, is 64 / lph heads of a token, 2 KB;
// consecutive waves take consecutive items, so that all of them together walk
// through memory in order (a wave that took whole tokens touched as many rows at
// once as there are waves: 82 us). Angles are computed once a pair and item, a
// pair a lane, and handed round through LDS; each lane computing its own eight
// cost more registers than the loads in flight can spare.
//
// Angles: a turn is 1, so only the fraction of pos * base^(-2i/rot) / 2 pi
// matters. The product and its fraction are taken in fp64 (fp32 would lose the
// angle of the fast pairs past a few thousand positions); the fraction, in
// [-1/2, 1/2], keeps 24 bits.
#include <algorithm>
#include <cmath>

#include "common.h"

namespace vsr {

namespace {

typedef uint32_t u32x4u __attribute__((ext_vector_type(4), aligned(2)));

// Sum over groups of lph (a power of two) consecutive lanes, in every lane.
__device__ __forceinline__ float group_sum(float v, int lph) {
  if (lph > 1) v += row_rotated<0xB1>(v);   // lane ^ 1
  if (lph > 2) v += row_rotated<0x4E>(v);   // lane ^ 2
  if (lph > 4) v += row_rotated<0x141>(v);  // mirrored in 8: the other quad
  if (lph > 8) v += row_rotated<0x140>(v);  // mirrored in 16: the other half row
  if (lph > 16) {
    const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(a[0]) + __uint_as_float(a[1]);
  }
  if (lph > 32) {
    const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(a[0]) + __uint_as_float(a[1]);
  }
  return v;
}

// The axis of pair i in the map (2 bits a pair, 16 pairs a word).
__device__ __forceinline__ uint32_t axis_bits(const RotaryAxes &r, int i) {
  uint32_t w = r.map[0];
#pragma unroll
  for (int x = 1; x < kAxisWords; ++x) w = i >> 4 == x ? r.map[x] : w;
  return w >> (2 * (i & 15));
}

__device__ __forceinline__ float gain_at(const void *g, int dtype, int d) {
  if (dtype == 0) return static_cast<const float *>(g)[d];
  if (dtype == 1) return to_f32(static_cast<const bf16 *>(g)[d]);
  return to_f32(static_cast<const f16 *>(g)[d]);
}

// Orders a wave's LDS writes before the other lanes' reads (no instruction: a
// wave's LDS accesses run in order).
__device__ __forceinline__ void wave_sync() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// cos and sin of r turns, |r| <= 1/2. The 16-bit types take the vector unit's
// own sine (absolute error up to 2^-23.0 over all turns, sincospif's 2^-24.2: measured).
template <typename T>
__device__ __forceinline__ float2 turn(float r) {
  if constexpr (sizeof(T) == 2) {
    return make_float2(__builtin_amdgcn_cosf(r), __builtin_amdgcn_sinf(r));
  } else {
    float s, c;
    sincospif(2.f * r, &s, &c);
    return make_float2(c, s);
  }
}

// A kernel argument, in scalar registers from here on. Without it a choice
// between two arguments by lane becomes a load through a chosen address, in
// every item, ahead of the loads that need it.
template <typename V>
__device__ __forceinline__ V kept(V v) {
  asm volatile("" : "+s"(v));
  return v;
}

// One item: the heads h0 .. h0 + 64 / lph - 1 of token t. The items of
// consecutive waves are neighbours in memory.
//
// SPLIT: values are fp16 pairs value + remainder (in_lo, out_lo). TABLE: the
// angles are rows of a rotary table (row_pos[t], or t) instead of positions.
// pos, k_rows and row_pos are a's (apart from it, so that they may be taken to
// differ from what is written: scalar loads).
// WIDE: more than 64 pairs a head. Loads are unconditional, at clamped places: a
// load in a branch would have to arrive before the branch's end.
template <typename T, int VEC, bool WIDE, bool NORM, bool SPLIT, bool TABLE>
__global__ __launch_bounds__(256) void k_rotate_heads(RotateArgs a, const int32_t *__restrict__ pos,
                                                      const int32_t *__restrict__ k_rows,
                                                      const int32_t *__restrict__ row_pos) {
  constexpr int NCH = VEC == 1 && WIDE ? 2 : 1;  // chunks of VEC pairs a lane holds
  constexpr int NA = WIDE ? 2 : 1;               // angles a lane computes
  typedef Pack<T, VEC> P;
  __shared__ float gains[NORM ? 2 * 256 : 1];
  __shared__ float angle[4][2][64 * NA];  // each wave's cos and sin of its item's pairs
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  float *const cosv = angle[w][0], *const sinv = angle[w][1];
  const int half = a.hd / 2, rh = a.axes.rot / 2, th = half - rh;
  const int li = lane & (a.lph - 1), hpw = 64 / a.lph, hl = lane / a.lph;
  const int nq = a.q.n, H = nq + a.k.n;
  // Keys are addressed from the queries' pointer.
  const auto apart = [](const void *k, const void *q) {
    return kept((reinterpret_cast<intptr_t>(k) - reinterpret_cast<intptr_t>(q)) / (long)sizeof(T));
  };
  const T *const q_in = static_cast<const T *>(a.q.in), *const q_in_lo = static_cast<const T *>(a.q.in_lo);
  T *const q_out = static_cast<T *>(a.q.out), *const q_out_lo = static_cast<T *>(a.q.out_lo);
  const long k_in = apart(a.k.in, a.q.in), k_out = apart(a.k.out, a.q.out);
  const long k_in_lo = SPLIT ? apart(a.k.in_lo, a.q.in_lo) : 0;
  const long k_out_lo = SPLIT ? apart(a.k.out_lo, a.q.out_lo) : 0;
  const long q_its = kept(a.q.in_ts), q_ihs = kept(a.q.in_hs), q_ots = kept(a.q.out_ts),
             q_ohs = kept(a.q.out_hs), k_its = kept(a.k.in_ts), k_ihs = kept(a.k.in_hs),
             k_ots = kept(a.k.out_ts), k_ohs = kept(a.k.out_hs);

  // A lane's chunks of VEC pairs: `rot_chunks` of them over the pairs that turn, then
  // those over the pairs of dims >= rot, th apart. The last of each ends where its
  // pairs end, so that it repeats up to VEC - 1 of the chunk before it (`twice`:
  // read and written by both with the same values, summed once).
  int s0[NCH], lo[NCH], hi[NCH], twice[NCH];
  bool on[NCH];
#pragma unroll
  for (int c = 0; c < NCH; ++c) {
    const int ch = li + c * a.lph;
    const bool turns = ch < a.rot_chunks;
    const int i = (turns ? ch : ch - a.rot_chunks) * VEC, n = turns ? rh : th;
    const int i0 = min(i, n - VEC);
    on[c] = i < n;
    twice[c] = on[c] ? i - i0 : VEC;
    s0[c] = on[c] ? (turns ? i0 : rh + i0) : 0;
    lo[c] = on[c] ? (turns ? i0 : 2 * rh + i0) : 0;
    hi[c] = on[c] ? lo[c] + n : 0;
  }
  // The angles of an item are computed once a pair, lane l those of pairs l and l
  // + 64: the axis and the turns per position, base^(-2i/rot) / 2 pi (a product of
  // the powers of two in i), of each.
  double f[NA];
  const int32_t *axis[NA];
  if constexpr (!TABLE) {
#pragma unroll
    for (int e = 0; e < NA; ++e) {
      const int i = lane + 64 * e;
      f[e] = i < rh ? 0.15915494309189535 : 0.0;
#pragma unroll
      for (int b = 0; b < kStepBits; ++b) f[e] *= i >> b & 1 ? a.pair_step[b] : 1.0;
      axis[e] = pos + (axis_bits(a.axes, i) & 3) * a.pos_stride;
    }
  }

  // A wave's item, loaded ahead.
  struct Item {
    int t, h0;
    P v0[NCH], v1[NCH], w0[NCH], w1[NCH];
    int p[NA], krow;
    float2 cs[NA];
  };
  // (A lane's own load of the key row: a scalar one would hold up the LDS reads.
  // Without k_rows the load goes to rows that hold a word a token, unused: positions,
  // or, where token t takes table row t, the table's.)
  int zero = 0;
  asm volatile("" : "+v"(zero));
  const int32_t *const krows = k_rows    ? k_rows
                               : !TABLE  ? pos
                               : row_pos ? row_pos
                                         : reinterpret_cast<const int32_t *>(a.table);
  int nt, nh;  // the next item to load: token and step over its heads
  {
    const int first = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + w);
    nt = first / a.steps;
    nh = first % a.steps;
  }
  const auto load_next = [&](Item &it) {
    const int t = nt, h = nh * hpw + hl;
    it.t = t;
    it.h0 = nh * hpw;
    nt += a.next_t;
    nh += a.next_step;
    if (nh >= a.steps) {
      nh -= a.steps;
      ++nt;
    }
    const int tc = min(t, a.T - 1), hc = min(h, H - 1);
    const bool isq = hc < nq;
    long kin = tc;
    if constexpr (TABLE) {
      if (k_rows) kin = min(max(k_rows[tc], 0), (int)a.k_cap - 1);
    }
    it.krow = krows[tc + zero];
    const long in = isq ? tc * q_its + hc * q_ihs : k_in + kin * k_its + (hc - nq) * k_ihs;
#pragma unroll
    for (int e = 0; e < NA; ++e) {
      if constexpr (TABLE) {
        const long row = row_pos ? row_pos[tc] : tc;
        it.cs[e] = a.table[row * half + min(lane + 64 * e, half - 1)];
      } else {
        it.p[e] = axis[e][tc];
      }
    }
#pragma unroll
    for (int c = 0; c < NCH; ++c) {
      it.v0[c] = *reinterpret_cast<const P *>(q_in + in + lo[c]);
      it.v1[c] = *reinterpret_cast<const P *>(q_in + in + hi[c]);
      if constexpr (SPLIT) {
        const long in_lo = isq ? in : in - k_in + k_in_lo;
        it.w0[c] = *reinterpret_cast<const P *>(q_in_lo + in_lo + lo[c]);
        it.w1[c] = *reinterpret_cast<const P *>(q_in_lo + in_lo + hi[c]);
      }
    }
  };
  // Works on `it` and loads the next into it as soon as its values are out.
  const auto work = [&](Item &it) {
    const int t = it.t, h = it.h0 + hl;
    const bool isq = h < nq;
    int krow = k_rows ? it.krow : t;
    asm volatile("" : "+v"(krow));
    const bool st = h < H && (isq || (krow >= 0 && krow < a.k_cap));
    const long out = isq ? t * q_ots + h * q_ohs : (long)krow * k_ots + (h - nq) * k_ohs;
#pragma unroll
    for (int e = 0; e < NA; ++e) {
      float2 cs;
      if constexpr (TABLE) {
        cs = it.cs[e];
      } else {
        const double r = (double)it.p[e] * f[e];
        cs = turn<T>((float)(r - rint(r)));
      }
      cosv[lane + 64 * e] = cs.x;
      sinv[lane + 64 * e] = cs.y;
    }
    wave_sync();
    float x[NCH][2 * VEC];
    float ss = 0.f;
#pragma unroll
    for (int c = 0; c < NCH; ++c) {
#pragma unroll
      for (int j = 0; j < VEC; ++j) {
        x[c][j] = to_f32(it.v0[c].v[j]);
        x[c][VEC + j] = to_f32(it.v1[c].v[j]);
        if constexpr (SPLIT) {
          x[c][j] += to_f32(it.w0[c].v[j]);
          x[c][VEC + j] += to_f32(it.w1[c].v[j]);
        }
      }
    }
    if constexpr (NORM) {
      const auto add = [&](bool even) {
#pragma unroll
        for (int c = 0; c < NCH; ++c)
#pragma unroll
          for (int j = 0; j < VEC; ++j) {
            const float sq = x[c][j] * x[c][j] + x[c][VEC + j] * x[c][VEC + j];
            ss += even || j >= twice[c] ? sq : 0.f;
          }
      };
      if (a.uneven) {
        asm volatile("");  // (a branch, not the masks of both)
        add(false);
      } else {
        add(true);
      }
    }
    // The values are out of the item's registers before its next loads, so that
    // these need no others (copies at the loop's end would wait for them).
#pragma unroll
    for (int c = 0; c < NCH; ++c)
#pragma unroll
      for (int j = 0; j < 2 * VEC; ++j) asm volatile("" : "+v"(x[c][j]));
    __builtin_amdgcn_sched_barrier(0);
    load_next(it);
    if constexpr (NORM) {
      ss = group_sum(ss, a.lph);
      const float rs = 1.f / sqrtf(ss / (float)a.hd + a.eps);
      const float *g = gains + (isq ? 0 : 256);
#pragma unroll
      for (int c = 0; c < NCH; ++c)
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
          x[c][j] *= rs * g[lo[c] + j];
          x[c][VEC + j] *= rs * g[hi[c] + j];
        }
    }
#pragma unroll
    for (int c = 0; c < NCH; ++c) {
      if (!(st && on[c])) continue;
      P o0, o1, l0, l1;
#pragma unroll
      for (int j = 0; j < VEC; ++j) {
        const float cj = cosv[s0[c] + j], sj = sinv[s0[c] + j];
        float y0 = x[c][j] * cj - x[c][VEC + j] * sj;
        float y1 = x[c][VEC + j] * cj + x[c][j] * sj;
        if (th > 0 && s0[c] >= rh) {  // a dim >= rot meets no other, an infinity among them
          y0 = x[c][j];
          y1 = x[c][VEC + j];
        }
        if constexpr (TABLE) {
          const float scale = isq ? a.q_scale : 1.f;
          y0 *= scale;
          y1 *= scale;
        }
        o0.v[j] = from_f32<T>(y0);
        o1.v[j] = from_f32<T>(y1);
        if constexpr (SPLIT) {
          l0.v[j] = from_f32<T>(y0 - to_f32(o0.v[j]));
          l1.v[j] = from_f32<T>(y1 - to_f32(o1.v[j]));
        }
      }
      T *o = q_out + (out + (isq ? 0 : k_out));
      bool stored = false;
      if constexpr (sizeof(P) == 16) {
        if (a.past_caches) {
          asm volatile("");  // (both keep the compiler from merging this with the plain stores)
          __builtin_nontemporal_store(__builtin_bit_cast(u32x4u, o0),
                                      reinterpret_cast<u32x4u *>(o + lo[c]));
          __builtin_nontemporal_store(__builtin_bit_cast(u32x4u, o1),
                                      reinterpret_cast<u32x4u *>(o + hi[c]));
          asm volatile("");
          stored = true;
        }
      }
      if (!stored) {
        *reinterpret_cast<P *>(o + lo[c]) = o0;
        *reinterpret_cast<P *>(o + hi[c]) = o1;
      }
      if constexpr (SPLIT) {
        T *ol = q_out_lo + (out + (isq ? 0 : k_out_lo));
        *reinterpret_cast<P *>(ol + lo[c]) = l0;
        *reinterpret_cast<P *>(ol + hi[c]) = l1;
      }
    }
    wave_sync();
  };
  Item it;
  load_next(it);
  if constexpr (NORM) {
    for (int d = threadIdx.x; d < a.hd; d += 256) {
      gains[d] = gain_at(a.q.gain, a.gain_dtype, d);
      if (a.k.n) gains[256 + d] = gain_at(a.k.gain, a.gain_dtype, d);
    }
    __syncthreads();
  }
  while (it.t < a.T) work(it);
}

// Chunks of vec pairs over the pairs that turn and the others.
int rot_chunks(const RotateArgs &a, int vec) { return (a.axes.rot / 2 + vec - 1) / vec; }
int tail_chunks(const RotateArgs &a, int vec) {
  return ((a.hd - a.axes.rot) / 2 + vec - 1) / vec;
}

// Widest VEC (16 bytes at most) that the head's two parts have pairs for and a wave
// has lanes for.
int pair_width(const RotateArgs &a, size_t esize) {
  const int rh = a.axes.rot / 2, th = a.hd / 2 - rh;
  int vec = (int)(16 / esize);
  while (vec > 1 && (rh < vec || (th > 0 && th < vec) ||
                     rot_chunks(a, vec) + tail_chunks(a, vec) > 64))
    vec /= 2;
  return vec;
}

template <typename T, int VEC, bool WIDE, bool NORM, bool SPLIT, bool TABLE>
hipError_t launch_wide(RotateArgs a, hipStream_t s) {
  a.rot_chunks = rot_chunks(a, VEC);
  const int chunks = a.rot_chunks + tail_chunks(a, VEC);
  for (int b = 0; b < kStepBits; ++b) a.pair_step[b] = std::exp2(-a.log2_step * (1 << b));
  a.lph = 1;
  while (a.lph < chunks && a.lph < 64) a.lph *= 2;
  a.uneven = a.axes.rot / 2 % VEC || (a.hd - a.axes.rot) / 2 % VEC || chunks % a.lph;
  const int hpw = 64 / a.lph;
  a.steps = (a.q.n + a.k.n + hpw - 1) / hpw;
  // Three blocks a CU: more keep more of the memory's rows open than it likes (16384
  // tokens of 48 heads: 76.7 us, 79.1 with four, 82 with eight), fewer wait on loads
  // (4096 tokens of 32 heads: 12.0 us, 12.4 with two).
  const unsigned blocks = (unsigned)std::min(((long)a.T * a.steps + 3) / 4, 768L);
  // What no cache holds until its reader comes is written past them (the same 16384
  // tokens: 71.4 us; 8192 with their norms: 40.9 -> 37.8, and with a copy of the queries
  // after it 73.3 -> 68.1; but 4096 tokens of 32 heads with that reader 23.4 -> 25.0).
  a.past_caches = (long)a.T * (a.q.n + a.k.n) * a.hd * sizeof(T) > kCachedBytes;
  a.next_t = blocks * 4 / a.steps;
  a.next_step = blocks * 4 % a.steps;
  k_rotate_heads<T, VEC, WIDE, NORM, SPLIT, TABLE>
      <<<blocks, 256, 0, s>>>(a, a.pos, a.k_rows, a.row_pos);
  return hipGetLastError();
}

template <typename T, int VEC, bool NORM, bool SPLIT, bool TABLE>
hipError_t launch_vec(const RotateArgs &a, hipStream_t s) {
  if (a.hd > 128) return launch_wide<T, VEC, true, NORM, SPLIT, TABLE>(a, s);
  return launch_wide<T, VEC, false, NORM, SPLIT, TABLE>(a, s);
}

template <typename T, bool NORM>
hipError_t launch_type(const RotateArgs &a, hipStream_t s) {
  switch (pair_width(a, sizeof(T))) {
    case 8:
      if constexpr (sizeof(T) == 2) return launch_vec<T, 8, NORM, false, false>(a, s);
      return hipErrorInvalidValue;
    case 4: return launch_vec<T, 4, NORM, false, false>(a, s);
    case 2: return launch_vec<T, 2, NORM, false, false>(a, s);
    default: return launch_vec<T, 1, NORM, false, false>(a, s);
  }
}

// Rotary table of a prefix with positions on several axes, as k_rope_table:
// row p < P holds the angles of prefix row p, row p >= P those of a row at
// position next + p - P on every axis (the candidates' rows).
__global__ void k_rope_axes_table(float2 *cs, int npos, RotaryAxes axes, double base,
                                  const int32_t *pos, long pos_stride, int P, int next) {
  const int half = axes.rot / 2;
  const long idx = (long)blockIdx.x * blockDim.x + threadIdx.x;
  if (idx >= (long)npos * half) return;
  const int p = (int)(idx / half), i = (int)(idx % half);
  const long at = p < P ? pos[(axis_bits(axes, i) & 3) * pos_stride + p] : (long)next + (p - P);
  const double ang = (double)at * pow(base, -2.0 * i / axes.rot);
  cs[idx] = make_float2((float)cos(ang), (float)sin(ang));
}

__global__ void k_no_turn(int32_t *zero_pos, long n, float2 *row, int half) {
  const long i = (long)blockIdx.x * blockDim.x + threadIdx.x;
  if (i < n) zero_pos[i] = 0;
  if (i < half) row[i] = make_float2(1.f, 0.f);
}

}  // namespace

hipError_t launch_no_turn(int32_t *zero_pos, long n, float2 *row, int half, hipStream_t s) {
  const long work = std::max(n, (long)half);
  k_no_turn<<<(unsigned)((work + 255) / 256), 256, 0, s>>>(zero_pos, n, row, half);
  return hipGetLastError();
}

hipError_t launch_rope_axes_table(float2 *cs, int npos, const RotaryAxes &axes, float base,
                                  const int32_t *pos, long pos_stride, int P, int next,
                                  hipStream_t s) {
  const long n = (long)npos * (axes.rot / 2);
  k_rope_axes_table<<<(unsigned)((n + 255) / 256), 256, 0, s>>>(cs, npos, axes, (double)base, pos,
                                                                pos_stride, P, next);
  return hipGetLastError();
}

hipError_t launch_norm_cached(const RotateArgs &a, bool f32, hipStream_t s) {
  if (a.T == 0) return hipSuccess;
  if (!f32)  // (head_dim 128; the workspace's planes are 256-byte aligned)
    return a.q.in_lo ? launch_wide<f16, 8, false, true, true, true>(a, s)
                     : launch_wide<f16, 8, false, true, false, true>(a, s);
  return a.hd >= 8 ? launch_vec<float, 4, true, false, true>(a, s)
                   : launch_vec<float, 1, true, false, true>(a, s);
}

hipError_t launch_rotate_heads(const RotateArgs &a, int dtype, bool norm, hipStream_t s) {
  if (a.T == 0) return hipSuccess;
  if (dtype == 0) return norm ? launch_type<float, true>(a, s) : launch_type<float, false>(a, s);
  if (dtype == 1) return norm ? launch_type<bf16, true>(a, s) : launch_type<bf16, false>(a, s);
  return norm ? launch_type<f16, true>(a, s) : launch_type<f16, false>(a, s);
}

}  // namespace vsr
