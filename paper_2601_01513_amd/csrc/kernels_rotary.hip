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
// The kernel reads and writes each head once and is bound by that traffic. A
// head is handed to lph consecutive lanes of a wave (8 for head_dim 128 in 16
// bits): a lane holds VEC consecutive pairs, both halves, so the rotation and
// the loads and stores of 16 bytes never leave the lane and the norm is a sum
// over lph lanes. A wave takes 64 / lph heads of one token at a time.
//
// Angles: a turn is 1, so only the fraction of pos * base^(-2i/rot) / 2 pi
// matters. The product and its fraction are taken in fp64 (fp32 would lose the
// angle of the fast pairs past a few thousand positions); the fraction, in
// [-1/2, 1/2], keeps 24 bits.
#include <algorithm>

#include "common.h"

namespace vsr {

namespace {

template <typename T, int VEC>
struct alignas(sizeof(T) * VEC) Pack {
  T v[VEC];
};

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

// The axis that turns pair i: consecutive sections, or axes in turn (pair i
// belongs to axis i % n while that axis has pairs left, else to axis 0).
__device__ __forceinline__ int pair_axis(const RotaryAxes &r, int i) {
  if (r.interleaved) {
    const int a = i % r.n_axes;
    return i < r.n_axes * r.sections[a] ? a : 0;
  }
  int a = 0, end = r.sections[0];
  while (a + 1 < r.n_axes && i >= end) end += r.sections[++a];
  return a;
}

__device__ __forceinline__ float gain_at(const void *g, int dtype, int d) {
  if (dtype == 0) return static_cast<const float *>(g)[d];
  if (dtype == 1) return to_f32(static_cast<const bf16 *>(g)[d]);
  return to_f32(static_cast<const f16 *>(g)[d]);
}

// cos and sin of r turns, |r| <= 1/2. The 16-bit types take the vector unit's
// own sine (absolute error below 2^-20, measured), far under their rounding.
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

// SPLIT: values are fp16 pairs value + remainder (in_lo, out_lo). TABLE: the
// angles are rows of a rotary table (row_pos[t], or t) instead of positions.
template <typename T, int VEC, bool NORM, bool SPLIT, bool TABLE>
__global__ __launch_bounds__(256) void k_rotate_heads(RotateArgs a) {
  constexpr int NCH = VEC == 1 ? 2 : 1;  // chunks of VEC pairs a lane holds
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (threadIdx.x >> 6));
  const int nwaves = gridDim.x * 4;
  const int half = a.hd / 2, rh = a.axes.rot / 2, th = half - rh;
  const int li = lane & (a.lph - 1), hpw = 64 / a.lph;
  const int H = a.q.n + a.k.n;

  // What a lane keeps for all its tokens: its pairs' places in a head, turns
  // per position, axes and gains.
  int lo[NCH], hi[NCH];
  bool on[NCH];
  double f[NCH][VEC];
  int ax[NCH];  // 2 bits a pair
  float gq[NCH][2 * VEC], gk[NCH][2 * VEC];
#pragma unroll
  for (int c = 0; c < NCH; ++c) {
    const int s0 = (li + c * a.lph) * VEC;
    on[c] = s0 < half;
    lo[c] = s0 < rh ? s0 : s0 + rh;  // the tail dims >= rot go in pairs th apart
    hi[c] = s0 < rh ? s0 + rh : s0 + rh + th;
    ax[c] = 0;
    if constexpr (!TABLE) {
      const double f0 = on[c] && s0 < rh ? exp2(-s0 * a.log2_step) * 0.15915494309189535 : 0.0;
#pragma unroll
      for (int j = 0; j < VEC; ++j) {
        f[c][j] = j == 0 ? f0 : f[c][j - 1] * a.step;
        if (on[c] && s0 < rh) ax[c] |= pair_axis(a.axes, s0 + j) << (2 * j);
      }
    }
    if constexpr (NORM) {
#pragma unroll
      for (int j = 0; j < VEC; ++j) {
        gq[c][j] = on[c] ? gain_at(a.q.gain, a.gain_dtype, lo[c] + j) : 0.f;
        gq[c][VEC + j] = on[c] ? gain_at(a.q.gain, a.gain_dtype, hi[c] + j) : 0.f;
        gk[c][j] = on[c] && a.k.n ? gain_at(a.k.gain, a.gain_dtype, lo[c] + j) : 0.f;
        gk[c][VEC + j] = on[c] && a.k.n ? gain_at(a.k.gain, a.gain_dtype, hi[c] + j) : 0.f;
      }
    }
  }

  for (int u = wave; u < a.T * a.nsplit; u += nwaves) {
    const int t = u / a.nsplit, part = u % a.nsplit;
    const long krow = a.k_rows ? a.k_rows[t] : t;
    const bool kkeep = !a.k_rows || (krow >= 0 && krow < a.k_cap);
    const long kin = a.k_rows_in && kkeep ? krow : t;
    float2 cs[NCH][VEC];
    if constexpr (TABLE) {
      const float2 *row = a.table + (long)(a.row_pos ? a.row_pos[t] : t) * half;
#pragma unroll
      for (int c = 0; c < NCH; ++c)
#pragma unroll
        for (int j = 0; j < VEC; ++j)
          cs[c][j] = on[c] ? row[lo[c] + j] : make_float2(1.f, 0.f);
    } else {
      int p[kMaxAxes];
#pragma unroll
      for (int x = 0; x < kMaxAxes; ++x)
        p[x] = x < a.axes.n_axes ? a.pos[x * a.pos_stride + t] : 0;
#pragma unroll
      for (int c = 0; c < NCH; ++c)
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
          const int x = (ax[c] >> (2 * j)) & 3;
          const int pj = x == 0 ? p[0] : x == 1 ? p[1] : x == 2 ? p[2] : p[3];
          const double r = (double)pj * f[c][j];
          cs[c][j] = turn<T>((float)(r - rint(r)));
        }
    }
    for (int h0 = part * hpw; h0 < H; h0 += a.nsplit * hpw) {
      const int h = h0 + lane / a.lph;
      const bool isq = h < a.q.n;
      const bool have = h < H;
      const int hh = isq ? h : h - a.q.n;
      const long in = isq ? t * a.q.in_ts + hh * a.q.in_hs : kin * a.k.in_ts + hh * a.k.in_hs;
      const long out = isq ? t * a.q.out_ts + hh * a.q.out_hs : krow * a.k.out_ts + hh * a.k.out_hs;
      const T *xin = static_cast<const T *>(isq ? a.q.in : a.k.in) + in;
      const T *xin_lo = SPLIT ? static_cast<const T *>(isq ? a.q.in_lo : a.k.in_lo) + in : nullptr;
      float x[NCH][2 * VEC];
      float ss = 0.f;
#pragma unroll
      for (int c = 0; c < NCH; ++c) {
        const bool ld = have && on[c];
        Pack<T, VEC> v0{}, v1{};
        if (ld) {
          v0 = *reinterpret_cast<const Pack<T, VEC> *>(xin + lo[c]);
          v1 = *reinterpret_cast<const Pack<T, VEC> *>(xin + hi[c]);
        }
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
          x[c][j] = to_f32(v0.v[j]);
          x[c][VEC + j] = to_f32(v1.v[j]);
        }
        if constexpr (SPLIT) {
          if (ld) {
            v0 = *reinterpret_cast<const Pack<T, VEC> *>(xin_lo + lo[c]);
            v1 = *reinterpret_cast<const Pack<T, VEC> *>(xin_lo + hi[c]);
          }
#pragma unroll
          for (int j = 0; j < VEC; ++j) {
            x[c][j] += ld ? to_f32(v0.v[j]) : 0.f;
            x[c][VEC + j] += ld ? to_f32(v1.v[j]) : 0.f;
          }
        }
        if constexpr (NORM) {
#pragma unroll
          for (int j = 0; j < 2 * VEC; ++j) ss += x[c][j] * x[c][j];
        }
      }
      if constexpr (NORM) {
        ss = group_sum(ss, a.lph);
        const float rs = 1.f / sqrtf(ss / (float)a.hd + a.eps);
#pragma unroll
        for (int c = 0; c < NCH; ++c)
#pragma unroll
          for (int j = 0; j < 2 * VEC; ++j) x[c][j] *= rs * (isq ? gq[c][j] : gk[c][j]);
      }
      const bool st = have && (isq || kkeep);
#pragma unroll
      for (int c = 0; c < NCH; ++c) {
        Pack<T, VEC> v0, v1, w0, w1;
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
          float y0 = x[c][j] * cs[c][j].x - x[c][VEC + j] * cs[c][j].y;
          float y1 = x[c][VEC + j] * cs[c][j].x + x[c][j] * cs[c][j].y;
          if (th > 0 && lo[c] >= rh) {  // a dim >= rot meets no other, an infinity among them
            y0 = x[c][j];
            y1 = x[c][VEC + j];
          }
          if constexpr (TABLE) {
            const float scale = isq ? a.q_scale : 1.f;
            y0 *= scale;
            y1 *= scale;
          }
          v0.v[j] = from_f32<T>(y0);
          v1.v[j] = from_f32<T>(y1);
          if constexpr (SPLIT) {
            w0.v[j] = from_f32<T>(y0 - to_f32(v0.v[j]));
            w1.v[j] = from_f32<T>(y1 - to_f32(v1.v[j]));
          }
        }
        if (st && on[c]) {
          T *o = static_cast<T *>(isq ? a.q.out : a.k.out) + out;
          *reinterpret_cast<Pack<T, VEC> *>(o + lo[c]) = v0;
          *reinterpret_cast<Pack<T, VEC> *>(o + hi[c]) = v1;
          if constexpr (SPLIT) {
            T *ol = static_cast<T *>(isq ? a.q.out_lo : a.k.out_lo) + out;
            *reinterpret_cast<Pack<T, VEC> *>(ol + lo[c]) = w0;
            *reinterpret_cast<Pack<T, VEC> *>(ol + hi[c]) = w1;
          }
        }
      }
    }
  }
}

// Widest VEC (16 bytes at most) that the head's two parts and every address
// allow.
int pair_width(const RotateArgs &a, size_t esize) {
  const int rh = a.axes.rot / 2, th = a.hd / 2 - rh;
  for (int vec = (int)(16 / esize); vec > 1; vec /= 2) {
    const size_t bytes = vec * esize;
    bool ok = rh % vec == 0 && th % vec == 0;
    for (const HeadSet *s : {&a.q, &a.k}) {
      if (!s->n) continue;
      for (const void *p : {s->in, s->in_lo, (const void *)s->out, (const void *)s->out_lo})
        ok = ok && reinterpret_cast<uintptr_t>(p) % bytes == 0;
      for (long st : {s->in_ts, s->in_hs, s->out_ts, s->out_hs}) ok = ok && st % vec == 0;
    }
    if (ok) return vec;
  }
  return 1;
}

template <typename T, int VEC, bool NORM, bool SPLIT, bool TABLE>
hipError_t launch_vec(RotateArgs a, hipStream_t s) {
  const int chunks = a.hd / 2 / VEC;
  a.lph = 1;
  while (a.lph < chunks && a.lph < 64) a.lph *= 2;
  const int hpw = 64 / a.lph, steps = (a.q.n + a.k.n + hpw - 1) / hpw;
  // Few tokens: a wave for each step over the heads, so that the call is one
  // load's latency long. Many: a wave takes whole tokens and computes their
  // angles once.
  a.nsplit = (long)a.T * steps <= 4096 ? steps : 1;
  const long units = (long)a.T * a.nsplit;
  const unsigned blocks = (unsigned)std::min<long>((units + 3) / 4, 2048);
  k_rotate_heads<T, VEC, NORM, SPLIT, TABLE><<<blocks, 256, 0, s>>>(a);
  return hipGetLastError();
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
  const long at = p < P ? pos[pair_axis(axes, i) * pos_stride + p] : (long)next + (p - P);
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
    return a.q.in_lo ? launch_vec<f16, 8, true, true, true>(a, s)
                     : launch_vec<f16, 8, true, false, true>(a, s);
  return pair_width(a, 4) == 4 ? launch_vec<float, 4, true, false, true>(a, s)
                               : launch_vec<float, 1, true, false, true>(a, s);
}

hipError_t launch_rotate_heads(const RotateArgs &a, int dtype, bool norm, hipStream_t s) {
  if (a.T == 0) return hipSuccess;
  if (dtype == 0) return norm ? launch_type<float, true>(a, s) : launch_type<float, false>(a, s);
  if (dtype == 1) return norm ? launch_type<bf16, true>(a, s) : launch_type<bf16, false>(a, s);
  return norm ? launch_type<f16, true>(a, s) : launch_type<f16, false>(a, s);
}

}  // namespace vsr
