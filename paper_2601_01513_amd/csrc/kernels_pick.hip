// Greedy pick of a token per row of logits under rules: penalties for repeated
// tokens, a bias, a grammar mask; with the pick's log-probability.
//
// For row r and token v, c the number of v in the row's output list, "seen"
// whether v is in its prompt or output list:
//   l = logit;  seen: l = l > 0 ? l / repetition : l * repetition
//   l = l - (frequency c + presence [c > 0]);  l = l + bias[v]
//   mask bit clear: l = -inf
//   token = lowest v of the largest l (-1 if that is -inf);
//   logprob = l[token] - log sum_v exp(l[v])
//
// Bound by one read of the logits (and one write, where the processed logits
// are asked for). A block takes a chunk of one row's vocabulary: it counts the
// row's lists into an LDS table of the chunk (one word an entry: bit 31 "in the
// prompt", the rest the output count; integer atomics, so no order shows), holds
// the chunk's processed logits in registers and leaves (largest, its index,
// sum of the others' exp); a second small kernel merges a row's chunks.
//
// The sums leave the largest entry out: with S' = sum over the others of
// exp(l - max), logprob = -log1p(S') keeps its relative accuracy where one token
// has nearly all the mass (a Yes / No answer), where log(1 + S') would not.
#include <algorithm>

#include "common.h"

namespace vsr {

namespace {

__device__ __forceinline__ int wave_min_int(int v) {
  return __float_as_int(wave_reduce(__int_as_float(v), [](float x, float y) {
    return __int_as_float(min(__float_as_int(x), __float_as_int(y)));
  }));
}

// Largest value m, its lowest index i (INT32_MAX: every value was -inf, m is
// -inf) and the sum s of exp(l - m) over the other values (NaN if one was NaN).
struct Best {
  float m;
  int i;
  float s;
};

// What entry b adds to the sum of exp(l - m), m >= b.m; `own`: b holds the
// entry that m is, which is left out.
__device__ __forceinline__ float share(const Best &b, float m, bool own) {
  if (own) return b.s;
  return b.i == INT32_MAX ? b.s : (1.f + b.s) * __expf(b.m - m);
}

// Over the lanes of a wave, in every lane.
__device__ __forceinline__ Best wave_best(Best b) {
  const float m = wave_max(b.m);
  const int i = wave_min_int(b.m == m ? b.i : INT32_MAX);
  return {m, i, wave_sum(share(b, m, b.i == i))};
}

// Over a block of NT threads, valid in the first wave.
template <int NT>
__device__ __forceinline__ Best block_best(Best b, Best *red) {
  b = wave_best(b);
  if constexpr (NT > 64) {
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    if (lane == 0) red[w] = b;
    __syncthreads();
    b = lane < NT / 64 ? red[lane] : Best{-INFINITY, INT32_MAX, 0.f};
    if (w == 0) b = wave_best(b);
  }
  return b;
}

template <typename T, int VEC>
struct alignas(sizeof(T) * VEC) Pack {
  T v[VEC];
};

// Rounded as written (no fused multiply-add): the same values as the same
// steps in any fp32 arithmetic, so that equal logits stay equal.
__device__ __forceinline__ float penalised(float l, uint32_t c, float rep, float freq, float pres) {
#pragma clang fp contract(off)
  if (c == 0) return l;
  l = l > 0.f ? l / rep : l * rep;
  const uint32_t n = c & 0x7fffffffu;
  const float a = freq * (float)n, b = n ? pres : 0.f;
  const float p = a + b;
  return l - p;
}

// Grid (chunks, rows), NT threads, NV packs of VEC entries a thread. VEC > 1:
// every row of logits, bias and processed starts at 16 bytes. cnt: the chunk's
// table where the row has lists.
template <typename T, int VEC, int NV, int NT>
__global__ __launch_bounds__(NT) void k_pick_chunks(PickArgs a, int chunks, Best *part) {
  extern __shared__ uint32_t cnt[];
  __shared__ Best red[NT / 64];
  constexpr int C = NT * NV * VEC;
  const int tid = threadIdx.x, r = blockIdx.y;
  const int v0 = blockIdx.x * C;
  const T *logits = static_cast<const T *>(a.logits) + r * a.stride;

  // The chunk's logits are on their way while the lists are counted.
  float x[NV][VEC];
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    const int v = v0 + (k * NT + tid) * VEC;
    if (v + VEC <= a.vocab) {
      const Pack<T, VEC> p = *reinterpret_cast<const Pack<T, VEC> *>(logits + v);
#pragma unroll
      for (int j = 0; j < VEC; ++j) x[k][j] = to_f32(p.v[j]);
    } else {
#pragma unroll
      for (int j = 0; j < VEC; ++j) x[k][j] = v + j < a.vocab ? to_f32(logits[v + j]) : 0.f;
    }
  }

  const bool lists = a.prompt || a.output;
  if (lists) {
    for (int i = tid; i < C; i += NT) cnt[i] = 0;
    __syncthreads();
    const auto list = [&](const int32_t *ids, int n, bool output) {
#pragma unroll 4
      for (int i = tid; i < n; i += NT) {
        const uint32_t o = (uint32_t)ids[i] - (uint32_t)v0;
        if (o < (uint32_t)C) {
          if (output)
            atomicAdd(&cnt[o], 1u);
          else
            atomicOr(&cnt[o], 0x80000000u);
        }
      }
    };
    if (a.prompt)
      list(a.prompt + r * a.prompt_stride, min(a.prompt_len ? a.prompt_len[r] : a.n_prompt, a.n_prompt),
           false);
    if (a.output)
      list(a.output + r * a.output_stride, min(a.output_len ? a.output_len[r] : a.n_output, a.n_output),
           true);
    __syncthreads();
    const float rep = a.repetition ? a.repetition[r] : 1.f;
    const float freq = a.frequency ? a.frequency[r] : 0.f;
    const float pres = a.presence ? a.presence[r] : 0.f;
#pragma unroll
    for (int k = 0; k < NV; ++k)
#pragma unroll
      for (int j = 0; j < VEC; ++j)
        x[k][j] = penalised(x[k][j], cnt[(k * NT + tid) * VEC + j], rep, freq, pres);
  }

  const float *bias = a.bias ? a.bias + r * a.bias_stride : nullptr;
  const uint32_t *mask = a.mask ? a.mask + r * a.mask_stride : nullptr;
  float *out = a.processed ? a.processed + r * a.processed_stride : nullptr;
  Best b{-INFINITY, INT32_MAX, 0.f};
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    const int v = v0 + (k * NT + tid) * VEC;
    const bool whole = v + VEC <= a.vocab;
    if (bias) {
      if (whole) {
#pragma unroll
        for (int j0 = 0; j0 < VEC; j0 += 4) {
          constexpr int W = VEC < 4 ? VEC : 4;
          const Pack<float, W> p = *reinterpret_cast<const Pack<float, W> *>(bias + v + j0);
#pragma unroll
          for (int j = 0; j < W; ++j) x[k][j0 + j] += p.v[j];
        }
      } else {
#pragma unroll
        for (int j = 0; j < VEC; ++j)
          if (v + j < a.vocab) x[k][j] += bias[v + j];
      }
    }
    // (v is a multiple of VEC, so that a pack's bits lie in one word.)
    uint32_t bits = ~0u;
    if (mask && v < a.vocab) bits = mask[v >> 5] >> (v & 31);
#pragma unroll
    for (int j = 0; j < VEC; ++j)
      if (v + j >= a.vocab || !((bits >> j) & 1)) x[k][j] = -INFINITY;
    if (out) {
      if (whole) {
#pragma unroll
        for (int j0 = 0; j0 < VEC; j0 += 4) {
          constexpr int W = VEC < 4 ? VEC : 4;
          Pack<float, W> p;
#pragma unroll
          for (int j = 0; j < W; ++j) p.v[j] = x[k][j0 + j];
          *reinterpret_cast<Pack<float, W> *>(out + v + j0) = p;
        }
      } else {
#pragma unroll
        for (int j = 0; j < VEC; ++j)
          if (v + j < a.vocab) out[v + j] = x[k][j];
      }
    }
    // Entries come in index order, so a strict > keeps the lowest.
#pragma unroll
    for (int j = 0; j < VEC; ++j)
      if (x[k][j] > b.m) {
        b.m = x[k][j];
        b.i = v + j;
      }
  }
  if (a.logprob) {
    // (A thread left with nothing sums against 0: exp(-inf) = 0, and a NaN shows.)
    const float m = b.i == INT32_MAX ? 0.f : b.m;
#pragma unroll
    for (int k = 0; k < NV; ++k)
#pragma unroll
      for (int j = 0; j < VEC; ++j)
        b.s += v0 + (k * NT + tid) * VEC + j == b.i ? 0.f : __expf(x[k][j] - m);
  }
  b = block_best<NT>(b, red);
  if (tid == 0) part[(long)r * chunks + blockIdx.x] = b;
}

// One wave a row: a row has at most a few hundred chunks.
__global__ __launch_bounds__(64) void k_pick_merge(PickArgs a, int chunks, const Best *part) {
  const int r = blockIdx.x;
  Best b{-INFINITY, INT32_MAX, 0.f};
  for (int c = threadIdx.x; c < chunks; c += 64) {
    const Best p = part[(long)r * chunks + c];
    const bool first = p.m > b.m || (p.m == b.m && p.i < b.i);
    const Best &hi = first ? p : b, &lo = first ? b : p;
    b = {hi.m, hi.i, hi.s + share(lo, hi.m, false)};
  }
  b = wave_best(b);
  if (threadIdx.x == 0) {
    const bool none = b.i == INT32_MAX;
    const int token = none ? -1 : b.i;
    a.token[r * a.token_stride] = token;
    // b.m is +inf only where a logit was: the sum is then no number either.
    if (a.logprob)
      a.logprob[r * a.token_stride] = none ? (b.s != b.s ? b.s : -INFINITY)
                                           : (b.m == INFINITY ? NAN : -log1pf(b.s));
    if (a.next_ids) a.next_ids[r] = none ? 0 : token;
  }
}

constexpr int kPickMinChunk = 2048;  // the smallest chunk of any variant below

template <typename T, int VEC, int NV, int NT>
hipError_t launch_pick_chunks(const PickArgs &a, Best *part, hipStream_t s) {
  constexpr int C = NT * NV * VEC;
  const int chunks = (a.vocab + C - 1) / C;
  const size_t lds = a.prompt || a.output ? C * sizeof(uint32_t) : 0;
  k_pick_chunks<T, VEC, NV, NT><<<dim3(chunks, a.rows), NT, lds, s>>>(a, chunks, part);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  k_pick_merge<<<a.rows, 64, 0, s>>>(a, chunks, part);
  return hipGetLastError();
}

template <typename T>
hipError_t launch_pick_type(const PickArgs &a, Best *part, hipStream_t s) {
  constexpr int VEC = 16 / sizeof(T);
  const bool aligned =
      ((reinterpret_cast<uintptr_t>(a.logits) | reinterpret_cast<uintptr_t>(a.bias) |
        reinterpret_cast<uintptr_t>(a.processed) | (size_t)a.stride * sizeof(T) |
        (a.bias ? (size_t)a.bias_stride * 4 : 0) |
        (a.processed ? (size_t)a.processed_stride * 4 : 0)) &
       15) == 0;
  if (!aligned) return launch_pick_chunks<T, 1, 8, 256>(a, part, s);
  return launch_pick_chunks<T, VEC, 16 / VEC, 256>(a, part, s);
}

}  // namespace

size_t pick_workspace_bytes(int rows, int vocab) {
  return (size_t)rows * ((vocab + kPickMinChunk - 1) / kPickMinChunk) * sizeof(Best);
}

hipError_t launch_pick(const PickArgs &a, int dtype, void *ws, hipStream_t s) {
  if (a.rows == 0) return hipSuccess;
  Best *part = static_cast<Best *>(ws);
  if (dtype == 0) return launch_pick_type<float>(a, part, s);
  if (dtype == 1) return launch_pick_type<bf16>(a, part, s);
  return launch_pick_type<f16>(a, part, s);
}

}  // namespace vsr
