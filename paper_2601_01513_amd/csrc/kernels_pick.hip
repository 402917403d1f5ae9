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
// Bound by one read of the logits (and of the bias, and one write where the
// processed logits are asked for): 256 rows of 152064 fp32 logits with every rule, a bias a
// row and the result kept, 472 MB, take 87 us (5.4 TB/s). Few rows are bound by two
// launches and the steps between loads: 3 rows 6.9 us, 1 masked row 5.3. Long lists
// are bound by their scans, one in every chunk: 16 rows with lists of 4600 11 us, for
// 2.7 us of bytes. Many 16-bit rows without rules are bound by the launch of their
// waves, 1 KB each: 256 rows of 152064 bf16 30 us, for 14 us of bytes.
//
// A block takes a chunk of one row's vocabulary: its loads go out first, then it
// counts the row's lists into an LDS table of the chunk (one word an entry: bit 31
// "in the prompt", the rest the output count; integer atomics, so no order shows),
// holds the chunk's processed logits in registers and leaves (largest, its index,
// sum of the others' exp); a second small kernel merges a row's chunks. Every block of
// a row reads its lists, so chunks are as large as a few rows can bear: 4096
// entries (256 rows 91.7 us with plain stores, against 98 with 1024, 99 with 8192 and
// 102 with 16384 entries; 3 rows 7.2, 6.8, 7.8 and 10.2).
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

typedef float f32x4u __attribute__((ext_vector_type(4), aligned(4)));

// Rounded as written (no fused multiply-add): the same values as the same
// steps in any fp32 arithmetic, so that equal logits stay equal.
__device__ __forceinline__ float penalised(float l, uint32_t c, float rep, float freq, float pres) {
#pragma clang fp contract(off)
  const float t = l > 0.f ? l / rep : l * rep;
  const uint32_t n = c & 0x7fffffffu;
  const float a = freq * (float)n, b = n ? pres : 0.f;
  const float p = a + b;
  return c ? t - p : l;
}

// A row's outputs, by one thread.
__device__ __forceinline__ void finish_row(const PickArgs &a, int r, const Best &b) {
  const bool none = b.i == INT32_MAX;
  const int token = none ? -1 : b.i;
  a.token[r * a.token_stride] = token;
  // b.m is +inf only where a logit was: the sum is then no number either.
  if (a.logprob)
    a.logprob[r * a.token_stride] = none ? (b.s != b.s ? b.s : -INFINITY)
                                         : (b.m == INFINITY ? NAN : -log1pf(b.s));
  if (a.next_ids) a.next_ids[r] = none ? 0 : token;
}

// Grid (chunks, rows), NT threads, NV packs of VEC entries (16 bytes of logits) a
// thread; cnt: the chunk's table where the row has lists.
template <typename T, int NV, int NT>
__global__ __launch_bounds__(NT) void k_pick_chunks(PickArgs a, Best *part) {
  extern __shared__ __align__(16) uint32_t cnt[];
  __shared__ Best red[NT / 64];
  constexpr int VEC = 16 / sizeof(T), C = NT * NV * VEC;
  typedef Pack<T, VEC> P;
  typedef Pack<float, 4> P4;
  const int tid = threadIdx.x, r = blockIdx.y;
  const int v0 = blockIdx.x * C;
  const T *logits = static_cast<const T *>(a.logits) + r * a.stride;
  const float *bias = a.bias ? a.bias + r * a.bias_stride : nullptr;
  const uint32_t *mask = a.mask ? a.mask + r * a.mask_stride : nullptr;

  // The lists, four ids a load (16 rows with lists of 4600: 12.0 -> 11.3 us), the last
  // load moved back to end with the list. The first of each goes out before all else, so that
  // counting does not wait for the logits.
  typedef Pack<int32_t, 4> I4;
  const auto length = [&](const int32_t *list, const int32_t *len, int most) {
    return !list ? 0 : len ? max(0, min(len[r], most)) : most;
  };
  const int32_t *prompt = a.prompt + r * a.prompt_stride, *output = a.output + r * a.output_stride;
  const int np = length(a.prompt, a.prompt_len, a.n_prompt);
  const int no = length(a.output, a.output_len, a.n_output);
  const auto ids_at = [](const int32_t *ids, int n, int i) {
    if (n >= 4) return *reinterpret_cast<const I4 *>(ids + min(i, n - 4));
    I4 p;
#pragma unroll
    for (int j = 0; j < 4; ++j) p.v[j] = j < n ? ids[j] : -1;
    return p;
  };
  I4 first_p, first_o;
  if (4 * tid < np) first_p = ids_at(prompt, np, 4 * tid);
  if (4 * tid < no) first_o = ids_at(output, no, 4 * tid);

  // Everything else the chunk reads is on its way before the lists are counted. Loads
  // past the row's end are moved back inside it (the pack the end cuts through is
  // read again below, the rest is not used).
  const auto at = [&](int k) { return v0 + (k * NT + tid) * VEC; };
  const auto inside = [&](int k) { return min(at(k), a.vocab - VEC); };
  P raw[NV];
  P4 add[NV][VEC / 4];
  uint32_t bits[NV];
  const bool wide = a.vocab >= VEC;
  if (wide) {
#pragma unroll
    for (int k = 0; k < NV; ++k) raw[k] = *reinterpret_cast<const P *>(logits + inside(k));
    if (bias) {
#pragma unroll
      for (int k = 0; k < NV; ++k)
#pragma unroll
        for (int j = 0; j < VEC / 4; ++j)
          add[k][j] = *reinterpret_cast<const P4 *>(bias + inside(k) + 4 * j);
    }
  }
  if (mask) {
#pragma unroll
    for (int k = 0; k < NV; ++k) bits[k] = mask[min(at(k), a.vocab - 1) >> 5];
  }

  const float rep = a.repetition ? a.repetition[r] : 1.f;
  const float freq = a.frequency ? a.frequency[r] : 0.f;
  const float pres = a.presence ? a.presence[r] : 0.f;
  const bool lists = a.prompt || a.output;
  if (lists) {
    for (int i = 4 * tid; i < C; i += 4 * NT) *reinterpret_cast<u32x4 *>(cnt + i) = u32x4{};
    __syncthreads();
    const auto count = [&](const I4 &p, int n, int i, bool output) {
      const int from = n >= 4 ? i - min(i, n - 4) : 0;  // (the ones before were the last load's)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const uint32_t o = (uint32_t)p.v[j] - (uint32_t)v0;
        if (j >= from && o < (uint32_t)C) {
          if (output)
            atomicAdd(&cnt[o], 1u);
          else
            atomicOr(&cnt[o], 0x80000000u);
        }
      }
    };
    if (4 * tid < np) count(first_p, np, 4 * tid, false);
    if (4 * tid < no) count(first_o, no, 4 * tid, true);
    for (int i = 4 * (tid + NT); i < np; i += 4 * NT) count(ids_at(prompt, np, i), np, i, false);
    for (int i = 4 * (tid + NT); i < no; i += 4 * NT) count(ids_at(output, no, i), no, i, true);
    __syncthreads();
  }
  float x[NV][VEC];
  float *out = a.processed ? a.processed + r * a.processed_stride : nullptr;
  Best b{-INFINITY, INT32_MAX, 0.f};
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    const int v = at(k);
#pragma unroll
    for (int j = 0; j < VEC; ++j) x[k][j] = to_f32(raw[k].v[j]);
    if (v < a.vocab && v + VEC > a.vocab) {  // cut by the row's end
#pragma unroll
      for (int j = 0; j < VEC; ++j) {
        x[k][j] = v + j < a.vocab ? to_f32(logits[v + j]) : 0.f;
        if (bias) add[k][j / 4].v[j % 4] = v + j < a.vocab ? bias[v + j] : 0.f;
      }
    }
    if (lists) {
      uint32_t c[VEC], any = 0;
#pragma unroll
      for (int j = 0; j < VEC; ++j) {
        if (j % 4 == 0)
          *reinterpret_cast<u32x4 *>(c + j) =
              *reinterpret_cast<const u32x4 *>(cnt + (k * NT + tid) * VEC + j);
        any |= c[j];
      }
      if (any) {
#pragma unroll
        for (int j = 0; j < VEC; ++j) x[k][j] = penalised(x[k][j], c[j], rep, freq, pres);
      }
    }
    if (bias) {
#pragma unroll
      for (int j = 0; j < VEC; ++j) x[k][j] += add[k][j / 4].v[j % 4];
    }
    // (v is a multiple of VEC, so that a pack's bits lie in one word.)
    const uint32_t allowed = mask ? bits[k] >> (v & 31) : ~0u;
#pragma unroll
    for (int j = 0; j < VEC; ++j)
      if (v + j >= a.vocab || !((allowed >> j) & 1)) x[k][j] = -INFINITY;
  }
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    const int v = at(k);
    if (out) {
      if (v + VEC <= a.vocab) {
#pragma unroll
        for (int j0 = 0; j0 < VEC; j0 += 4) {
          const f32x4u p = {x[k][j0], x[k][j0 + 1], x[k][j0 + 2], x[k][j0 + 3]};
          if (a.past_caches) {
            asm volatile("");  // (both keep the compiler from merging this with the plain store)
            __builtin_nontemporal_store(p, reinterpret_cast<f32x4u *>(out + v + j0));
            asm volatile("");
          } else {
            *reinterpret_cast<f32x4u *>(out + v + j0) = p;
          }
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
      for (int j = 0; j < VEC; ++j) b.s += at(k) + j == b.i ? 0.f : __expf(x[k][j] - m);
  }
  b = block_best<NT>(b, red);
  if (tid == 0) {
    if (gridDim.x == 1)
      finish_row(a, r, b);
    else
      part[(long)r * gridDim.x + blockIdx.x] = b;
  }
}

template <int NT>
__global__ __launch_bounds__(NT) void k_pick_merge(PickArgs a, int chunks, const Best *part) {
  __shared__ Best red[NT / 64];
  const int r = blockIdx.x;
  Best b{-INFINITY, INT32_MAX, 0.f};
  for (int c = threadIdx.x; c < chunks; c += NT) {
    const Best p = part[(long)r * chunks + c];
    const bool better = p.m > b.m || (p.m == b.m && p.i < b.i);
    const Best hi = better ? p : b, lo = better ? b : p;
    b = {hi.m, hi.i, hi.s + share(lo, hi.m, false)};
  }
  b = block_best<NT>(b, red);
  if (threadIdx.x == 0) finish_row(a, r, b);
}

constexpr int kPickMinChunk = 4096;  // the smallest chunk of any variant below

template <typename T, int NV, int NT>
hipError_t launch_pick_chunks(const PickArgs &a, Best *part, hipStream_t s) {
  constexpr int C = NT * NV * (16 / sizeof(T));
  static_assert(C >= kPickMinChunk, "the workspace holds a partial for each smallest chunk");
  const int chunks = (a.vocab + C - 1) / C;
  const size_t lds = a.prompt || a.output ? C * sizeof(uint32_t) : 0;
  k_pick_chunks<T, NV, NT><<<dim3(chunks, a.rows), NT, lds, s>>>(a, part);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || chunks == 1) return e;
  if (chunks <= 64)
    k_pick_merge<64><<<a.rows, 64, 0, s>>>(a, chunks, part);
  else
    k_pick_merge<256><<<a.rows, 256, 0, s>>>(a, chunks, part);
  return hipGetLastError();
}

template <typename T>
hipError_t launch_pick_type(const PickArgs &a, Best *part, hipStream_t s) {
  constexpr int VEC = 16 / sizeof(T);
  // Eight entries a thread, 512 threads: chunks of 4096. A vocabulary between one and two
  // of them takes a block of 1024 threads and no second launch.
  if (a.vocab > 4096 && a.vocab <= 8192)
    return launch_pick_chunks<T, 8 / VEC, 1024>(a, part, s);
  return launch_pick_chunks<T, 8 / VEC, 512>(a, part, s);
}

}  // namespace

size_t pick_workspace_bytes(int rows, int vocab) {
  return (size_t)rows * ((vocab + kPickMinChunk - 1) / kPickMinChunk) * sizeof(Best);
}

hipError_t launch_pick(PickArgs a, int dtype, void *ws, hipStream_t s) {
  if (a.rows == 0) return hipSuccess;
  // (256 rows of 152064 kept: 91.7 us, written past the caches 88.3; 16 rows alone
  // 12.0 and 10.6, but there the next reader still finds them in the caches.)
  a.past_caches = a.processed && (long)a.rows * a.vocab * 4 > kCachedBytes;
  Best *part = static_cast<Best *>(ws);
  if (dtype == 0) return launch_pick_type<float>(a, part, s);
  if (dtype == 1) return launch_pick_type<bf16>(a, part, s);
  return launch_pick_type<f16>(a, part, s);
}

}  // namespace vsr
