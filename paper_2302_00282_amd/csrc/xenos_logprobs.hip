// What is read from logits: log probabilities of given tokens, entropy, the likeliest tokens.
//
// One pass over a row.  Each lane keeps a running maximum m with s = sum e^(x - m) and t = sum (x - m) e^(x - m), so that log p = x - m - log s and
// the entropy is log s - t / s; each wavefront keeps the best tokens it has seen sorted over its lanes, and an element is looked at closely only if it beats the
// last of those that count.  Order is that of one whole number per element: the value's bits, ordered, above the inverted index.
#include <algorithm>
#include "token_device.h"

namespace xenos {

namespace {

constexpr float kLowest = -3.402823466e38f, kLog2e = 1.44269504088896340736f;
constexpr int kPer = 16, kBlock = 64 * kPer;                  // elements per lane and wavefront at a time

// (bits of v in their order, ties to the lower index); NaN above all, -0 as 0
__device__ __forceinline__ uint64_t order_of(float v, int index) {
  const uint32_t u = v != v ? 0x7fc00000u : __float_as_uint(v + 0.f);
  return (uint64_t)(u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u)) << 32 | (uint32_t)~index;
}
__device__ __forceinline__ float value_of(uint64_t o) {
  const uint32_t u = (uint32_t)(o >> 32);
  return __uint_as_float(u & 0x80000000u ? u ^ 0x80000000u : ~u);
}
__device__ __forceinline__ int index_of(uint64_t o) { return (int)~(uint32_t)o; }

// a b, and 0 where either is 0
__device__ __forceinline__ float times_or_zero(float a, float b) {
  float r;
  asm("v_mul_legacy_f32 %0, %1, %2" : "=v"(r) : "v"(a), "v"(b));
  return r;
}

// Maximum and sums of some of a row's elements.  m is finite or +infinity: where nothing was added, s is 0.
struct Sums {
  float m, s, t;
  __device__ __forceinline__ void raise(float to) {           // to >= m
    const float d = fmaxf(m - to, -200.f), e = __builtin_amdgcn_exp2f(d * kLog2e);   // (2^-288 flushes to 0)
    t = e * (t + d * s);
    s *= e;
    m = to;
  }
  __device__ __forceinline__ void add(float x) {              // x <= m, or NaN
    const float d = x - m, e = __builtin_amdgcn_exp2f(d * kLog2e);
    s += e;
    t += times_or_zero(d, e);                                 // (-infinity adds nothing)
  }
  __device__ __forceinline__ void join(Sums o) {
    const float to = fmaxf(m, o.m);
    raise(to);
    o.raise(to);
    s += o.s;
    t += o.t;
  }
};
__device__ __forceinline__ uint64_t from_lane(uint64_t v, int lane) {
  return (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(v >> 32), lane) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)v, lane);
}

// Finishes a row whose sums and best tokens are known.
template <typename T>
__device__ __forceinline__ void finish(const LogprobsArgs& a, int row, const Sums& z) {
  const float ls = logf(z.s);
  if (a.entropy) a.entropy[row] = ls - z.t / z.s;
  if (a.logprob) {
    const long long t = a.targets[row];
    a.logprob[row] = t >= 0 && t < a.vocab ? Tr<T>::ld(a.x, row * a.stride + t) - z.m - ls : 0.f;
  }
}

// Elements that beat the last one that counts (`last`, 0 while there are fewer than `top`) join the sorted list `best`, one at a time.
__device__ __forceinline__ void best_insert(uint64_t& best, uint64_t& last, uint64_t o, int top, int lane) {
  for (uint64_t found; (found = __ballot(o > last)) != 0;) {
    const int from = __builtin_ctzll(found);
    const uint64_t take = from_lane(o, from);
    const int at = __builtin_popcountll(__ballot(best > take));
    const uint64_t up = (uint64_t)(uint32_t)__shfl_up((int)(best >> 32), 1) << 32 | (uint32_t)__shfl_up((int)best, 1);
    best = lane < at ? best : lane == at ? take : up;
    last = from_lane(best, top - 1);
    if (lane == from) o = 0;
  }
}

// The four wavefronts' sums and lists put together, and the row's results, or the part's, written.
template <typename T, bool TOP>
__device__ __forceinline__ void join_waves(const LogprobsArgs& a, Sums z, uint64_t best, int row, int part, bool partial) {
  __shared__ Sums s_sums[4];
  __shared__ uint64_t s_best[4 * kTopMost];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int o = 32; o; o >>= 1) {
    Sums other;
    other.m = __shfl_xor(z.m, o), other.s = __shfl_xor(z.s, o), other.t = __shfl_xor(z.t, o);
    z.join(other);
  }
  if (lane == 0) s_sums[wave] = z;
  if (TOP) s_best[threadIdx.x] = lane < a.top ? best : 0;
  __syncthreads();
  z = s_sums[0];
#pragma unroll
  for (int w = 1; w < 4; ++w) z.join(s_sums[w]);
  uint32_t* to = a.part + ((long long)row * a.parts + part) * (3 + 2 * a.top);
  if (threadIdx.x == 0) {
    if (partial) to[0] = __float_as_uint(z.m), to[1] = __float_as_uint(z.s), to[2] = __float_as_uint(z.t);
    else finish<T>(a, row, z);
  }
  if (!TOP) return;
  // an element's place is the number of those before it (all differ, but for the zeros of places not filled)
  const uint64_t mine = s_best[threadIdx.x];
  int at = 0;
  for (int w = 0; w < 4; ++w)
    for (int i = 0; i < a.top; ++i) at += s_best[w * kTopMost + i] > mine;
  if (mine && at < a.top) {
    if (partial) to[3 + 2 * at] = (uint32_t)mine, to[4 + 2 * at] = (uint32_t)(mine >> 32);
    else {
      a.top_token[(long long)row * a.top + at] = index_of(mine);
      a.top_logprob[(long long)row * a.top + at] = value_of(mine) - z.m - logf(z.s);
    }
  }
  // (a part that has fewer elements than are asked for: the places behind them)
  if (partial && (int)threadIdx.x < a.top) {
    int have = 0;
    for (int w = 0; w < 4; ++w)
      for (int i = 0; i < a.top; ++i) have += s_best[w * kTopMost + i] != 0;
    if ((int)threadIdx.x >= have) to[3 + 2 * threadIdx.x] = to[4 + 2 * threadIdx.x] = 0;
  }
}

// A workgroup per part of a row; its wavefronts take blocks of the part in turn.
template <typename T, bool TOP>
__global__ __launch_bounds__(256) void logprobs_kernel(LogprobsArgs a) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, row = (int)blockIdx.x / a.parts, part = (int)blockIdx.x - row * a.parts;
  const T* x = (const T*)a.x + row * a.stride;
  const int begin = part * a.part_len, end = begin + a.part_len < a.vocab ? begin + a.part_len : a.vocab;
  // vectors start where memory is aligned to 16 bytes, before `begin` by up to CE - 1 elements
  constexpr int CE = Tr<T>::CE, NV = kPer / CE;
  const int shift = (int)(((uintptr_t)(x + begin) & 15) / sizeof(T)), first = begin - shift + lane * CE;
  Sums z{kLowest, 0.f, 0.f};
  uint64_t best = 0, last = 0;                                // lane i: the i-th best so far; the last one that counts
  for (int b = wave * kBlock; b < end - begin + shift; b += 4 * kBlock) {
    float f[kPer];
#pragma unroll
    for (int c = 0; c < NV; ++c) {
      const int i = first + b + c * 64 * CE;
      if (i >= begin && i + CE <= end) Tr<T>::unpack(*(const u32x4_t*)(x + i), f + c * CE);
      else {
#pragma unroll
        for (int e = 0; e < CE; ++e) f[c * CE + e] = i + e >= begin && i + e < end ? Tr<T>::ld(x, i + e) : -INFINITY;
      }
    }
    float top = f[0];
#pragma unroll
    for (int e = 1; e < kPer; ++e) top = fmaxf(top, f[e]);
    z.raise(fmaxf(z.m, top));
#pragma unroll
    for (int e = 0; e < kPer; ++e) z.add(f[e]);
    // (what equals the last one comes after it: its index is higher than any seen in an earlier block)
    if (TOP && (last == 0 || __any(top > value_of(last) || z.s != z.s))) {
#pragma unroll
      for (int c = 0; c < NV; ++c)
#pragma unroll
        for (int e = 0; e < CE; ++e) {
          const int i = first + b + c * 64 * CE + e;
          const uint64_t o = i >= begin && i < end ? order_of(f[c * CE + e], i) : 0;
          best_insert(best, last, o, a.top, lane);
        }
    }
  }
  join_waves<T, TOP>(a, z, best, row, part, a.parts > 1);
}

// The parts of a row put together, in the order of the parts.
template <typename T, bool TOP>
__global__ __launch_bounds__(256) void logprobs_join_kernel(LogprobsArgs a) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, row = (int)blockIdx.x, words = 3 + 2 * a.top;
  const uint32_t* parts = a.part + (long long)row * a.parts * words;
  Sums z{kLowest, 0.f, 0.f};
  if (wave == 0 && lane < a.parts) {
    const uint32_t* p = parts + lane * words;
    z.m = __uint_as_float(p[0]), z.s = __uint_as_float(p[1]), z.t = __uint_as_float(p[2]);
  }
  uint64_t best = 0, last = 0;
  if (TOP)
    for (int i = wave; i < a.parts; i += 4) {
      const uint32_t* p = parts + i * words + 3 + 2 * lane;
      best_insert(best, last, lane < a.top ? (uint64_t)p[1] << 32 | p[0] : 0, a.top, lane);
    }
  join_waves<T, TOP>(a, z, best, row, 0, false);
}

template <typename T>
int logprobs(const LogprobsArgs& a, hipStream_t st) {
  const int grid = a.rows * a.parts;
  if (a.top) logprobs_kernel<T, true><<<grid, 256, 0, st>>>(a);
  else logprobs_kernel<T, false><<<grid, 256, 0, st>>>(a);
  if (a.parts > 1) {
    if (a.top) logprobs_join_kernel<T, true><<<a.rows, 256, 0, st>>>(a);
    else logprobs_join_kernel<T, false><<<a.rows, 256, 0, st>>>(a);
  }
  return (int)hipGetLastError();
}

}  // namespace

// Rows are read whole where there are enough of them to fill the units, else in up to 64 parts of at least four blocks.
void logprobs_split(int rows, int vocab, int* parts, int* part_len) {
  const long long want = std::max(1, std::min(64, 1024 / std::max(1, rows))), most = std::max(1, vocab / (4 * kBlock));
  const int len = (int)((vocab + std::min(want, most) - 1) / std::min(want, most));
  *part_len = len;
  *parts = (vocab + len - 1) / len;
}

int launch_logprobs(const LogprobsArgs& a, int dtype, void* stream) {
  return dtype ? logprobs<bf16_t>(a, (hipStream_t)stream) : logprobs<float>(a, (hipStream_t)stream);
}

}  // namespace xenos
