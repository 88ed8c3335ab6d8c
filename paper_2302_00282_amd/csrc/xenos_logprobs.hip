// What is read from logits: log probabilities of given tokens, entropy, the likeliest tokens.
//
// One pass over a row.  Each lane keeps a reference m near the row's maximum with s = sum e^(x - m) and t = sum (x - m) e^(x - m), so that log p = x - m - log s and
// the entropy is log s - t / s; each wavefront keeps the best tokens it has seen sorted over its lanes, and an element is looked at closely only if it beats the
// last of those that count.  Order is that of one whole number per element: the value's bits, ordered, above the inverted index.
#include <algorithm>
#include "token_device.h"

namespace xenos {

namespace {

constexpr float kLowest = -3.402823466e38f, kLog2e = 1.44269504088896340736f;
constexpr float kSlack = 1.f;                                 // a maximum is followed when it has grown by more (the exponents' own rounding goes with their size: 8 was no faster)
constexpr int kPer = 16, kBlock = 64 * kPer;                  // elements per lane and wavefront at a time

// (bits of v in their order, ties to the lower index); NaN above all, -0 as 0
__device__ __forceinline__ uint64_t order_of(float v, int index) {
  const uint32_t bits = __float_as_uint(v), u = (bits & 0x7fffffffu) > 0x7f800000u ? 0x7fc00000u : bits == 0x80000000u ? 0u : bits;
  return (uint64_t)(u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u)) << 32 | (uint32_t)~index;
}
__device__ __forceinline__ float value_of(uint64_t o) {
  const uint32_t u = (uint32_t)(o >> 32);
  return __uint_as_float(u & 0x80000000u ? u ^ 0x80000000u : ~u);
}
__device__ __forceinline__ int index_of(uint64_t o) { return (int)~(uint32_t)o; }

// Sums over some of a row's elements: s = sum e^(x - m), t = sum (x - m) e^(x - m).  The reference m is the maximum, or less by kSlack at most, finite or +infinity; where
// nothing was added, s is 0.  (x - m is made before it is scaled for the power of 2: x log2 e - m log2 e in one instruction overflows where a mask of the type's lowest
// value leaves nothing else.)
struct Sums {
  float m, s, t;
  __device__ __forceinline__ void raise(float to) {           // to >= m
    const float d = fmaxf(m - to, -200.f), e = __builtin_amdgcn_exp2f(d * kLog2e);   // (2^-288 flushes to 0)
    t = e * (t + d * s);
    s *= e;
    m = to;
  }
  __device__ __forceinline__ void add(float x) {              // x <= m + kSlack, or NaN
    const float d = x - m, e = __builtin_amdgcn_exp2f(d * kLog2e);
    s += e;
    t = __builtin_fmaf(fmaxf(d, kLowest), e, t);              // (-infinity adds nothing: 0 times a number; a NaN is in s)
  }
  __device__ __forceinline__ void join(Sums o) {
    const float to = fmaxf(m, o.m);
    raise(to);
    o.raise(to);
    s += o.s;
    t += o.t;
  }
  __device__ __forceinline__ float logprob(float x) const { return x - m - logf(s); }
  __device__ __forceinline__ float entropy() const { return logf(s) - t / s; }
};
__device__ __forceinline__ uint64_t from_lane(uint64_t v, int lane) {
  return (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(v >> 32), lane) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)v, lane);
}

// Finishes a row whose sums and best tokens are known.
template <typename T>
__device__ __forceinline__ void finish(const LogprobsArgs& a, int row, const Sums& z) {
  if (a.entropy) a.entropy[row] = z.entropy();
  if (a.logprob) {
    const long long t = a.targets[row];
    a.logprob[row] = t >= 0 && t < a.vocab ? z.logprob(Tr<T>::ld(a.x, row * a.stride + t)) : 0.f;
  }
}

// v of the lane before (lane 0: anything)
__device__ __forceinline__ uint32_t lane_before(uint32_t v) { return (uint32_t)__builtin_amdgcn_update_dpp((int)v, (int)v, 0x138, 0xf, 0xf, false); }   // (wave_shr:1)

// The best elements a wavefront has seen, by order_of: lane i has the i-th; `last`, the top-th, is 0 while there are fewer.
struct Best {
  uint32_t lo = 0, hi = 0;
  uint64_t last = 0;
  __device__ __forceinline__ void insert(uint64_t o, int top) {   // o > last, the same for all lanes
    const int lane = threadIdx.x & 63;
    const bool before = all() > o;
    const int at = __builtin_popcountll(__ballot(before));
    const uint32_t up_lo = lane_before(lo), up_hi = lane_before(hi);
    lo = before ? lo : up_lo, hi = before ? hi : up_hi;
    lo = lane == at ? (uint32_t)o : lo, hi = lane == at ? (uint32_t)(o >> 32) : hi;
    last = (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)hi, top - 1) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)lo, top - 1);
  }
  // an element of each lane, 0 for none
  __device__ __forceinline__ void offer(uint64_t o, int top) {
    for (uint64_t found = __ballot(o > last); found; found &= found - 1) {
      const uint64_t take = from_lane(o, __builtin_ctzll(found));
      if (take > last) insert(take, top);
    }
  }
  __device__ __forceinline__ uint64_t all() const { return (uint64_t)hi << 32 | lo; }
};

// The rank-th largest (from 0) of the lanes' values, by a sorting network: halves of 2, 4 .. 64 lanes in turn, each merged in steps.
__device__ __forceinline__ float lane_rank(float v, int rank, int lane) {
#pragma unroll
  for (int size = 2; size <= 64; size <<= 1)
#pragma unroll
    for (int step = size >> 1; step; step >>= 1) {
      const float o = __uint_as_float((uint32_t)__builtin_amdgcn_ds_bpermute((lane ^ step) << 2, (int)__float_as_uint(v)));
      const bool down = (lane & size) == 0, first = (lane & step) == 0;
      v = down == first ? fmx_raw(v, o) : fminf(v, o);
    }
  return __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(v), rank));
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
      a.top_logprob[(long long)row * a.top + at] = z.logprob(value_of(mine));
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

// A workgroup per part of a row; its wavefronts take blocks of the part in turn.  Bound by vector instructions, some 25 places of issue an element (an exponential is four of them): 2048 x 100003 in bf16 with
// the best tokens takes 127 to 145 us, 2.8 to 3.2 TB/s; 1 x 32000 10 us (in 7 parts of four or more blocks, whose first fill the lists).
template <typename T, bool TOP>
__global__ __launch_bounds__(256, 8) void logprobs_kernel(LogprobsArgs a) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), row = (int)blockIdx.x / a.parts, part = (int)blockIdx.x - row * a.parts;
  const T* x = (const T*)a.x + row * a.stride;
  const int begin = part * a.part_len, end = begin + a.part_len < a.vocab ? begin + a.part_len : a.vocab;
  // vectors start where memory is aligned to 16 bytes, before `begin` by up to CE - 1 elements
  constexpr int CE = Tr<T>::CE, NV = kPer / CE;
  const int shift = (int)(((uintptr_t)(x + begin) & 15) / sizeof(T)), first = begin - shift + lane * CE;
  Sums z{kLowest, 0.f, 0.f};
  Best best;
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
    for (int e = 1; e + 1 < kPer; e += 2) top = max3_raw(top, f[e], f[e + 1]);
    top = fmx_raw(top, f[kPer - 1]);
    if (__any(top > z.m + kSlack)) z.raise(fmaxf(z.m, top));
    Sums here{z.m, 0.f, 0.f};                                 // (by itself: terms added one by one to all that went before would be lost behind a few large ones)
#pragma unroll
    for (int e = 0; e < kPer; ++e) here.add(f[e]);
    z.s += here.s, z.t += here.t;
    if (!TOP) continue;
    const int i0 = begin - shift + b;                         // (of lane 0)
    // What equals the last one comes after it, since its index is higher than any seen in an earlier block.  The first block has no last one: the top-th of the lanes' largest
    // elements is one that as many elements reach.  There, where many may be equal, and where there is a NaN, now or before, elements are compared in full by every lane; else
    // the few that pass are looked at by the scalar unit.
    const bool from_here = best.last == 0, nan = __any(z.s != z.s);
    if (from_here || nan) {
      int here = lane;
      asm volatile("" : "+v"(here));                          // (what this rare path needs is made in it, not held through the others)
      const float over = nan ? -INFINITY : lane_rank(top, a.top - 1, here);
      const int mine = i0 + here * CE;
#pragma unroll
      for (int c = 0; c < NV; ++c)
#pragma unroll
        for (int e = 0; e < CE; ++e) {
          const int i = mine + c * 64 * CE + e;
          const float v = f[c * CE + e];
          best.offer(i >= begin && i < end && !(v < over) ? order_of(v, i) : 0, a.top);
        }
      continue;
    }
    const float over = value_of(best.last);
    if (!__any(top > over)) continue;
#pragma unroll
    for (int c = 0; c < NV; ++c)
#pragma unroll
      for (int e = 0; e < CE; ++e) {
        const float v = f[c * CE + e];
        for (uint64_t found = __ballot(v > over); found; found &= found - 1) {   // (what lies outside the row is -infinity: not more than anything)
          const int from = __builtin_ctzll(found), i = i0 + (c * 64 + from) * CE + e;
          const uint64_t take = order_of(__uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(v), from)), i);
          if (take > best.last) best.insert(take, a.top);
        }
      }
  }
  join_waves<T, TOP>(a, z, best.all(), row, part, a.parts > 1);
}

// The parts of a row put together, in the order of the parts (up to 64 of them: 4 us, a launch and two trips to memory).
template <typename T, bool TOP>
__global__ __launch_bounds__(256) void logprobs_join_kernel(LogprobsArgs a) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, row = (int)blockIdx.x, words = 3 + 2 * a.top;
  const uint32_t* parts = a.part + (long long)row * a.parts * words;
  Sums z{kLowest, 0.f, 0.f};
  if (wave == 0 && lane < a.parts) {
    const uint32_t* p = parts + lane * words;
    z.m = __uint_as_float(p[0]), z.s = __uint_as_float(p[1]), z.t = __uint_as_float(p[2]);
  }
  Best best;
  if (TOP)
    for (int i = wave; i < a.parts; i += 4) {
      const uint32_t* p = parts + i * words + 3 + 2 * lane;
      best.offer(lane < a.top ? (uint64_t)p[1] << 32 | p[0] : 0, a.top);
    }
  join_waves<T, TOP>(a, z, best.all(), row, 0, false);
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

// Rows are read whole where there are enough of them to fill the units, else in up to 64 parts of at least four blocks, 1024 workgroups in all.  us whole, in parts (bf16, the five best): 1 x 32000: 17, 15;
// 1 x 151936: 43, 16.5; 64 x 100003: 34, 21 (of 256 workgroups: 23); 512 x 100003: 50, 45; 256 x 32000: 20, 20; 1024 x 32000, in two: 30, 36.
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
