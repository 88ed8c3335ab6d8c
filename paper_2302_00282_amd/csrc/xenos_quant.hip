// Rows in 8-bit integers with a scale each, and their product: the linear layers of a token model.
#include "device_common.h"
#include <algorithm>
#include "token_device.h"
#include "wave_gemm.h"

namespace xenos {

// Shares of K that the smallest tiles of a product are made in, while there are units for them: what is least of the steps of a share (0.3 us each for a workgroup of its
// own unit), the second launch (5 us with the gap before it) and its sums, written and read at 3.5 TB/s.  32 x 25088 x 4096 in 8: 57 us become 23;
// 300 x 8192 x 640 in 10: 21 become 14; 128 x 4096 x 4096 stays whole: 12.7 would be 14.
int quant_splits(int rows, int out_c, long long pitch) {
  const long long tiles = (long long)((rows + 63) / 64) * ((out_c + 63) / 64), steps = pitch / 128;
  int best = 1;
  double least = 0.3 * (double)steps;
  for (int s = 2; s <= 16 && tiles * s <= 512 && s <= steps; ++s) {
    const long long share = (steps + s - 1) / s;
    if (share * (s - 1) >= steps) continue;                   // (a share would be left without steps)
    const double t = 0.3 * (double)share + 5.0 + 8.0 * rows * out_c * s / 3.5e6;
    if (t < least) least = t, best = s;
  }
  return best;
}

// Eight values of a row from element i on, those behind the row's end as zeros.
template <typename T>
__device__ __forceinline__ void load8(const T* row, int i, int cols, int vec, float* f) {
  if (vec && i + 8 <= cols) {
#pragma unroll
    for (int c = 0; c < 8 / Tr<T>::CE; ++c) Tr<T>::unpack(*(const u32x4_t*)(row + i + c * Tr<T>::CE), f + c * Tr<T>::CE);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = i + e < cols ? Tr<T>::ld(row, i + e) : 0.f;
  }
}
// Behind a norm: each value of f shown to `see`, and times its weight in v (f itself, maybe).
template <typename See>
__device__ __forceinline__ void times_gamma(const QuantRowsArgs& a, int i, const float* f, float* v, See see) {
  if (!a.gamma) {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = f[e];
    return;
  }
  float w[8];
  load8<float>(a.gamma, i, a.cols, a.vec_gamma, w);
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    see(f[e]);
    v[e] = f[e] * w[e];
  }
}
// Eight values in whole steps.  A sum with 1.5 2^23 rounds to nearest even and leaves the number's low byte in the lowest eight bits (a NaN's are 0).
__device__ __forceinline__ uint2 packed8(const RowStep& step, const float* v) {
#pragma clang fp contract(off)
  uint32_t u[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) u[e] = __float_as_uint(v[e] * step.inv + 12582912.f);
  const auto four = [](const uint32_t* w) { return __builtin_amdgcn_perm(__builtin_amdgcn_perm(w[3], w[2], 0x0c0c0400u), __builtin_amdgcn_perm(w[1], w[0], 0x0c0c0400u), 0x05040100u); };
  return make_uint2(four(u), four(u + 4));
}
// What a row's values are multiplied by before they are squared: 1, and only where that sum has overflowed, or lost bits below the least normal number that eps does not
// cover, a power of 2 that brings every value's square into range.  (Such a row is read once more.)
__device__ __forceinline__ float square_unit(const QuantRowsArgs& a, float sq) {
  return !a.gamma ? 1.f : sq == INFINITY ? 0x1p-75f : sq / (float)a.cols + a.eps < 0x1p-70f ? 0x1p64f : 1.f;
}
// This thread's share of a row's squares, elements `first` to `first` + 7 and so on in steps of `step`, in that unit.
template <typename T>
__device__ __forceinline__ float squares(const QuantRowsArgs& a, const T* row, int first, int step, float by) {
  float sq = 0.f;
  for (int i = first; i < a.cols; i += step) {
    float f[8];
    load8<T>(row, i, a.cols, a.vec, f);
#pragma unroll
    for (int e = 0; e < 8; ++e) sq += (f[e] * by) * (f[e] * by);
  }
  return sq;
}
__device__ __forceinline__ float row_scale(const QuantRowsArgs& a, const RowStep& step, float sq, float by) {
  return a.gamma ? step.scale() * (1.f / sqrtf(sq / (float)a.cols + a.eps * by * by)) * by : step.scale();
}

// One workgroup per row: q = rint(x g 127 / a), a = max|x g|, scale = a / 127 [/ rms(x)].  The norm's factor is one number per row: it
// cancels in q, so that the rounded values do not depend on how the squares are summed.  A thread keeps its NV x 8 values in registers, one pass over memory
// (8192 x 8192 bf16: 63 us in two passes, 45 so: 4.5 TB/s read and written, what memory gives); NV = 0: rows of any length in two passes, the second from the cache (where there are few of them, the same time: 32 x 25088 takes 7 us).
template <typename T, int NV>
__global__ __launch_bounds__(1024) void quant_rows_kernel(QuantRowsArgs a) {
  __shared__ uint32_t s_max[16];
  __shared__ float s_sum[16];
  const int step = (int)blockDim.x * 8, waves = (int)blockDim.x / 64;
  for (int at = (int)blockIdx.x; at < a.rows; at += (int)gridDim.x) {
    const T* row = (const T*)a.x + at * a.stride;
    int8_t* q = a.q + at * a.pitch;
    uint32_t m = 0;
    float sq = 0.f, v[NV ? NV : 1][8];
    const auto look = [&](int i, float* f) {
      times_gamma(a, i, f, f, [&](float x) { sq += x * x; });
#pragma unroll
      for (int e = 0; e < 8; ++e) m = umax(m, magnitude(f[e]));
    };
    if constexpr (NV > 0) {
#pragma unroll
      for (int c = 0; c < NV; ++c) load8<T>(row, (int)threadIdx.x * 8 + c * step, a.cols, a.vec, v[c]);
#pragma unroll
      for (int c = 0; c < NV; ++c) look((int)threadIdx.x * 8 + c * step, v[c]);
    } else {
      for (int i = (int)threadIdx.x * 8; i < a.cols; i += step) {
        load8<T>(row, i, a.cols, a.vec, v[0]);
        look(i, v[0]);
      }
    }
    m = wave_max(m);
    sq = wave_sum(sq);
    if ((threadIdx.x & 63) == 0) { s_max[threadIdx.x >> 6] = m; s_sum[threadIdx.x >> 6] = sq; }
    __syncthreads();
    m = 0, sq = 0.f;
    for (int w = 0; w < waves; ++w) { m = umax(m, s_max[w]); sq += s_sum[w]; }
    const RowStep unit(m);
    if constexpr (NV > 0) {
#pragma unroll
      for (int c = 0; c < NV; ++c) {
        const int i = (int)threadIdx.x * 8 + c * step;
        if (i < (int)a.pitch) *(uint2*)(q + i) = packed8(unit, v[c]);
      }
    } else {
      for (int i = (int)threadIdx.x * 8; i < (int)a.pitch; i += step) {
        load8<T>(row, i, a.cols, a.vec, v[0]);
        times_gamma(a, i, v[0], v[0], [](float) {});
        *(uint2*)(q + i) = packed8(unit, v[0]);
      }
    }
    const float by = square_unit(a, sq);
    if (by != 1.f) {                                          // (the same for every thread)
      sq = wave_sum(squares(a, row, (int)threadIdx.x * 8, step, by));
      __syncthreads();
      if ((threadIdx.x & 63) == 0) s_sum[threadIdx.x >> 6] = sq;
      __syncthreads();
      sq = 0.f;
      for (int w = 0; w < waves; ++w) sq += s_sum[w];
    }
    if (threadIdx.x == 0) a.scale[at] = row_scale(a, unit, sq, by);
    __syncthreads();                                          // (s_max and s_sum are free again)
  }
}

template <typename T>
static int quant_rows(const QuantRowsArgs& a, hipStream_t st) {
  const int grid = a.rows < 65536 ? a.rows : 65536;
  if (a.pitch <= 2048) quant_rows_kernel<T, 1><<<grid, 256, 0, st>>>(a);
  else if (a.pitch <= 4096) quant_rows_kernel<T, 2><<<grid, 256, 0, st>>>(a);
  else if (a.pitch <= 8192) quant_rows_kernel<T, 2><<<grid, 512, 0, st>>>(a);
  else if (a.pitch <= 16384) quant_rows_kernel<T, 2><<<grid, 1024, 0, st>>>(a);
  else quant_rows_kernel<T, 0><<<grid, 1024, 0, st>>>(a);
  return (int)hipGetLastError();
}
int launch_quant_rows(const QuantRowsArgs& a, int dtype, void* stream) {
  return dtype ? quant_rows<bf16_t>(a, (hipStream_t)stream) : quant_rows<float>(a, (hipStream_t)stream);
}

// y = act(acc xs ws + bias + residual) for four neighbouring columns n of row m.
template <typename T>
__device__ __forceinline__ void store4(const QuantMatmulArgs& a, int m, int n, const i32x4_t& acc, float xs) {
  if (m >= a.M || n >= a.N) return;
  T* out = (T*)a.out + (long long)m * a.out_stride + n;
  const T* res = a.res ? (const T*)a.res + (long long)m * a.res_stride + n : nullptr;
  const bool whole = a.vec_out && n + 4 <= a.N;
  float y[4], r[4] = {0.f, 0.f, 0.f, 0.f};
  if (res) {
    if (whole && sizeof(T) == 4) {
      const float4 v = *(const float4*)res;
      r[0] = v.x, r[1] = v.y, r[2] = v.z, r[3] = v.w;
    } else if (whole) {
      const uint2 v = *(const uint2*)res;
      r[0] = bf2f(v.x & 0xffff), r[1] = bf2f(v.x >> 16), r[2] = bf2f(v.y & 0xffff), r[3] = bf2f(v.y >> 16);
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (n + e < a.N) r[e] = Tr<T>::ld(res, e);
    }
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const int c = n + e < a.N ? n + e : n;
    y[e] = (float)acc[e] * xs * a.ws[c] + (a.bias ? a.bias[c] : 0.f) + r[e];
    if (a.relu) y[e] = y[e] < 0.f ? 0.f : y[e];               // (a NaN stays)
  }
  if (whole && sizeof(T) == 4) *(float4*)out = make_float4(y[0], y[1], y[2], y[3]);
  else if (whole) *(uint2*)out = make_uint2(f2bf2(y[0], y[1]), f2bf2(y[2], y[3]));
  else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (n + e < a.N) Tr<T>::st(out, e, y[e]);
  }
}

// The same for eight columns, whose scales and biases are at hand.
template <typename T>
__device__ __forceinline__ void store8(const QuantMatmulArgs& a, int m, int n, const i32x4_t& lo, const i32x4_t& hi, float xs, const float* ws, const float* bias) {
  T* out = (T*)a.out + (long long)m * a.out_stride + n;
  const T* res = a.res ? (const T*)a.res + (long long)m * a.res_stride + n : nullptr;
  const bool whole = a.vec_out && n + 8 <= a.N;
  float y[8], v[8];
  if (res) {
    if (whole) {
#pragma unroll
      for (int c = 0; c < 8 / Tr<T>::CE; ++c) Tr<T>::unpack(*(const u32x4_t*)(res + c * Tr<T>::CE), v + c * Tr<T>::CE);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = n + e < a.N ? Tr<T>::ld(res, e) : 0.f;
    }
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    y[e] = (float)(e < 4 ? lo[e & 3] : hi[e & 3]) * xs * ws[e] + bias[e];
    if (res) y[e] += v[e];
    if (a.relu) y[e] = y[e] < 0.f ? 0.f : y[e];
  }
  if (whole) {
#pragma unroll
    for (int c = 0; c < 8 / Tr<T>::CE; ++c) *(u32x4_t*)(out + c * Tr<T>::CE) = Tr<T>::pack(y + c * Tr<T>::CE);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (n + e < a.N) Tr<T>::st(out, e, y[e]);
  }
}

// The rows of x that a workgroup of eight wavefronts multiplies, quantised by itself into LDS (`pitch` bytes a row) as quant_rows_kernel does: eight, four, two wavefronts
// or one to a row.
template <typename T>
__device__ __forceinline__ void quant_into_lds(const QuantRowsArgs& a, int8_t* q, float* scale) {
  __shared__ uint32_t s_max[16];
  __shared__ float s_sum[16][8];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, share = a.rows > 4 ? 1 : a.rows > 2 ? 2 : a.rows > 1 ? 4 : 8, piece = wave % share;
  if (threadIdx.x < 16) s_max[threadIdx.x] = 0;
  __syncthreads();
  for (int r = wave / share; r < a.rows; r += 8 / share) {
    const T* row = (const T*)a.x + r * a.stride;
    uint32_t m = 0;
    float sq = 0.f;
    for (int i = (piece * 64 + lane) * 8; i < a.cols; i += share * 512) {
      float f[8], v[8];
      load8<T>(row, i, a.cols, a.vec, f);
      times_gamma(a, i, f, v, [&](float x) { sq += x * x; });
#pragma unroll
      for (int e = 0; e < 8; ++e) m = umax(m, magnitude(v[e]));
    }
    m = wave_max(m);
    sq = wave_sum(sq);
    if (lane == 0) atomicMax(&s_max[r], m), s_sum[r][piece] = sq;
  }
  __syncthreads();
  for (int r = wave / share; r < a.rows; r += 8 / share) {
    const T* row = (const T*)a.x + r * a.stride;
    const RowStep step(s_max[r]);
    for (int i = (piece * 64 + lane) * 8; i < (int)a.pitch; i += share * 512) {
      float f[8], v[8];
      load8<T>(row, i, a.cols, a.vec, f);
      times_gamma(a, i, f, v, [](float) {});
      *(uint2*)(q + r * a.pitch + i) = packed8(step, v);
    }
    if (piece == 0) {
      float sq = 0.f;
      for (int w = 0; w < share; ++w) sq += s_sum[r][w];
      const float by = square_unit(a, sq);
      if (by != 1.f) sq = wave_sum(squares(a, row, lane * 8, 512, by));
      if (lane == 0) scale[r] = row_scale(a, step, sq, by);
    }
  }
  __syncthreads();
}

// Few rows: the weights are the work.  A workgroup has 16 output channels and all of K, which its wavefronts share; every fragment of the weights goes
// from memory to registers, a lane's 16 bytes of one weight row at a time, and the sums (whole numbers: exact in any order) meet in LDS.
// Bound by the weights' bytes where there are many (1 x 25088 x 4096: 17.7 us, 5.8 TB/s), by its chain of trips to memory and LDS where there are few.
// OWN: x comes as it is, and every workgroup quantises all of it for itself (1 x 512 x 2048 in one launch: 5.9 us; linear_in_one).
template <typename T, int MT, bool OWN>
__global__ __launch_bounds__(512) void quant_matvec_kernel(QuantMatmulArgs a, QuantRowsArgs qa) {
  __shared__ i32x4_t part[8][MT][64];
  extern __shared__ __attribute__((aligned(16))) int8_t s_q[];
  __shared__ float s_scale[16];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = lane & 15, g = lane >> 4;
  const int n0 = (int)blockIdx.x * 16, pitch = (int)a.pitch;
  const rsrc_t w = make_window(a.w + (long long)n0 * a.pitch, (unsigned)((a.N - n0 < 16 ? a.N - n0 : 16) * pitch));
  const unsigned w_at = (unsigned)(r * pitch + g * 16), x_at = w_at;
  const rsrc_t x = make_window(OWN ? a.w : a.x, (unsigned)(a.M * pitch));
  i32x4_t acc[MT] = {};
  // AHEAD steps are asked for at a time; what lies behind the rows, or behind the last row, reads as zeros
  constexpr int AHEAD = MT == 1 ? 8 : MT == 2 ? 4 : 2;
  u32x4_t fw[AHEAD][2], fx[AHEAD][2][MT];
  const auto request = [&](int k) {
#pragma unroll
    for (int u = 0; u < AHEAD; ++u)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int at = k + 1024 * u;
        fw[u][h] = load_window_if(w, at < pitch, w_at + at + 64 * h);
        if (OWN) continue;
#pragma unroll
        for (int t = 0; t < MT; ++t) fx[u][h][t] = load_window_if(x, at < pitch, x_at + 16 * t * pitch + at + 64 * h);
      }
  };
  const auto multiply = [&](int k) {
#pragma unroll
    for (int u = 0; u < AHEAD; ++u)
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int t = 0; t < MT; ++t) {
          if (OWN) fx[u][h][t] = r < a.M && k + 1024 * u < pitch ? *(const u32x4_t*)(s_q + r * pitch + g * 16 + k + 1024 * u + 64 * h) : u32x4_t{0, 0, 0, 0};
          acc[t] = __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(i32x4_t, fw[u][h]), __builtin_bit_cast(i32x4_t, fx[u][h][t]), acc[t], 0, 0, 0);
        }
  };
  if (OWN) {                                                  // (rows of at most 8192 bytes: one turn, whose weights are on their way while x is quantised)
    static_assert(!OWN || AHEAD == 8, "");
    request(wave * 128);
    __builtin_amdgcn_sched_barrier(0);
    quant_into_lds<T>(qa, s_q, s_scale);
    multiply(wave * 128);
  } else {
    for (int k = wave * 128; k < pitch; k += 1024 * AHEAD) {
      request(k);
      __builtin_amdgcn_sched_barrier(0);                      // (all of it before the first product: the compiler would ask for as little as fits few registers)
      multiply(k);
    }
  }
#pragma unroll
  for (int t = 0; t < MT; ++t) part[wave][t][lane] = acc[t];
  __syncthreads();
  for (int t = wave; t < MT; t += 8) {
    i32x4_t sum = part[0][t][lane];
#pragma unroll
    for (int v = 1; v < 8; ++v) sum += part[v][t][lane];
    const int m = 16 * t + r;
    store4<T>(a, m, n0 + 4 * g, sum, OWN ? s_scale[m < 16 ? m : 0] : m < a.M ? a.xs[m] : 0.f);
  }
}

// Waits until no more than min(behind, MOST) steps of LOADS requests are on their way.
template <int MOST, int LOADS>
__device__ __forceinline__ void wait_behind(int behind) {
  if constexpr (MOST <= 0) wait_requests<0>();
  else if (behind >= MOST) wait_requests<MOST * LOADS>();
  else wait_behind<MOST - 1, LOADS>(behind);
}

// Many rows: a workgroup of WM x WN wavefronts makes a tile of 32 TM WM rows of x times 32 TN WN rows of w, each wavefront TM x TN blocks of 32 x 32.
// K passes in steps of 128 bytes through STAGES stages of LDS that the loads write themselves (whole lines of the cache: with steps of 64 bytes a unit got 16 bytes a cycle).
// A step is read in two halves, each while the half before it is multiplied; behind the second read the stage is free, and one barrier tells that to all and that the
// next stage has arrived.
// Bound by the matrix units: 8192 x 8192 x 8192 takes 510 to 560 us, 2.0 to 2.15 POP/s, with tiles of 256.  Tiles of 64 in shares of K stream weights: 32 x 25088 x 4096 21 us, 4.9 TB/s.
template <typename T, int WM, int WN, int TM, int TN, int STAGES>
__global__ __launch_bounds__(64 * WM * WN) void quant_matmul_kernel(QuantMatmulArgs a, int tiles_m, int tiles_n, int splits) {
  constexpr int BM = 32 * TM * WM, BN = 32 * TN * WN, WAVES = WM * WN, STAGE = (BM + BN) * 128, LOADS = (BM + BN) / 8 / WAVES;
  static_assert(LOADS * WAVES * 8 == BM + BN && LOADS * (STAGES - 1) < 64, "whole loads of eight rows; waits can count them");
  extern __shared__ __attribute__((aligned(16))) unsigned char s_stage[];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = lane & 31, half = lane >> 5;
  // an XCD has a run of the tiles, and goes through it in columns of eight rows of tiles: what its units read at a time is shared in its L2
  const int tiles = tiles_m * tiles_n, xcd = (int)blockIdx.x % NUM_XCD, each = (tiles * splits + NUM_XCD - 1) / NUM_XCD, item = xcd * each + (int)blockIdx.x / NUM_XCD;
  if (item >= tiles * splits) return;
  const int split = item / tiles, at = item - split * tiles;
  const int band = at / (8 * tiles_n), in_band = at - band * 8 * tiles_n, high = tiles_m - 8 * band < 8 ? tiles_m - 8 * band : 8;
  const int m0 = (8 * band + in_band % high) * BM, n0 = in_band / high * BN;
  const int wm = wave % WM * 32 * TM, wn = wave / WM * 32 * TN, pitch = (int)a.pitch;

  // this workgroup's share of K
  const int all = pitch / 128, share = (all + splits - 1) / splits, step0 = split * share, steps = all - step0 < share ? all - step0 : share;
  rsrc_t window[LOADS];
  unsigned from[LOADS];
#pragma unroll
  for (int i = 0; i < LOADS; ++i) {
    const int first = __builtin_amdgcn_readfirstlane((wave * LOADS + i) * 8);
    const bool is_w = first < BN;
    const int have = is_w ? a.N - n0 : a.M - m0, in = (is_w ? first : first - BN) + lane / 8, edge = is_w ? BN : BM;
    window[i] = make_window(is_w ? a.w + (long long)n0 * a.pitch : a.x + (long long)m0 * a.pitch, (unsigned)((have < edge ? have : edge) * pitch));   // (rows behind the last one: zeros)
    from[i] = (unsigned)(in * pitch + ((lane & 7) ^ wave_swizzle(in)) * 16);
  }
  const auto request = [&](int s, int slot) {
#pragma unroll
    for (int i = 0; i < LOADS; ++i) load_to_lds(window[i], s_stage + slot * STAGE + (wave * LOADS + i) * 1024, from[i], (unsigned)((step0 + s) * 128));
  };
  int place[4];                                               // (rows that differ by multiples of 32 have the same places)
#pragma unroll
  for (int k = 0; k < 4; ++k) place[k] = r * 128 + ((2 * k + half) ^ wave_swizzle(r)) * 16;
  struct Fragments { i32x4_t w[2][TN], x[2][TM]; };
  const auto fetch = [&](int slot, int second, Fragments& f) {
    const unsigned char* stage = s_stage + slot * STAGE;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
#pragma unroll
      for (int t = 0; t < TN; ++t) f.w[k][t] = *(const i32x4_t*)(stage + (wn + 32 * t) * 128 + place[2 * second + k]);
#pragma unroll
      for (int t = 0; t < TM; ++t) f.x[k][t] = *(const i32x4_t*)(stage + (BN + wm + 32 * t) * 128 + place[2 * second + k]);
    }
  };
  i32x16_t acc[TM][TN] = {};
  const auto multiply = [&](const Fragments& f) {
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
      for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(f.w[k][j], f.x[k][i], acc[i][j], 0, 0, 0);
  };
  // this wavefront's reads are done and stage s has arrived (up to STAGES - 2 behind it are on their way), for every wavefront
  const auto meet = [&](int s) {
    wait_behind<STAGES - 2, LOADS>(steps - 1 - s);
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
  };
  Fragments f0, f1;
  for (int s = 0; s < STAGES - 1 && s < steps; ++s) request(s, s);
  meet(0);
  if (STAGES - 1 < steps) request(STAGES - 1, STAGES - 1);
  fetch(0, 0, f0);
  int slot = 0;
#pragma unroll 1
  for (int s = 0; s < steps; ++s) {
    fetch(slot, 1, f1);
    __builtin_amdgcn_sched_barrier(0);
    multiply(f0);
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_waitcnt(0xc07f);                       // (f1: as the builtin, since of an instruction in assembly the compiler does not know what it waited for)
    asm volatile("" ::: "memory");
    if (s + 1 < steps) {
      const int next = slot + 1 == STAGES ? 0 : slot + 1;
      meet(s + 1);
      if (s + STAGES < steps) request(s + STAGES, slot);
      fetch(next, 0, f0);
      slot = next;
    }
    __builtin_amdgcn_sched_barrier(0);
    multiply(f1);
  }
  // 32 rows at a time turn in this wavefront's LDS, so that a lane has eight neighbouring results and a row's are stored together
  constexpr int PITCH = 32 * TN + 4, LANES = 4 * TN, ROWS = 64 / LANES;
  static_assert(WAVES * 32 * PITCH * 4 <= STAGE * STAGES, "the sums fit where the operands were");
  __syncthreads();
  int* turn = (int*)s_stage + wave * 32 * PITCH;
  const int col = lane % LANES * 8, n = n0 + wn + col;
  float ws[8], bias[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const int c = n + e < a.N ? n + e : a.N - 1;
    ws[e] = a.ws[c], bias[e] = a.bias ? a.bias[c] : 0.f;
  }
#pragma unroll
  for (int i = 0; i < TM; ++i) {
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        *(i32x4_t*)(turn + r * PITCH + 32 * j + 8 * e + 4 * half) = i32x4_t{acc[i][j][4 * e], acc[i][j][4 * e + 1], acc[i][j][4 * e + 2], acc[i][j][4 * e + 3]};
#pragma unroll
    for (int p = 0; p < 32 / ROWS; ++p) {
      const int row = p * ROWS + lane / LANES, m = m0 + wm + 32 * i + row;
      const i32x4_t lo = *(const i32x4_t*)(turn + row * PITCH + col), hi = *(const i32x4_t*)(turn + row * PITCH + col + 4);
      if (m >= a.M) continue;
      if (splits > 1) {                                       // (the sums of the shares are added by quant_finish_kernel)
        int* to = a.part + ((long long)split * a.M + m) * a.part_pitch + n;
        if (n < a.part_pitch) *(i32x4_t*)to = lo, *(i32x4_t*)(to + 4) = hi;
      } else store8<T>(a, m, n, lo, hi, a.xs[m], ws, bias);
    }
  }
}

// The shares of a product whose K was split, added (whole numbers: in any order), and its results.  (A thread has eight columns; 32 x 4096 of 8 shares: 4.6 us, a launch and two trips to memory.)
template <typename T>
__global__ __launch_bounds__(256) void quant_finish_kernel(QuantMatmulArgs a, int splits) {
  const int eights = a.part_pitch / 8, at = (int)blockIdx.x * 256 + (int)threadIdx.x, m = at / eights, n = (at - m * eights) * 8;
  if (m >= a.M) return;
  const int* from = a.part + (long long)m * a.part_pitch + n;
  i32x4_t lo = {0, 0, 0, 0}, hi = lo;
#pragma unroll 4
  for (int s = 0; s < splits; ++s) {
    lo += *(const i32x4_t*)(from + (long long)s * a.M * a.part_pitch);
    hi += *(const i32x4_t*)(from + (long long)s * a.M * a.part_pitch + 4);
  }
  float ws[8], bias[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const int c = n + e < a.N ? n + e : a.N - 1;
    ws[e] = a.ws[c], bias[e] = a.bias ? a.bias[c] : 0.f;
  }
  store8<T>(a, m, n, lo, hi, a.xs[m], ws, bias);
}

template <typename T, int WM, int WN, int TM, int TN, int STAGES>
static int quant_tiles_of(const QuantMatmulArgs& a, int splits, hipStream_t st) {
  constexpr int BM = 32 * TM * WM, BN = 32 * TN * WN, lds = (BM + BN) * 128 * STAGES;
  static PerDevice raised;
  const int tiles_m = (a.M + BM - 1) / BM, tiles_n = (a.N + BN - 1) / BN;
  const hipError_t e = raise_lds_limit(quant_matmul_kernel<T, WM, WN, TM, TN, STAGES>, raised);
  if (e != hipSuccess) return (int)e;
  quant_matmul_kernel<T, WM, WN, TM, TN, STAGES><<<(tiles_m * tiles_n * splits + NUM_XCD - 1) / NUM_XCD * NUM_XCD, 64 * WM * WN, lds, st>>>(a, tiles_m, tiles_n, splits);
  if (splits > 1) quant_finish_kernel<T><<<(int)(((long long)a.M * (a.part_pitch / 8) + 255) / 256), 256, 0, st>>>(a, splits);
  return (int)hipGetLastError();
}
static long long quant_tiles_in(int M, int N, int edge) { return (long long)((M + edge - 1) / edge) * ((N + edge - 1) / edge); }
// The largest tiles that leave every unit one.  us in tiles of 256, 128, 64: 8192 x 8192 x 8192: 480 to 590, 563 to 600; 2048 x 4096 x 4096: 57, 42; 512 x 4096 x 4096: -, 25, 16.5.
template <typename T>
static int quant_tiles(const QuantMatmulArgs& a, hipStream_t st) {
  if (quant_tiles_in(a.M, a.N, 256) >= 256) return quant_tiles_of<T, 2, 4, 4, 2, 2>(a, 1, st);
  if (quant_tiles_in(a.M, a.N, 128) >= 256) return quant_tiles_of<T, 2, 2, 2, 2, 2>(a, 1, st);
  return quant_tiles_of<T, 2, 2, 1, 1, 4>(a, a.part ? quant_splits(a.M, a.N, a.pitch) : 1, st);
}

template <typename T>
static int quant_matmul(const QuantMatmulArgs& a, hipStream_t st) {
  // Up to 64 rows whose x every workgroup can read for itself: 16 columns a workgroup.  Beyond 128 KB of x that reading costs more than the weights do (32 x 25088 x 4096: 35 us, in
  // shares 23; 32 x 4096 x 4096: 7.6, in tiles 12), and with 256 tiles of 64 columns or more those stream the weights faster (1 x 4096 x 16384: 18 us, in tiles 13).
  const bool few = a.M <= 64 && quant_tiles_in(a.M, a.N, 64) < 256 && (!a.part || a.M * a.pitch <= 131072);
  const int nt = (a.N + 15) / 16;
  const QuantRowsArgs none{};
  if (!few) return quant_tiles<T>(a, st);
  if (a.M <= 16) quant_matvec_kernel<T, 1, false><<<nt, 512, 0, st>>>(a, none);
  else if (a.M <= 32) quant_matvec_kernel<T, 2, false><<<nt, 512, 0, st>>>(a, none);
  else quant_matvec_kernel<T, 4, false><<<nt, 512, 0, st>>>(a, none);
  return (int)hipGetLastError();
}
int launch_quant_matmul(const QuantMatmulArgs& a, int dtype, void* stream) {
  return dtype ? quant_matmul<bf16_t>(a, (hipStream_t)stream) : quant_matmul<float>(a, (hipStream_t)stream);
}

int launch_linear(const QuantRowsArgs& r, const QuantMatmulArgs& a, int dtype, void* stream) {
  if (linear_in_one(a.M, a.pitch, a.N)) {
    const int nt = (a.N + 15) / 16, lds = a.M * (int)a.pitch;
    if (dtype) quant_matvec_kernel<bf16_t, 1, true><<<nt, 512, lds, (hipStream_t)stream>>>(a, r);
    else quant_matvec_kernel<float, 1, true><<<nt, 512, lds, (hipStream_t)stream>>>(a, r);
    return (int)hipGetLastError();
  }
  const int err = launch_quant_rows(r, dtype, stream);
  return err ? err : launch_quant_matmul(a, dtype, stream);
}

}  // namespace xenos
