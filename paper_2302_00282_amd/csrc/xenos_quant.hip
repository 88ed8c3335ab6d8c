// Rows in 8-bit integers with a scale each, and their product: the linear layers of a token model.
#include "device_common.h"
#include "token_device.h"

namespace xenos {

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
__device__ __forceinline__ void times_gamma(const QuantRowsArgs& a, int i, const float* f, float* v) {
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = a.gamma ? f[e] * (i + e < a.cols ? a.gamma[i + e] : 0.f) : f[e];
}
__device__ __forceinline__ uint2 packed8(const RowStep& step, const float* v) {
  uint32_t w[2] = {0, 0};
#pragma unroll
  for (int e = 0; e < 8; ++e) w[e >> 2] |= ((uint32_t)step(v[e]) & 0xffu) << (8 * (e & 3));
  return make_uint2(w[0], w[1]);
}
__device__ __forceinline__ float row_scale(const QuantRowsArgs& a, const RowStep& step, float sq) {
  return a.gamma ? step.scale() * (1.f / sqrtf(sq / (float)a.cols + a.eps)) : step.scale();
}

// One workgroup per row: q = rint(x g 127 / a), a = max|x g|, scale = a / 127 [/ rms(x)].  The norm's factor is one number per row: it
// cancels in q, so that the rounded values do not depend on how the squares are summed.  Two passes over the row, the second from the cache.
template <typename T>
__global__ __launch_bounds__(1024) void quant_rows_kernel(QuantRowsArgs a) {
  __shared__ uint32_t s_max[16];
  __shared__ float s_sum[16];
  const int step = (int)blockDim.x * 8, waves = (int)blockDim.x / 64;
  for (int at = (int)blockIdx.x; at < a.rows; at += (int)gridDim.x) {
    const T* row = (const T*)a.x + at * a.stride;
    int8_t* q = a.q + at * a.pitch;
    uint32_t m = 0;
    float sq = 0.f;
    for (int i = (int)threadIdx.x * 8; i < a.cols; i += step) {
      float f[8], v[8];
      load8<T>(row, i, a.cols, a.vec, f);
      times_gamma(a, i, f, v);
#pragma unroll
      for (int e = 0; e < 8; ++e) sq += f[e] * f[e], m = umax(m, magnitude(v[e]));
    }
    m = wave_max(m);
    sq = wave_sum(sq);
    if ((threadIdx.x & 63) == 0) { s_max[threadIdx.x >> 6] = m; s_sum[threadIdx.x >> 6] = sq; }
    __syncthreads();
    m = 0, sq = 0.f;
    for (int w = 0; w < waves; ++w) { m = umax(m, s_max[w]); sq += s_sum[w]; }
    const RowStep unit(m);
    for (int i = (int)threadIdx.x * 8; i < (int)a.pitch; i += step) {
      float f[8], v[8];
      load8<T>(row, i, a.cols, a.vec, f);
      times_gamma(a, i, f, v);
      *(uint2*)(q + i) = packed8(unit, v);
    }
    if (threadIdx.x == 0) a.scale[at] = row_scale(a, unit, sq);
    __syncthreads();                                          // (s_max and s_sum are free again)
  }
}

template <typename T>
static int quant_rows(const QuantRowsArgs& a, hipStream_t st) {
  const int threads = a.pitch <= 2048 ? 256 : 1024, grid = a.rows < 65536 ? a.rows : 65536;
  quant_rows_kernel<T><<<grid, threads, 0, st>>>(a);
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
      times_gamma(a, i, f, v);
#pragma unroll
      for (int e = 0; e < 8; ++e) sq += f[e] * f[e], m = umax(m, magnitude(v[e]));
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
      times_gamma(a, i, f, v);
      *(uint2*)(q + r * a.pitch + i) = packed8(step, v);
    }
    if (piece == 0 && lane == 0) {
      float sq = 0.f;
      for (int w = 0; w < share; ++w) sq += s_sum[r][w];
      scale[r] = row_scale(a, step, sq);
    }
  }
  __syncthreads();
}

// Few rows: the weights are the work.  A workgroup has 16 output channels and all of K, which its wavefronts share; every fragment of the weights goes
// from memory to registers, a lane's 16 bytes of one weight row at a time, and the sums (whole numbers: exact in any order) meet in LDS.
// OWN: x comes as it is, and every workgroup quantises all of it for itself.
template <typename T, int MT, bool OWN>
__global__ __launch_bounds__(512) void quant_matvec_kernel(QuantMatmulArgs a, QuantRowsArgs qa) {
  __shared__ i32x4_t part[8][MT][64];
  extern __shared__ __attribute__((aligned(16))) int8_t s_q[];
  __shared__ float s_scale[16];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = lane & 15, g = lane >> 4;
  const int n0 = (int)blockIdx.x * 16, pitch = (int)a.pitch;
  const int8_t* w = a.w + (long long)(n0 + r < a.N ? n0 + r : a.N - 1) * a.pitch + g * 16;
  if (OWN) quant_into_lds<T>(qa, s_q, s_scale);
  const int8_t* x[MT];
#pragma unroll
  for (int t = 0; t < MT; ++t) x[t] = (OWN ? s_q : a.x) + (16 * t + r < a.M ? 16 * t + r : a.M - 1) * a.pitch + g * 16;
  i32x4_t acc[MT] = {};
#pragma unroll 4
  for (int k = wave * 128; k < pitch; k += 1024) {
    const i32x4_t w0 = *(const i32x4_t*)(w + k), w1 = *(const i32x4_t*)(w + k + 64);
#pragma unroll
    for (int t = 0; t < MT; ++t) {
      acc[t] = __builtin_amdgcn_mfma_i32_16x16x64_i8(w0, *(const i32x4_t*)(x[t] + k), acc[t], 0, 0, 0);
      acc[t] = __builtin_amdgcn_mfma_i32_16x16x64_i8(w1, *(const i32x4_t*)(x[t] + k + 64), acc[t], 0, 0, 0);
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

// Many rows: tiles of 128 x 128 with the next 128 bytes of K on their way in registers while the matrix unit works on the present ones in LDS.
template <typename T>
__global__ __launch_bounds__(256) void quant_matmul_kernel(QuantMatmulArgs a) {
  constexpr int ROW = 144;                                    // bytes: nine 16-byte slots, so that neighbouring rows start at other banks
  __shared__ __attribute__((aligned(16))) int8_t lds[2][256][ROW];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = lane & 15, g = lane >> 4;
  const int tiles_m = (a.M + 127) / 128, n0 = (int)blockIdx.x / tiles_m * 128, m0 = (int)blockIdx.x % tiles_m * 128;
  const int wn = (wave & 1) * 64, wm = (wave >> 1) * 64;
  i32x4_t acc[4][4] = {}, next[8];
  const int8_t* src[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int row = (int)threadIdx.x / 8 + 32 * i;
    const int n = n0 + row, m = m0 + row - 128;
    src[i] = (i < 4 ? a.w + (long long)(n < a.N ? n : a.N - 1) * a.pitch : a.x + (long long)(m < a.M ? m : a.M - 1) * a.pitch) + threadIdx.x % 8 * 16;
    next[i] = *(const i32x4_t*)src[i];
  }
  const int steps = (int)(a.pitch / 128);
  for (int s = 0; s < steps; ++s) {
#pragma unroll
    for (int i = 0; i < 8; ++i) *(i32x4_t*)&lds[s & 1][threadIdx.x / 8 + 32 * i][threadIdx.x % 8 * 16] = next[i];
    __syncthreads();
    if (s + 1 < steps) {
#pragma unroll
      for (int i = 0; i < 8; ++i) next[i] = *(const i32x4_t*)(src[i] + (long long)(s + 1) * 128);
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      i32x4_t w[4], x[4];
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        w[t] = *(const i32x4_t*)&lds[s & 1][wn + 16 * t + r][64 * h + 16 * g];
        x[t] = *(const i32x4_t*)&lds[s & 1][128 + wm + 16 * t + r][64 * h + 16 * g];
      }
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(w[i], x[j], acc[i][j], 0, 0, 0);
    }
  }
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int m = m0 + wm + 16 * j + r;
    const float xs = m < a.M ? a.xs[m] : 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) store4<T>(a, m, n0 + wn + 16 * i + 4 * g, acc[i][j], xs);
  }
}

template <typename T>
static int quant_matmul(const QuantMatmulArgs& a, hipStream_t st) {
  const int nt = (a.N + 15) / 16;
  const QuantRowsArgs none{};
  if (a.M <= 16) quant_matvec_kernel<T, 1, false><<<nt, 512, 0, st>>>(a, none);
  else if (a.M <= 32) quant_matvec_kernel<T, 2, false><<<nt, 512, 0, st>>>(a, none);
  else if (a.M <= 64) quant_matvec_kernel<T, 4, false><<<nt, 512, 0, st>>>(a, none);
  else quant_matmul_kernel<T><<<(a.N + 127) / 128 * ((a.M + 127) / 128), 256, 0, st>>>(a);
  return (int)hipGetLastError();
}
int launch_quant_matmul(const QuantMatmulArgs& a, int dtype, void* stream) {
  return dtype ? quant_matmul<bf16_t>(a, (hipStream_t)stream) : quant_matmul<float>(a, (hipStream_t)stream);
}

int launch_linear(const QuantRowsArgs& r, const QuantMatmulArgs& a, int dtype, void* stream) {
  if (linear_in_one(a.M, a.pitch)) {
    const int nt = (a.N + 15) / 16, lds = a.M * (int)a.pitch;
    if (dtype) quant_matvec_kernel<bf16_t, 1, true><<<nt, 512, lds, (hipStream_t)stream>>>(a, r);
    else quant_matvec_kernel<float, 1, true><<<nt, 512, lds, (hipStream_t)stream>>>(a, r);
    return (int)hipGetLastError();
  }
  const int err = launch_quant_rows(r, dtype, stream);
  return err ? err : launch_quant_matmul(a, dtype, stream);
}

}  // namespace xenos
