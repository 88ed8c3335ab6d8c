// The quantised cache of keys and values: rows into it, and back.
#include "token_device.h"

namespace xenos {

// Where a slot's row of head h lies, and whether there is such a slot.
struct CacheRow {
  long long first;                                            // of the head's page_tokens rows of `page`
  int at;                                                     // token in the page
  bool ok;
  __device__ __forceinline__ CacheRow(const CacheArgs& c, long long slot, int h) {
    const long long page = slot / c.page;
    ok = slot >= 0 && page < c.n_pages;
    at = ok ? (int)(slot - page * c.page) : 0;
    first = ok ? (page * c.heads + h) * c.page : 0;
  }
  __device__ __forceinline__ long long k(const CacheArgs& c, int d) const { return (first + at) * c.dim + d; }
  __device__ __forceinline__ long long v(const CacheArgs& c, int d) const { return first * c.dim + ((long long)(at >> 4) * c.dim + d) * 16 + (at & 15); }
};

// A wavefront per token and head.
template <typename T>
__global__ __launch_bounds__(256) void cache_write_kernel(CacheWriteArgs a) {
  const int row = (int)blockIdx.x * 4 + (int)(threadIdx.x >> 6), lane = threadIdx.x & 63;
  if (row >= a.tokens * a.c.heads) return;
  const int t = row / a.c.heads, h = row - t * a.c.heads;
  const CacheRow to(a.c, a.slots[t], h);
  if (!to.ok) return;
#pragma unroll
  for (int part = 0; part < 2; ++part) {
    const T* src = part ? (const T*)a.v + t * a.v_token + h * a.v_head : (const T*)a.k + t * a.k_token + h * a.k_head;
    float f[4];
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      f[i] = lane + 64 * i < a.c.dim ? Tr<T>::ld(src, lane + 64 * i) : 0.f;
      m = umax(m, magnitude(f[i]));
    }
    const RowStep step(wave_max(m));
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int d = lane + 64 * i;
      if (d < a.c.dim) (part ? a.c.v[to.v(a.c, d)] : a.c.k[to.k(a.c, d)]) = (int8_t)step(f[i]);
    }
    if (lane == 0) (part ? a.c.v_scale : a.c.k_scale)[to.first + to.at] = step.scale();
  }
}

template <typename T>
__global__ __launch_bounds__(256) void cache_read_kernel(CacheReadArgs a) {
  const int row = (int)blockIdx.x * 4 + (int)(threadIdx.x >> 6), lane = threadIdx.x & 63;
  if (row >= a.tokens * a.c.heads) return;
  const int t = row / a.c.heads, h = row - t * a.c.heads;
  const CacheRow from(a.c, a.slots[t], h);
  const float ks = from.ok ? a.c.k_scale[from.first + from.at] : 0.f, vs = from.ok ? a.c.v_scale[from.first + from.at] : 0.f;
  for (int d = lane; d < a.c.dim; d += 64) {
    Tr<T>::st(a.k, (long long)row * a.c.dim + d, from.ok ? (float)a.c.k[from.k(a.c, d)] * ks : 0.f);
    Tr<T>::st(a.v, (long long)row * a.c.dim + d, from.ok ? (float)a.c.v[from.v(a.c, d)] * vs : 0.f);
  }
}

template <typename F, typename A>
static int per_row(F* kernel, const A& a, void* stream) {
  kernel<<<(a.tokens * a.c.heads + 3) / 4, 256, 0, (hipStream_t)stream>>>(a);
  return (int)hipGetLastError();
}
int launch_cache_write(const CacheWriteArgs& a, int dtype, void* stream) {
  return dtype ? per_row(cache_write_kernel<bf16_t>, a, stream) : per_row(cache_write_kernel<float>, a, stream);
}
int launch_cache_read(const CacheReadArgs& a, int dtype, void* stream) {
  return dtype ? per_row(cache_read_kernel<bf16_t>, a, stream) : per_row(cache_read_kernel<float>, a, stream);
}

}  // namespace xenos
