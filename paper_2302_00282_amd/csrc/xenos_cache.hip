// The quantised cache of keys and values: rows into it, and back.
#include "token_device.h"

namespace xenos {

// A workgroup has 16 tokens of one head.  Their slots, and whether they are a run (neighbours, as those of a prompt are but at the seams of its pages): then the
// values lie in one or two blocks of 16 tokens and move in words and whole blocks, else byte by byte.
constexpr int kGroup = 16, kMostDim = 256;
// Which group and head a workgroup has: the heads of a group follow one another on one XCD, whose L2 puts together the lines that two heads' rows share.
struct Share {
  int group, head;
  __device__ __forceinline__ explicit Share(int heads) {
    const int at = (int)blockIdx.x / NUM_XCD;
    group = at / heads * NUM_XCD + (int)blockIdx.x % NUM_XCD, head = at % heads;
  }
};
struct Group {
  long long row[kGroup];                                      // a token's row among those of all pages and heads, -1: it has none
  int low[kGroup];                                            // its place in its block of 16
  int run;
};
__device__ __forceinline__ void group_slots(const CacheArgs& c, const long long* slots, int first, int n, int h, Group& g) {
  if (threadIdx.x < 64) {
    const int t = (int)threadIdx.x;
    const long long s = t < n ? slots[first + t] : -1;
    const bool in = s >= 0 && s < (long long)c.n_pages * c.page;
    const bool all = __all(t >= n || (in && s == __shfl(s, 0) + t));
    if (t < kGroup) {
      const long long page = in ? s / c.page : 0;             // (the only division by the page of a group's whole work)
      g.row[t] = in ? (page * c.heads + h) * c.page + (s - page * c.page) : -1;
      g.low[t] = (int)(s & 15);
    }
    if (t == 0) g.run = all;
  }
  __syncthreads();
}
// Offset of dimension 0 in the block of 16 values a token lies in
__device__ __forceinline__ long long block_of(const CacheArgs& c, const Group& g, int t) { return (g.row[t] - g.low[t]) * c.dim; }

// Bound by memory: 8197 fp32 tokens of 10 heads of 80 take 23 us, 66 MB read and written at 2.9 TB/s (the launch fills 5200 workgroups, each with three trips after one another: slots, elements, scales).
// Rows of four elements each: the largest magnitude of a row meets in LDS, the quantised keys go out in words, the values turn in LDS.
template <typename T>
__global__ __launch_bounds__(256) void cache_write_kernel(CacheWriteArgs a) {
  __shared__ Group s_group;
  __shared__ uint32_t s_max[2][kGroup];
  __shared__ int8_t s_v[kMostDim][kGroup + 1];                // (the odd pitch spreads a wavefront's writes over the banks)
  const Share mine(a.c.heads);
  const int first = mine.group * kGroup, h = mine.head, n = a.tokens - first < kGroup ? a.tokens - first : kGroup;
  if (n <= 0) return;
  const int dim = a.c.dim, quads = dim / 4, per = kGroup * quads;   // fours of a row; of the group's keys (as many of its values)
  const SmallDiv by_quads(quads), by_dim(dim);
  if (threadIdx.x < 2 * kGroup) s_max[threadIdx.x / kGroup][threadIdx.x % kGroup] = 0;
  constexpr int MOST = 2 * kGroup * (kMostDim / 4) / 256;
  float f[MOST][4];
#pragma unroll
  for (int i = 0; i < MOST; ++i) {
    const int id = (int)threadIdx.x + 256 * i;
    if (id >= 2 * per) break;
    const bool is_v = id >= per;
    const int at = is_v ? id - per : id, t = by_quads(at), d = (at - t * quads) * 4;
    if (t < n) {
      const T* src = is_v ? (const T*)a.v + (first + t) * a.v_token + h * a.v_head + d : (const T*)a.k + (first + t) * a.k_token + h * a.k_head + d;
      if (a.vec && sizeof(T) == 4) {
        const float4 x = *(const float4*)src;
        f[i][0] = x.x, f[i][1] = x.y, f[i][2] = x.z, f[i][3] = x.w;
      } else if (a.vec) {
        const uint2 x = *(const uint2*)src;
        f[i][0] = bf2f(x.x & 0xffff), f[i][1] = bf2f(x.x >> 16), f[i][2] = bf2f(x.y & 0xffff), f[i][3] = bf2f(x.y >> 16);
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) f[i][e] = Tr<T>::ld(src, e);
      }
    }
  }
  group_slots(a.c, a.slots, first, n, h, s_group);            // (behind the requests for the rows, which do not wait for it)
#pragma unroll
  for (int i = 0; i < MOST; ++i) {
    const int id = (int)threadIdx.x + 256 * i;
    if (id >= 2 * per) break;
    const bool is_v = id >= per;
    const int t = by_quads(is_v ? id - per : id);
    if (t >= n) continue;
    uint32_t m = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) m = umax(m, magnitude(f[i][e]));
    atomicMax(&s_max[is_v][t], m);
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < MOST; ++i) {
    const int id = (int)threadIdx.x + 256 * i;
    if (id >= 2 * per) break;
    const bool is_v = id >= per;
    const int at = is_v ? id - per : id, t = by_quads(at), d = (at - t * quads) * 4;
    if (t >= n) continue;
    const RowStep step(s_max[is_v][t]);
    uint32_t w = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) w |= ((uint32_t)step(f[i][e]) & 0xffu) << (8 * e);
    if (is_v) {
#pragma unroll
      for (int e = 0; e < 4; ++e) s_v[d + e][t] = (int8_t)(w >> (8 * e));
    }
    const long long row = s_group.row[t];
    if (row < 0) continue;
    if (!is_v) *(uint32_t*)(a.c.k + row * dim + d) = w;
    if (d == 0) (is_v ? a.c.v_scale : a.c.k_scale)[row] = step.scale();
  }
  __syncthreads();
  if (s_group.run) {
    // word w of the 32 bytes that the run's first block and the next one hold of dimension d: token 4 w - off of the group in its lowest byte
    const int off = s_group.low[0], blocks = (off + n + 15) / 16;
    const long long block0 = block_of(a.c, s_group, 0), block1 = blocks > 1 ? block_of(a.c, s_group, 16 - off) : 0;
    for (int id = (int)threadIdx.x; id < dim * 4 * blocks; id += 256) {
      const int w = by_dim(id), d = id - w * dim, t = 4 * w - off;
      int8_t* at = a.c.v + (w >= 4 ? block1 : block0) + d * 16 + 4 * (w & 3);
      if (t >= 0 && t + 4 <= n) {
        uint32_t x = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) x |= (uint32_t)(uint8_t)s_v[d][t + e] << (8 * e);
        *(uint32_t*)at = x;
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (t + e >= 0 && t + e < n) at[e] = s_v[d][t + e];
      }
    }
  } else {
    for (int id = (int)threadIdx.x; id < dim * n; id += 256) {
      const int t = by_dim(id), d = id - t * dim;
      if (s_group.row[t] >= 0) a.c.v[block_of(a.c, s_group, t) + d * 16 + s_group.low[t]] = s_v[d][t];
    }
  }
}

// As write, backwards: 22 us, 3.0 TB/s at the same size.  Sixteen values of a token at a time, the values turned in LDS first.
template <typename T>
__global__ __launch_bounds__(256) void cache_read_kernel(CacheReadArgs a) {
  __shared__ Group s_group;
  __shared__ __attribute__((aligned(16))) int8_t s_v[kGroup][kMostDim + 16];
  const Share mine(a.c.heads);
  const int first = mine.group * kGroup, h = mine.head, n = a.tokens - first < kGroup ? a.tokens - first : kGroup;
  if (n <= 0) return;
  group_slots(a.c, a.slots, first, n, h, s_group);
  // a thread has sixteen dimensions of at most one token (16 tokens of at most 256); its keys are on their way while the values turn
  const int dim = a.c.dim, chunks = dim / 16;
  const int t = SmallDiv(chunks)((int)threadIdx.x), d = ((int)threadIdx.x - t * chunks) * 16;
  const long long row = t < n ? s_group.row[t] : -1;
  u32x4_t key = {0, 0, 0, 0};
  float k_scale = 0.f, v_scale = 0.f;
  if (row >= 0) key = *(const u32x4_t*)(a.c.k + row * dim + d), k_scale = a.c.k_scale[row], v_scale = a.c.v_scale[row];
  if (s_group.run) {
    const int off = s_group.low[0], blocks = (off + n + 15) / 16;
    const long long block0 = block_of(a.c, s_group, 0), block1 = blocks > 1 ? block_of(a.c, s_group, 16 - off) : 0;
    u32x4_t x[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int id = (int)threadIdx.x + 256 * i, b = id >= dim;
      if (id < dim * blocks) x[i] = *(const u32x4_t*)(a.c.v + (b ? block1 : block0) + (id - b * dim) * 16);
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int id = (int)threadIdx.x + 256 * i, b = id >= dim;
      if (id >= dim * blocks) continue;
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const int at = 16 * b + e - off;
        if (at >= 0 && at < n) s_v[at][id - b * dim] = (int8_t)(x[i][e >> 2] >> (8 * (e & 3)));
      }
    }
  } else {
    const SmallDiv by_dim(dim);
    for (int id = (int)threadIdx.x; id < dim * n; id += 256) {
      const int at = by_dim(id), e = id - at * dim;
      if (s_group.row[at] >= 0) s_v[at][e] = a.c.v[block_of(a.c, s_group, at) + e * 16 + s_group.low[at]];
    }
  }
  const auto give = [&](void* to, const u32x4_t& x, float scale) {
    T* out = (T*)to + ((long long)(first + t) * a.c.heads + h) * dim + d;
#pragma unroll
    for (int c = 0; c < 16 / Tr<T>::CE; ++c) {
      float y[Tr<T>::CE];
#pragma unroll
      for (int e = 0; e < Tr<T>::CE; ++e) y[e] = (float)(int8_t)(x[(c * Tr<T>::CE + e) >> 2] >> (8 * ((c * Tr<T>::CE + e) & 3))) * scale;
      *(u32x4_t*)(out + c * Tr<T>::CE) = Tr<T>::pack(y);
    }
  };
  if (t < n) give(a.k, key, k_scale);
  __syncthreads();
  if (t < n) give(a.v, row >= 0 ? *(const u32x4_t*)&s_v[t][d] : u32x4_t{0, 0, 0, 0}, v_scale);
}

template <typename F, typename A>
static int per_group(F* kernel, const A& a, void* stream) {
  kernel<<<(a.tokens + kGroup * NUM_XCD - 1) / (kGroup * NUM_XCD) * NUM_XCD * a.c.heads, 256, 0, (hipStream_t)stream>>>(a);
  return (int)hipGetLastError();
}
int launch_cache_write(const CacheWriteArgs& a, int dtype, void* stream) {
  return dtype ? per_group(cache_write_kernel<bf16_t>, a, stream) : per_group(cache_write_kernel<float>, a, stream);
}
int launch_cache_read(const CacheReadArgs& a, int dtype, void* stream) {
  return dtype ? per_group(cache_read_kernel<bf16_t>, a, stream) : per_group(cache_read_kernel<float>, a, stream);
}

}  // namespace xenos
