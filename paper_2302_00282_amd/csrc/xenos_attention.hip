// Attention of a batch of sequences to the quantised cache, with a prefix they share.
//
// Keys pass once, 64 at a time, with the running maximum m and sum l of a softmax per row.  The scores are computed transposed, S^T = K Q^T, so that a lane ends up with
// 16 neighbouring keys of one row (tile t of a wavefront's four takes key 16 (r / 4) + 4 t + r % 4 as its row r): the maximum is over registers and two exchanges, and the lane's
// probabilities are, as they lie, the operand of O^T += V^T P^T, whose other operand is what the cache holds for one dimension: 16 keys side by side.
// Nothing passes through LDS.  The 8-bit keys become bf16 and the values fp16 without rounding; the keys' scales multiply the scores, the values' the probabilities.
// Those are rounded to fp16 for the product, after division by the largest value scale so far: eight times as fine as bf16, whose error would be as large as that of the
// rounding of the result (relative error of the output against 64 bits: 1.7e-3 in place of 2.4e-3), and in range whatever the scales are.
#include <algorithm>
#include <math.h>
#include "token_device.h"

namespace xenos {

namespace {

constexpr int kKeys = 64;                                     // of a step
constexpr int kWaves = 4;

// Eight bytes as bf16: whole numbers up to 127, exact.
__device__ __forceinline__ bf16x8_t whole8(uint32_t lo, uint32_t hi) {
  u32x4_t w;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const uint32_t v = e < 2 ? lo : hi;
    w[e] = f2bf2((float)(int8_t)(v >> (16 * (e & 1))), (float)(int8_t)(v >> (16 * (e & 1) + 8)));
  }
  return __builtin_bit_cast(bf16x8_t, w);
}

typedef __attribute__((ext_vector_type(8))) _Float16 f16x8_t;
typedef __attribute__((ext_vector_type(2))) _Float16 f16x2_t;

// Eight bytes as fp16: a byte plus 128 below the bits of 1024 is 1024 + 128 + the byte.
__device__ __forceinline__ f16x8_t half8(uint32_t lo, uint32_t hi) {
  const f16x2_t off = {(_Float16)-1152.f, (_Float16)-1152.f};
  lo ^= 0x80808080u, hi ^= 0x80808080u;
  u32x4_t w;
#pragma unroll
  for (int e = 0; e < 4; ++e)
    w[e] = __builtin_bit_cast(uint32_t, __builtin_bit_cast(f16x2_t, __builtin_amdgcn_perm(0x64646464u, e < 2 ? lo : hi, e & 1 ? 0x04030402u : 0x04010400u)) + off);
  return __builtin_bit_cast(f16x8_t, w);
}
__device__ __forceinline__ uint32_t f2h2(float lo, float hi) { return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2_t){lo, hi}, f16x2_t)); }

// What a workgroup does: rows of queries, and a piece of the keys they see.
struct Item {
  int head;                                                   // of the cache
  const int* table;
  int tokens;                                                 // of the segment
  int first_query, queries;
  int row0, rows;                                             // first row of the tile; rows of the item in all (queries times the group)
  int begin, end;                                             // keys
  int slot;
  bool prefix, whole;
};

__device__ __forceinline__ Item item_of(const AttentionArgs& a, int at, int waves_rows) {
  Item it;
  const int front = a.prefix.parts * a.prefix.tiles * a.c.heads;
  it.prefix = at < front;
  const AttentionShare& s = it.prefix ? a.prefix : a.own;
  if (!it.prefix) at -= front;
  const int tile = at % s.tiles;
  at /= s.tiles;
  it.head = at % a.c.heads;
  at /= a.c.heads;
  const int part = at % s.parts, seq = at / s.parts;
  it.whole = s.whole;
  if (it.prefix) {
    it.table = a.prefix_table, it.tokens = a.prefix_len, it.first_query = 0, it.queries = a.n_queries, it.slot = part;
  } else {
    const long long held = (long long)a.table_stride * a.c.page;
    const int n = a.lengths[seq];
    it.table = a.tables + (long long)seq * a.table_stride;
    it.tokens = n < 0 ? 0 : n < held ? n : (int)held;
    const int lo = a.starts ? a.starts[seq] : seq, hi = a.starts ? a.starts[seq + 1] : seq + 1;
    it.first_query = lo < 0 ? 0 : lo < a.n_queries ? lo : a.n_queries;
    it.queries = hi <= it.first_query ? 0 : (hi < a.n_queries ? hi : a.n_queries) - it.first_query;
    it.slot = a.prefix.parts + part;
  }
  if (a.c.n_pages == 0) it.tokens = 0;
  it.rows = it.queries * a.group;
  it.row0 = tile * (it.whole ? waves_rows : kWaves * waves_rows);
  it.begin = part * s.part_len;
  it.end = part == s.parts - 1 || it.begin + s.part_len > it.tokens ? it.tokens : it.begin + s.part_len;
  return it;
}

// NB: blocks of 64 dimensions; MT: tiles of 16 rows per wavefront.
template <int NB, int MT>
__global__ __launch_bounds__(64 * kWaves) void attention_kernel(AttentionArgs a) {
  constexpr int DT = 4 * NB, REC = MT * (4 * DT + 2);         // tiles of 16 dimensions; floats of a lane's state
  __shared__ float s_state[kWaves / 2][REC][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = lane & 15, g = lane >> 4, dim = a.c.dim;
  Item it = item_of(a, (int)blockIdx.x, 16 * MT);
  const AttentionShare& share = it.prefix ? a.prefix : a.own;
  const int step_rows = share.tiles * (it.whole ? 16 * MT : kWaves * 16 * MT);
  for (; it.row0 < it.rows; it.row0 += step_rows) {           // (once, unless a sequence has more queries than was said)
    const int row_first = it.row0 + (it.whole ? 0 : wave * 16 * MT);
    // rows of this lane: queries in bf16, and the keys they see
    bf16x8_t q[MT][NB][2];
    int limit[MT], least = 0x7fffffff, most = 0;
#pragma unroll
    for (int t = 0; t < MT; ++t) {
      const int row = row_first + 16 * t + r, query = row / a.group, h = it.head * a.group + row - query * a.group;
      const bool ok = row < it.rows;
      limit[t] = !ok ? 0 : it.prefix ? it.tokens : it.tokens - it.queries + query + 1;
      least = min(least, limit[t]), most = max(most, limit[t]);
      const uint16_t* src = a.q + (ok ? (long long)(it.first_query + query) * a.q_token + h * a.q_head : 0);
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          const int d = 64 * b + 16 * g + 8 * half;
          u32x4_t w = {0, 0, 0, 0};
          if (ok && d < dim) {
            if (a.vec_q) w = *(const u32x4_t*)(src + d);
            else {
#pragma unroll
              for (int e = 0; e < 8; ++e) w[e >> 1] |= (uint32_t)src[d + e] << (16 * (e & 1));
            }
          }
          q[t][b][half] = __builtin_bit_cast(bf16x8_t, w);
        }
    }
#pragma unroll
    for (int o = 1; o < 16; o <<= 1) least = min(least, __shfl_xor(least, o)), most = max(most, __shfl_xor(most, o));
    const int end = min(it.end, most);

    f32x4_t o[MT][DT];
    float m[MT], l[MT], unit = 7.5e-37f, unit_inv = 1.f / 7.5e-37f;   // (o counts in `unit`: the largest scale of a value so far)
#pragma unroll
    for (int t = 0; t < MT; ++t) {
      m[t] = -INFINITY, l[t] = 0.f;
#pragma unroll
      for (int d = 0; d < DT; ++d) o[t][d] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    }
    for (int key = it.begin + (it.whole ? wave * kKeys : 0); key < end; key += it.whole ? kWaves * kKeys : kKeys) {
      // the blocks of 16 keys that this lane reads: of keys (for the scores' rows) and of values
      const int kb = key + 16 * (r >> 2), vb = key + 16 * g;
      const int kp = kb < it.tokens ? it.table[kb / a.c.page] : -1, vp = vb < it.tokens ? it.table[vb / a.c.page] : -1;
      const bool k_ok = (unsigned)kp < (unsigned)a.c.n_pages, v_ok = (unsigned)vp < (unsigned)a.c.n_pages;
      const long long k_row = k_ok ? ((long long)kp * a.c.heads + it.head) * a.c.page + kb % a.c.page : 0;
      const long long v_row = v_ok ? ((long long)vp * a.c.heads + it.head) * a.c.page + vb % a.c.page : 0;
      const int8_t* kt = a.c.k + (k_row + (r & 3)) * dim + 16 * g;
      const int8_t* vt = a.c.v + v_row * dim + r * 16;
      u32x4_t k[4][NB], v[DT];
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int t = 0; t < 4; ++t) k[t][b] = 64 * b + 16 * g < dim ? *(const u32x4_t*)(kt + 4 * t * dim + 64 * b) : u32x4_t{0, 0, 0, 0};
      f32x4_t ks[4], vs[4];
#pragma unroll
      for (int t = 0; t < 4; ++t) ks[t] = *(const f32x4_t*)(a.c.k_scale + v_row + 4 * t), vs[t] = *(const f32x4_t*)(a.c.v_scale + v_row + 4 * t);
#pragma unroll
      for (int d = 0; d < DT; ++d) v[d] = 16 * d < dim ? *(const u32x4_t*)(vt + 256 * d) : u32x4_t{0, 0, 0, 0};

      f32x4_t s[MT][4];
#pragma unroll
      for (int t = 0; t < 4; ++t) {
#pragma unroll
        for (int j = 0; j < MT; ++j) s[j][t] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
          for (int half = 0; half < 2; ++half) {
            const bf16x8_t kk = whole8(k[t][b][2 * half], k[t][b][2 * half + 1]);
#pragma unroll
            for (int j = 0; j < MT; ++j) s[j][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kk, q[j][b][half], s[j][t], 0, 0, 0);
          }
        ks[t] *= a.scale2;
      }
      float rescale = 1.f;
      {
        float big = 0.f;
        const int there = v_ok ? it.tokens - vb : 0;
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
          for (int e = 0; e < 4; ++e) big = fmaxf(big, 4 * t + e < there && vs[t][e] < INFINITY ? vs[t][e] : 0.f);
        if (__any(big > unit)) {
          big = fmaxf(big, __shfl_xor(big, 16));
          big = fmaxf(big, __shfl_xor(big, 32));
          big = fmaxf(big, unit);
          rescale = unit / big;
          unit = big, unit_inv = 1.f / big;
        }
      }
      f16x8_t p[MT][2];
#pragma unroll
      for (int j = 0; j < MT; ++j) {
        const int seen = v_ok ? limit[j] - vb : 0;             // of this lane's 16 keys
        float top = m[j];
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            s[j][t][e] = 4 * t + e < seen ? s[j][t][e] * ks[t][e] : -INFINITY;
            top = fmaxf(top, s[j][t][e]);
          }
        top = fmaxf(top, __shfl_xor(top, 16));
        top = fmaxf(top, __shfl_xor(top, 32));
        const float base = top == -INFINITY ? 0.f : top, keep = __builtin_amdgcn_exp2f(m[j] - base);
        m[j] = top;
        float sum = 0.f;
        u32x4_t w[2];
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          float pv[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float x = __builtin_amdgcn_exp2f(s[j][t][e] - base);
            sum += x;
            pv[e] = 4 * t + e < seen ? x * (vs[t][e] * unit_inv) : 0.f;   // (a scale that was never written may be anything)
          }
          w[t >> 1][2 * (t & 1)] = f2h2(pv[0], pv[1]);
          w[t >> 1][2 * (t & 1) + 1] = f2h2(pv[2], pv[3]);
        }
        p[j][0] = __builtin_bit_cast(f16x8_t, w[0]), p[j][1] = __builtin_bit_cast(f16x8_t, w[1]);
        l[j] = l[j] * keep + sum;
#pragma unroll
        for (int d = 0; d < DT; ++d) o[j][d] *= keep * rescale;
      }
#pragma unroll
      for (int d = 0; d < DT; ++d) {
        const f16x8_t v0 = half8(v[d][0], v[d][1]), v1 = half8(v[d][2], v[d][3]);
#pragma unroll
        for (int j = 0; j < MT; ++j) {
          o[j][d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v0, p[j][0], o[j][d], 0, 0, 0);
          o[j][d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v1, p[j][1], o[j][d], 0, 0, 0);
        }
      }
    }
#pragma unroll
    for (int j = 0; j < MT; ++j) {
      l[j] += __shfl_xor(l[j], 16);
      l[j] += __shfl_xor(l[j], 32);
#pragma unroll
      for (int d = 0; d < DT; ++d) o[j][d] *= unit;
    }
    if (it.whole) {                                            // two by two, the upper ones' state into the lower ones'
#pragma unroll
      for (int half = kWaves / 2; half; half >>= 1) {
        if (wave >= half && wave < 2 * half) {
          float (*to)[64] = s_state[wave - half];
#pragma unroll
          for (int j = 0; j < MT; ++j) {
            to[j * (4 * DT + 2)][lane] = m[j], to[j * (4 * DT + 2) + 1][lane] = l[j];
#pragma unroll
            for (int d = 0; d < 4 * DT; ++d) to[j * (4 * DT + 2) + 2 + d][lane] = o[j][d >> 2][d & 3];
          }
        }
        __syncthreads();
        if (wave < half) {
          float (*from)[64] = s_state[wave];
#pragma unroll
          for (int j = 0; j < MT; ++j) {
            const float om = from[j * (4 * DT + 2)][lane], top = fmaxf(m[j], om), base = top == -INFINITY ? 0.f : top;
            const float mine = __builtin_amdgcn_exp2f(m[j] - base), other = __builtin_amdgcn_exp2f(om - base);
            m[j] = top;
            l[j] = l[j] * mine + from[j * (4 * DT + 2) + 1][lane] * other;
#pragma unroll
            for (int d = 0; d < 4 * DT; ++d) o[j][d >> 2][d & 3] = o[j][d >> 2][d & 3] * mine + from[j * (4 * DT + 2) + 2 + d][lane] * other;
          }
        }
        __syncthreads();
      }
    }
    if (!it.whole || wave == 0) {
      const int slots = a.own.parts + a.prefix.parts;
#pragma unroll
      for (int j = 0; j < MT; ++j) {
        const int row = row_first + 16 * j + r, query = row / a.group, h = it.head * a.group + row - query * a.group;
        if (row >= it.rows) continue;
        if (slots > 1) {
          float* to = a.part + (((long long)(it.first_query + query) * a.heads + h) * slots + it.slot) * (dim + 2);
          if (g == 0) to[dim] = m[j], to[dim + 1] = l[j];
#pragma unroll
          for (int d = 0; d < DT; ++d)
            if (16 * d < dim)
#pragma unroll
              for (int e = 0; e < 4; ++e) to[16 * d + 4 * g + e] = o[j][d][e];
        } else {
          uint16_t* to = a.out + (long long)(it.first_query + query) * a.out_token + h * a.out_head;
          const float inv = l[j] == 0.f ? 0.f : 1.f / l[j];
#pragma unroll
          for (int d = 0; d < DT; ++d)
            if (16 * d < dim) {
              const uint32_t lo = f2bf2(o[j][d][0] * inv, o[j][d][1] * inv), hi = f2bf2(o[j][d][2] * inv, o[j][d][3] * inv);
              uint16_t* at = to + 16 * d + 4 * g;
              if (a.vec_out) *(uint2*)at = make_uint2(lo, hi);
              else at[0] = (uint16_t)lo, at[1] = (uint16_t)(lo >> 16), at[2] = (uint16_t)hi, at[3] = (uint16_t)(hi >> 16);
            }
        }
      }
    }
  }
}

// The pieces of each row put together: a wavefront per row.
__global__ __launch_bounds__(256) void attention_join_kernel(AttentionArgs a) {
  const int row = (int)blockIdx.x * 4 + (int)(threadIdx.x >> 6), lane = threadIdx.x & 63, slots = a.own.parts + a.prefix.parts, dim = a.c.dim;
  if (row >= a.n_queries * a.heads) return;
  const float* from = a.part + (long long)row * slots * (dim + 2);
  float top = -INFINITY;
  for (int s = lane; s < slots; s += 64) top = fmaxf(top, from[s * (dim + 2) + dim]);
#pragma unroll
  for (int x = 32; x; x >>= 1) top = fmaxf(top, __shfl_xor(top, x));
  const float base = top == -INFINITY ? 0.f : top;
  float o[4] = {0.f, 0.f, 0.f, 0.f}, l = 0.f;
  for (int s = 0; s < slots; ++s) {
    const float* p = from + s * (dim + 2);
    const float w = __builtin_amdgcn_exp2f(p[dim] - base);
    l += w * p[dim + 1];
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (lane + 64 * i < dim) o[i] += w * p[lane + 64 * i];
  }
  const float inv = l == 0.f ? 0.f : 1.f / l;
  const int query = row / a.heads, h = row - query * a.heads;
  uint16_t* to = a.out + (long long)query * a.out_token + h * a.out_head;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (lane + 64 * i < dim) to[lane + 64 * i] = f2bf(o[i] * inv);
}

template <int NB>
int attention(const AttentionArgs& a, hipStream_t st) {
  const int grid = (a.prefix.parts * a.prefix.tiles + a.n_seqs * a.own.tiles * a.own.parts) * a.c.heads;
  if (a.row_tiles == 1) attention_kernel<NB, 1><<<grid, 64 * kWaves, 0, st>>>(a);
  else attention_kernel<NB, 2><<<grid, 64 * kWaves, 0, st>>>(a);
  if (attention_slots(a) > 1) attention_join_kernel<<<(a.n_queries * a.heads + 3) / 4, 256, 0, st>>>(a);
  return (int)hipGetLastError();
}

// Pieces of `tokens` keys such that `tiles` row tiles in all make some workgroups per unit, none shorter than two steps of a workgroup.
void share_out(AttentionShare& s, long long rows, int row_tiles, long long times, long long tokens) {
  s.whole = rows <= 16 * row_tiles;
  s.tiles = (int)std::max(1ll, (rows + 16 * row_tiles * (s.whole ? 1 : kWaves) - 1) / (16 * row_tiles * (s.whole ? 1 : kWaves)));
  const long long want = std::max(1ll, 1024 / std::max(1ll, s.tiles * times)), step = kKeys * (s.whole ? kWaves : 1);
  const long long most = std::max(1ll, std::min(64ll, tokens / (2 * step)));
  const long long parts = std::min(want, most);
  s.part_len = (int)(std::max(1ll, (tokens + parts * step - 1) / (parts * step)) * step);
  s.parts = (int)std::max(1ll, (tokens + s.part_len - 1) / s.part_len);
}

}  // namespace

void attention_split(AttentionArgs& a, int max_queries, int max_length) {
  const long long own = (long long)max_queries * a.group, all = (long long)a.n_queries * a.group;
  a.row_tiles = own <= 16 && (a.prefix_len == 0 || all <= 16) ? 1 : 2;
  share_out(a.own, own, a.row_tiles, (long long)std::max(1, a.n_seqs) * a.c.heads, max_length);
  if (a.prefix_len > 0) share_out(a.prefix, all, a.row_tiles, a.c.heads, a.prefix_len);
  else a.prefix = AttentionShare{1, 0, kKeys, 1};
}

int launch_attention(const AttentionArgs& a, void* stream) {
  hipStream_t st = (hipStream_t)stream;
  switch ((a.c.dim + 63) / 64) {
    case 1: return attention<1>(a, st);
    case 2: return attention<2>(a, st);
    case 3: return attention<3>(a, st);
    default: return attention<4>(a, st);
  }
}

}  // namespace xenos
