// Attention of a batch of sequences to the quantised cache, with a prefix they share.
//
// Keys pass once, 64 at a time, with a running reference and sum of a softmax per row.  The scores are computed transposed, S^T = K Q^T, so that a lane ends up with
// 16 neighbouring keys of one row (tile t of a wavefront's four takes key 16 (r / 4) + 4 t + r % 4 as its row r): the maximum is over registers and two exchanges, and the lane's
// probabilities are, as they lie, the operand of O^T += V^T P^T, whose other operand is what the cache holds for one dimension: 16 keys side by side.
// With few rows keys and values go from memory to registers as they are, and only the scales round through LDS; with many the wavefronts share both there.  The 8-bit keys become bf16 and the values fp16 without rounding; the keys' scales multiply the scores, the values' the probabilities.
// Those weights are rounded to fp16 for the product, relative to the row's largest (kHead): eight times as fine as bf16, whose error would be as large as that of the
// rounding of the result (relative error of the output against 64 bits: 1.7e-3 in place of 2.4e-3), and in range whatever the scales are.  Nothing else is rounded on the way.
#include <algorithm>
#include <math.h>
#include "token_device.h"

namespace xenos {

namespace {

constexpr int kKeys = 64;                                     // of a step
constexpr int kWaves = 4, kMostParts = 64;                    // of a workgroup, of a segment

// Eight bytes as bf16: whole numbers up to 127, exact.  One conversion a byte (the compiler makes two instructions of the cast) and one a pair.
template <int B>
__device__ __forceinline__ float byte_of(uint32_t v) {
  float r;
  if constexpr (B == 0) asm("v_cvt_f32_i32_sdwa %0, sext(%1) dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:BYTE_0" : "=v"(r) : "v"(v));
  else if constexpr (B == 1) asm("v_cvt_f32_i32_sdwa %0, sext(%1) dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:BYTE_1" : "=v"(r) : "v"(v));
  else if constexpr (B == 2) asm("v_cvt_f32_i32_sdwa %0, sext(%1) dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:BYTE_2" : "=v"(r) : "v"(v));
  else asm("v_cvt_f32_i32_sdwa %0, sext(%1) dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:BYTE_3" : "=v"(r) : "v"(v));
  return r;
}
__device__ __forceinline__ bf16x8_t whole8(uint32_t lo, uint32_t hi) {
  return __builtin_bit_cast(bf16x8_t, (u32x4_t){f2bf2(byte_of<0>(lo), byte_of<1>(lo)), f2bf2(byte_of<2>(lo), byte_of<3>(lo)),
                                               f2bf2(byte_of<0>(hi), byte_of<1>(hi)), f2bf2(byte_of<2>(hi), byte_of<3>(hi))});
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
  int tokens;                                                 // of the segment that its table holds
  int length;                                                 // of a sequence: its last query sees the tokens up to this one
  int seq, tile;
  int first_query, queries;
  int row0, rows;                                             // first row of the tile; rows of the item in all (queries times the group)
  int begin, end;                                             // keys
  int slot;
  bool prefix;
};

// The workgroup's item of a launch; its row tiles have tile_rows rows.  Heads change fastest (an XCD then reads the keys of few of them), and the last rows, which see
// the most keys, come first.
__device__ __forceinline__ Item item_of(const AttentionArgs& a, int at, int tile_rows) {
  Item it;
  const int front = a.skip_prefix ? 0 : a.prefix.parts * a.prefix.tiles * a.c.heads;
  it.prefix = at < front;
  const AttentionShare& s = it.prefix ? a.prefix : a.own;
  if (!it.prefix) at -= front;
  it.head = at % a.c.heads;
  at /= a.c.heads;
  const int tile = s.tiles - 1 - at % s.tiles;
  at /= s.tiles;
  const int part = at % s.parts, seq = at / s.parts;
  it.seq = seq, it.tile = tile;
  if (it.prefix) {
    it.table = a.prefix_table, it.tokens = it.length = a.prefix_len, it.first_query = 0, it.queries = a.n_queries, it.slot = part;
  } else {
    const int held = a.table_stride * a.c.page, n = max(a.lengths[seq], 0);   // (held: at most 2^30)
    it.table = a.tables + (long long)seq * a.table_stride;
    it.length = n, it.tokens = min(n, held);
    const int lo = a.starts ? a.starts[seq] : seq, hi = a.starts ? a.starts[seq + 1] : seq + 1;
    it.first_query = lo < 0 ? 0 : lo < a.n_queries ? lo : a.n_queries;
    it.queries = hi <= it.first_query ? 0 : (hi < a.n_queries ? hi : a.n_queries) - it.first_query;
    it.slot = a.prefix.parts + part;
  }
  if (a.c.n_pages == 0) it.tokens = 0;
  it.rows = it.queries * a.group;
  it.row0 = tile * tile_rows;
  it.begin = part * s.part_len;
  it.end = part == s.parts - 1 || it.begin + s.part_len > it.tokens ? it.tokens : it.begin + s.part_len;
  return it;
}

// The keys of a segment that a query sees, from its first one on.
__device__ __forceinline__ int seen_by(const Item& it, int query) { return it.prefix ? it.tokens : min(it.tokens, it.length - it.queries + query + 1); }

// The rows of q that no sequence has, before the first one's and behind the last one's, see no keys of their own.  Where there are no pieces to be joined nobody else writes their
// results: the first tile of the first sequence, and of the last one, does.
__device__ __forceinline__ void blank_rows(const AttentionArgs& a, const Item& it) {
  if (it.prefix || it.tile || !a.starts || a.own.parts + a.prefix.parts > 1) return;
  const int width = a.group * a.c.dim;
  const auto blank = [&](int from, int to) {
    for (long long i = (long long)from * width + threadIdx.x; i < (long long)to * width; i += 64 * kWaves) {
      const int query = (int)(i / width), at = (int)(i - (long long)query * width), h = at / a.c.dim;
      a.out[query * a.out_token + (it.head * a.group + h) * a.out_head + at - h * a.c.dim] = 0;
    }
  };
  if (it.seq == 0) blank(0, it.first_query);
  if (it.seq == a.n_seqs - 1) blank(it.first_query + it.queries, a.n_queries);
}

// Eight values of a query, infinities as NaN: each of its scores is an infinity or a NaN, and their softmax no number; scores that all are -infinity would look like keys that
// are not seen.
__device__ __forceinline__ bf16x8_t query8(u32x4_t w) {
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    if ((w[e] & 0x7fffu) == 0x7f80u) w[e] |= 0x40u;
    if ((w[e] & 0x7fff0000u) == 0x7f800000u) w[e] |= 0x400000u;
  }
  return __builtin_bit_cast(bf16x8_t, w);
}

// Where a block of 16 keys of a segment lies: its first row among the cache's, if it has a page.
struct Block16 {
  long long row;
  bool ok;
  __device__ __forceinline__ Block16(const AttentionArgs& a, const Item& it, int key, int page) {
    ok = key < it.tokens && (unsigned)page < (unsigned)a.c.n_pages;
    row = ok ? ((long long)page * a.c.heads + it.head) * a.c.page + key % a.c.page : 0;
  }
};

// A key's weight is its probability times its value's scale, and is rounded to fp16, in steps of 2^-24 at the least; so each row counts weights, and the probabilities' sum l with
// them, in 2^ref of its own: ref is log2 of the largest weight that the row has seen less kHead, and follows only when a weight passes 2^kSlack (the exchange of maxima and the
// rescaling of O are then rare).  What a row may not see, or hardly looks at, takes no bits from it, however large its value.
// A scale counts as 2^-88 at the least here: rows of zeros, whose scale is 2^-107, then leave l at 2^15 2^88 a key, in range, and a weight of 2^-107 still has fp16's 11 bits.
constexpr float kHead = 7.f, kSlack = 15.f, kLeastScale = 0x1p-88f;
// log2 of a scale (of v_log_f32's error, some 2^-22, a weight's range is the only thing that depends on it)
__device__ __forceinline__ float size_of_scale(float s) { return __builtin_amdgcn_logf(fmaxf(fabsf(s), kLeastScale)); }

// Few rows: the wavefronts of a workgroup have the same 16 rows and take turns with the keys; their states meet in LDS at the end.  NB: blocks of 64 dimensions.
// Bound by the cache's bytes: 16 sequences of 100 to 32768 tokens, 8 heads of 128, 32 of queries: 506 MB in 100 to 112 us, 4.5 to 5 TB/s; all of 32768: 1.1 GB in 206, 5.4 TB/s.
template <int NB>
__global__ __launch_bounds__(64 * kWaves, NB <= 2 ? 4 - NB : 1) void attention_kernel(AttentionArgs a) {
  constexpr int DT = 4 * NB, REC = 4 * DT + 2;              // tiles of 16 dimensions; floats of a lane's state
  __shared__ float s_state[kWaves / 2][REC][64];
  __shared__ __attribute__((aligned(16))) float s_scale[kWaves][3][kKeys];
  Item it = item_of(a, (int)blockIdx.x, 16);
  blank_rows(a, it);
  const int step_rows = (it.prefix ? a.prefix : a.own).tiles * 16;
  for (; it.row0 < it.rows; it.row0 += step_rows) {           // (once, unless a sequence has more queries than was said)
    int lane = threadIdx.x & 63, dim = a.c.dim;
    asm volatile("" : "+v"(lane), "+s"(dim));                 // (nothing is made before this loop, and kept in registers through it)
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, g = lane >> 4;
    // rows of this lane: queries in bf16, and the keys they see
    bf16x8_t q[NB][2];
    int limit, most;
    {
      const int row = it.row0 + r, query = row / a.group, h = it.head * a.group + row - query * a.group;
      const bool ok = row < it.rows;
      limit = ok ? seen_by(it, query) : 0;
      most = limit;
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
          q[b][half] = query8(w);
        }
    }
#pragma unroll
    for (int o = 1; o < 16; o <<= 1) most = max(most, __shfl_xor(most, o));
    const int end = min(it.end, most);

    f32x4_t o[DT];
    float ref = -INFINITY, l = 0.f;                           // (o and l count in 2^ref)
#pragma unroll
    for (int d = 0; d < DT; ++d) o[d] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    // The blocks of 16 keys that this lane reads: of keys (for the scores' rows), of values, and of its own key's scales.  Their pages are looked up a step ahead, the keys are
    // asked for while the scores are turned into probabilities, the values while the scores are made.
    int page_k, page_v, page_s;
    const auto page_of = [&](int key) { return it.table[min(key, it.tokens - 1) / a.c.page]; };
    const auto look_up = [&](int key) { page_k = page_of(key + 16 * (r >> 2)), page_v = page_of(key + 16 * g), page_s = page_of(key + lane / 16 * 16); };
    u32x4_t k[4][NB], v[DT];
    const auto request_keys = [&](int key) {
      const Block16 at(a, it, key + 16 * (r >> 2), page_k);
      const int8_t* from = a.c.k + (at.row + (r & 3)) * dim + 16 * g;
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int t = 0; t < 4; ++t) k[t][b] = *(const u32x4_t*)(from + 4 * t * dim + (64 * b + 16 * g < dim ? 64 * b : -16 * g));
    };
    constexpr int STEP = kWaves * kKeys;
    int key = it.begin + wave * kKeys;
    if (key < end) look_up(key), request_keys(key);
    for (; key < end; key += STEP) {
      const Block16 at(a, it, key + 16 * g, page_v), as(a, it, key + lane / 16 * 16, page_s);
      float scale_k = a.c.k_scale[as.row + lane % 16], scale_v = a.c.v_scale[as.row + lane % 16];
      const int8_t* from = a.c.v + at.row * dim + r * 16;
#pragma unroll
      for (int d = 0; d < DT; ++d) v[d] = *(const u32x4_t*)(from + (16 * d < dim ? 256 * d : 0));
      look_up(key + STEP);
      __builtin_amdgcn_sched_barrier(0);
      f32x4_t s[4];
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        s[t] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
          for (int half = 0; half < 2; ++half) {
            const bf16x8_t kk = whole8(k[t][b][2 * half], k[t][b][2 * half + 1]);
            s[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kk, q[b][half], s[t], 0, 0, 0);
          }
      }
      __builtin_amdgcn_sched_barrier(0);
      request_keys(key + STEP);
      __builtin_amdgcn_sched_barrier(0);
      // the scales of the step's keys, one a lane, go round through LDS
      // (a value scale that is no number makes the score one that is none, for the rows that see it; the others multiply it by a probability of 0)
      const float known = fabsf(scale_v) < INFINITY ? scale_v : 0.f;
      s_scale[wave][0][lane] = fabsf(scale_v) < INFINITY ? scale_k * a.scale2 : __builtin_nanf("");
      s_scale[wave][1][lane] = known;
      s_scale[wave][2][lane] = size_of_scale(known);
      f16x8_t p[2];
      const int seen = at.ok ? limit - key - 16 * g : 0;      // of this lane's 16 keys
      float top = -INFINITY;
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        const f32x4_t ks = *(const f32x4_t*)&s_scale[wave][0][16 * g + 4 * t], size = *(const f32x4_t*)&s_scale[wave][2][16 * g + 4 * t];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          s[t][e] = 4 * t + e < seen ? s[t][e] * ks[e] : -INFINITY;
          top = fmaxf(top, s[t][e] + size[e]);
        }
      }
      float keep = 1.f;
      if (__any(top > ref + kSlack)) {
        top = fmaxf(top, __shfl_xor(top, 16));
        top = fmaxf(top, __shfl_xor(top, 32));
        if (top > ref + kSlack) {
          keep = __builtin_amdgcn_exp2f(ref - (top - kHead));
          ref = top - kHead;
          l *= keep;
        }
      }
      const float base = ref == -INFINITY ? 0.f : ref;
      float sum = 0.f;
      u32x4_t w[2];
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        const f32x4_t vs = *(const f32x4_t*)&s_scale[wave][1][16 * g + 4 * t];
        float pv[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float x = __builtin_amdgcn_exp2f(s[t][e] - base);
          sum += x;
          pv[e] = x * vs[e];
        }
        w[t >> 1][2 * (t & 1)] = f2h2(pv[0], pv[1]);
        w[t >> 1][2 * (t & 1) + 1] = f2h2(pv[2], pv[3]);
      }
      p[0] = __builtin_bit_cast(f16x8_t, w[0]), p[1] = __builtin_bit_cast(f16x8_t, w[1]);
      l += sum;
      if (__any(keep != 1.f)) {
#pragma unroll
        for (int d = 0; d < DT; ++d) o[d] *= keep;
      }
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int d = 0; d < DT; ++d) {
        const f16x8_t v0 = half8(v[d][0], v[d][1]), v1 = half8(v[d][2], v[d][3]);
        o[d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v0, p[0], o[d], 0, 0, 0);
        o[d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v1, p[1], o[d], 0, 0, 0);
      }
    }
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
    // the states two by two, the upper ones' into the lower ones'
#pragma unroll
    for (int half = kWaves / 2; half; half >>= 1) {
      if (wave >= half && wave < 2 * half) {
        float (*to)[64] = s_state[wave - half];
        to[0][lane] = ref, to[1][lane] = l;
#pragma unroll
        for (int d = 0; d < 4 * DT; ++d) to[2 + d][lane] = o[d >> 2][d & 3];
      }
      __syncthreads();
      if (wave < half) {
        float (*from)[64] = s_state[wave];
        const float theirs = from[0][lane], top = fmaxf(ref, theirs), base = top == -INFINITY ? 0.f : top;
        const float mine = __builtin_amdgcn_exp2f(ref - base), other = __builtin_amdgcn_exp2f(theirs - base);
        ref = top;
        l = l * mine + from[1][lane] * other;
#pragma unroll
        for (int d = 0; d < 4 * DT; ++d) o[d >> 2][d & 3] = o[d >> 2][d & 3] * mine + from[2 + d][lane] * other;
      }
      __syncthreads();
    }
    if (wave == 0) {
      const int slots = a.own.parts + a.prefix.parts;
      const int row = it.row0 + r, query = row / a.group, h = it.head * a.group + row - query * a.group;
      if (row >= it.rows) continue;
      if (slots > 1) {
        const long long at = ((long long)(it.first_query + query) * a.heads + h) * slots + it.slot;
        if (g == 0) *(float2*)(a.part_ml + 2 * at) = make_float2(ref, l);
        if (ref == -INFINITY && l == 0.f) continue;          // (nothing seen: its sums are not looked at)
#pragma unroll
        for (int d = 0; d < DT; ++d)
          if (16 * d < dim) *(f32x4_t*)(a.part + at * dim + 16 * d + 4 * g) = o[d];
      } else {
        uint16_t* to = a.out + (long long)(it.first_query + query) * a.out_token + h * a.out_head;
        const float inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
        for (int d = 0; d < DT; ++d)
          if (16 * d < dim) {
            const uint32_t lo = f2bf2(o[d][0] * inv, o[d][1] * inv), hi = f2bf2(o[d][2] * inv, o[d][3] * inv);
            uint16_t* at = to + 16 * d + 4 * g;
            if (a.vec_out) *(uint2*)at = make_uint2(lo, hi);
            else at[0] = (uint16_t)lo, at[1] = (uint16_t)(lo >> 16), at[2] = (uint16_t)hi, at[3] = (uint16_t)(hi >> 16);
          }
      }
    }
  }
}

// Many rows: the four wavefronts of a workgroup have 32 rows each and pass over the same keys, which the workgroup turns into bf16 and fp16 once, in LDS, while the steps before
// them are multiplied.  S^T = K Q^T in blocks of 32 keys x 32 rows, whose row 8 a + 4 h + b is key 16 (a / 2) + 8 h + 4 (a % 2) + b: a lane of half h then holds eight
// neighbouring keys at a time, an operand of O^T += V^T P^T as it is.
// Bound by the vector instructions beside the products (the softmax's, a dozen a score, and the conversions): a prompt of 4097, 20 heads of 128 on 4: 86 GFLOP in 144 to 168 us, 510 to 600 TFLOP/s;
// 512 rows to 16384 shared keys on 4 heads of 128: 17 GFLOP in 39 us.
// Whether a weight may pass 2^kSlack is judged by the largest scale of a step, whoever sees it; only if it may are the scales of the keys that a row sees looked at one by one.
template <int NB>
__global__ __launch_bounds__(64 * kWaves, NB <= 2 ? 2 : 1) void attention_tile_kernel(AttentionArgs a) {
  constexpr int DT = 2 * NB, KP = 128 * NB + 16, VP = 2 * kKeys + 16, KB = kKeys * KP, VB = 64 * NB * VP, CH = 4 * NB;   // pitches (odd numbers of 16-byte places), buffers in bytes
  extern __shared__ __attribute__((aligned(16))) unsigned char s_kv[];
  float (*s_ks)[kKeys] = (float (*)[kKeys])(s_kv + 2 * (KB + VB));
  int* s_ok = (int*)(s_ks + 2);
  float (*s_vs)[kKeys] = (float (*)[kKeys])(s_ok + 4);
  Item it = item_of(a, (int)blockIdx.x, 32 * kWaves);
  blank_rows(a, it);
  const int step_rows = (it.prefix ? a.prefix : a.own).tiles * 32 * kWaves;
  for (; it.row0 < it.rows; it.row0 += step_rows) {           // (once, unless a sequence has more queries than was said)
    int lane = threadIdx.x & 63, dim = a.c.dim;
    asm volatile("" : "+v"(lane), "+s"(dim));                 // (nothing is made before this loop, and kept in registers through it)
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 31, half = lane >> 5, thread = 64 * wave + lane;
    const int row = it.row0 + wave * 32 + r, query = row / a.group, h = it.head * a.group + row - query * a.group;
    const bool have = row < it.rows;
    const int limit = have ? seen_by(it, query) : 0;
    // keys that the workgroup, and the wavefront, look at; up to `least` none is hidden from any row
    int most = limit, least = have ? limit : 0x7fffffff;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) most = max(most, __shfl_xor(most, o)), least = min(least, __shfl_xor(least, o));
    most = __builtin_amdgcn_readfirstlane(most), least = __builtin_amdgcn_readfirstlane(least);
    int last = it.row0 + 32 * kWaves < it.rows ? it.row0 + 32 * kWaves - 1 : it.rows - 1;
    const int end = min(it.end, seen_by(it, last / a.group));
    bf16x8_t q[2 * DT];
    {
      const uint16_t* src = a.q + (have ? (long long)(it.first_query + query) * a.q_token + h * a.q_head : 0);
#pragma unroll
      for (int s = 0; s < 2 * DT; ++s) {
        const int d = 16 * s + 8 * half;
        u32x4_t w = {0, 0, 0, 0};
        if (have && d < dim) {
          if (a.vec_q) w = *(const u32x4_t*)(src + d);
          else {
#pragma unroll
            for (int e = 0; e < 8; ++e) w[e >> 1] |= (uint32_t)src[d + e] << (16 * (e & 1));
          }
        }
        q[s] = query8(w);
      }
    }
    f32x16_t o[DT];
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
      for (int e = 0; e < 16; ++e) o[d][e] = 0.f;
    float ref = -INFINITY, l = 0.f;                           // (o and l count in 2^ref)
    float most_scale = kLeastScale, room = 0.f;               // no value of the step has a larger scale; exponents up to which no weight of it passes 2^kSlack

    // ---- a step's keys and values on their way: 16 bytes of a key (chunk c of key j), 16 keys of a dimension, the scales of key `lane`
    const int vr = lane & 15, vg = lane >> 4;
    int next_page = 0;
    u32x4_t raw_k[NB], raw_v[NB];
    float scale_k = 0.f, scale_v = 0.f;
    int raw_key = 0;
    bool raw_ok = false;
    const AnyDiv per_page(a.c.page);
    const auto look_up = [&](int key) { next_page = it.table[per_page(min(key + 16 * vg, it.tokens - 1))]; };   // of this lane's block of 16 keys
    const auto request = [&](int key) {
      const int first = key + 16 * vg;
      raw_key = key;
      raw_ok = first < it.tokens && (unsigned)next_page < (unsigned)a.c.n_pages;
      const long long row = raw_ok ? ((long long)next_page * a.c.heads + it.head) * a.c.page + (first - per_page(first) * a.c.page) : 0;
#pragma unroll
      for (int i = 0; i < NB; ++i) {
        const int id = thread + 256 * i, j = id / CH, c = id - j * CH;
        const long long at = (long long)(uint32_t)__shfl((int)row, j & 48) | (long long)__shfl((int)(row >> 32), j & 48) << 32;
        raw_k[i] = *(const u32x4_t*)(a.c.k + (at + j % 16) * dim + (16 * c < dim ? 16 * c : 0));   // (what lies behind dim meets zeros of q)
      }
      const int8_t* v = a.c.v + row * dim + vr * 16;
#pragma unroll
      for (int i = 0; i < NB; ++i) raw_v[i] = *(const u32x4_t*)(v + (16 * (wave * NB + i) < dim ? 256 * (wave * NB + i) : 0));
      scale_k = a.c.k_scale[row + vr], scale_v = a.c.v_scale[row + vr];
    };
    // they become operands in buffer b
    const auto store = [&](int b) {
      unsigned char *k = s_kv + b * (KB + VB), *v = k + KB;
#pragma unroll
      for (int i = 0; i < NB; ++i) {
        const int id = thread + 256 * i, j = id / CH, c = id - j * CH;
        *(bf16x8_t*)(k + j * KP + 32 * c) = whole8(raw_k[i][0], raw_k[i][1]);
        *(bf16x8_t*)(k + j * KP + 32 * c + 16) = whole8(raw_k[i][2], raw_k[i][3]);
      }
      // (a value scale that is no number makes the score one that is none: for the rows that see it; the others multiply it by a probability of 0)
      const bool number = fabsf(scale_v) < INFINITY;
      const float size = raw_ok && raw_key + lane < it.tokens && number ? fabsf(scale_v) : 0.f;
      if (__any(size > most_scale)) {                         // (the same for every wavefront)
        most_scale = size;
#pragma unroll
        for (int x = 32; x; x >>= 1) most_scale = fmaxf(most_scale, __shfl_xor(most_scale, x));
      } else if (!__any(size > most_scale * 0.0625f)) most_scale = fmaxf(most_scale * 0.0625f, kLeastScale);
      room = kSlack - size_of_scale(most_scale);
#pragma unroll
      for (int i = 0; i < NB; ++i)
#pragma unroll
        for (int p = 0; p < 2; ++p) *(f16x8_t*)(v + (16 * (wave * NB + i) + vr) * VP + 32 * vg + 16 * p) = half8(raw_v[i][2 * p], raw_v[i][2 * p + 1]);
      if (wave == 0) {
        s_ks[b][lane] = number ? scale_k * a.scale2 : __builtin_nanf("");
        s_vs[b][lane] = number ? scale_v : 0.f;
        const uint64_t there = __ballot(raw_ok && vr == 0);
        if (lane == 0) s_ok[b] = (int)((there & 1) | (there >> 15 & 2) | (there >> 30 & 4) | (there >> 45 & 8));
      }
    };

    __syncthreads();
    if (it.begin < end) {
      look_up(it.begin);
      request(it.begin);
      store(0);
      look_up(it.begin + kKeys);
      request(it.begin + kKeys);
    }
    int b = 0;
    for (int key = it.begin; key < end; key += kKeys, b ^= 1) {
      __syncthreads();
      look_up(key + 2 * kKeys);
      if (key < most) {
        const unsigned char *k = s_kv + b * (KB + VB), *v = k + KB;
        f32x16_t s[2];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
#pragma unroll
          for (int e = 0; e < 16; ++e) s[t][e] = 0.f;
          const int j = 32 * t + 16 * (r >> 4) + 8 * (r >> 2 & 1) + 4 * (r >> 3 & 1) + (r & 3);
#pragma unroll
          for (int i = 0; i < 2 * DT; ++i) {
            s[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(*(const bf16x8_t*)(k + j * KP + 32 * i + 16 * half), q[i], s[t], 0, 0, 0);
            if (i % 4 == 3) __builtin_amdgcn_sched_barrier(0);   // (else the operands of all products are read at once, and registers spill)
          }
        }
        // exponents relative to ref (to 0 before a first weight), in place of the scores
        const int ok = s_ok[b];
        const bool open = key + kKeys <= least && __builtin_amdgcn_readfirstlane(ok) == 15;
        const float base = ref == -INFINITY ? 0.f : ref;
        float top = -INFINITY;
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int x = 0; x < 4; ++x) {
            const f32x4_t ks = *(const f32x4_t*)&s_ks[b][32 * t + 16 * (x >> 1) + 8 * half + 4 * (x & 1)];
#pragma unroll
            for (int e = 0; e < 4; ++e) s[t][4 * x + e] = __builtin_fmaf(s[t][4 * x + e], ks[e], -base);
          }
        if (!open) {
          asm volatile("");                                   // (a branch: as selections of every element this is a tenth of a step)
#pragma unroll
          for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int e = 0; e < 16; ++e) {
              const int j = 32 * t + 16 * (e >> 3) + 8 * half + 4 * (e >> 2 & 1) + (e & 3);
              if (!(key + j < limit && (ok >> (2 * t + (e >> 3)) & 1))) s[t][e] = -INFINITY;
            }
        }
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int e = 0; e < 16; e += 2) top = fmaxf(fmaxf(top, s[t][e]), s[t][e + 1]);
        if (__any(top > (ref == -INFINITY ? -INFINITY : room))) {   // (a weight may pass: with the scales of the keys that each row sees)
          top = -INFINITY;
#pragma unroll
          for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int x = 0; x < 4; ++x) {
              const f32x4_t vs = *(const f32x4_t*)&s_vs[b][32 * t + 16 * (x >> 1) + 8 * half + 4 * (x & 1)];
#pragma unroll
              for (int e = 0; e < 4; ++e) top = fmaxf(top, s[t][4 * x + e] + size_of_scale(vs[e]));
            }
          top = fmaxf(top, __shfl_xor(top, 32));
          const bool passes = top > (ref == -INFINITY ? -INFINITY : kSlack);
          if (__any(passes)) {
            const float up = passes ? top - kHead : 0.f, keep = !passes ? 1.f : ref == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(-up);
            if (passes) ref = base + up;
            l *= keep;
#pragma unroll
            for (int d = 0; d < DT; ++d) o[d] *= keep;
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
              for (int e = 0; e < 16; ++e) s[t][e] -= up;
          }
        }
        float sum = 0.f;
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          u32x4_t w[2];
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const float p0 = __builtin_amdgcn_exp2f(s[t][2 * e]), p1 = __builtin_amdgcn_exp2f(s[t][2 * e + 1]);
            const float2 vs = *(const float2*)&s_vs[b][32 * t + 16 * (e >> 2) + 8 * half + 2 * (e & 3)];
            sum += p0 + p1;
            w[e >> 2][e & 3] = f2h2(p0 * vs.x, p1 * vs.y);
          }
#pragma unroll
          for (int c = 0; c < 2; ++c) {
#pragma unroll
            for (int d = 0; d < DT; ++d)
              o[d] = __builtin_amdgcn_mfma_f32_32x32x16_f16(*(const f16x8_t*)(v + (32 * d + r) * VP + 64 * t + 32 * c + 16 * half), __builtin_bit_cast(f16x8_t, w[c]), o[d], 0, 0, 0);
            __builtin_amdgcn_sched_barrier(0);
          }
        }
        l += sum;
      }
      if (key + kKeys < end) {
        store(b ^ 1);
        request(key + 2 * kKeys);
      }
    }
    l += __shfl_xor(l, 32);
    if (have) {
      const int slots = a.own.parts + a.prefix.parts;
      if (slots > 1) {
        const long long at = ((long long)(it.first_query + query) * a.heads + h) * slots + it.slot;
        if (half == 0) *(float2*)(a.part_ml + 2 * at) = make_float2(ref, l);
        if (ref != -INFINITY || l != 0.f) {                     // (nothing seen: its sums are not looked at)
#pragma unroll
          for (int d = 0; d < DT; ++d)
#pragma unroll
            for (int x = 0; x < 4; ++x)
              if (32 * d + 8 * x < dim)
                *(f32x4_t*)(a.part + at * dim + 32 * d + 8 * x + 4 * half) = f32x4_t{o[d][4 * x], o[d][4 * x + 1], o[d][4 * x + 2], o[d][4 * x + 3]};
        }
      } else {
        uint16_t* to = a.out + (long long)(it.first_query + query) * a.out_token + h * a.out_head;
        const float inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
          for (int x = 0; x < 4; ++x)
            if (32 * d + 8 * x < dim) {
              const uint32_t lo = f2bf2(o[d][4 * x] * inv, o[d][4 * x + 1] * inv), hi = f2bf2(o[d][4 * x + 2] * inv, o[d][4 * x + 3] * inv);
              uint16_t* at = to + 32 * d + 8 * x + 4 * half;
              if (a.vec_out) *(uint2*)at = make_uint2(lo, hi);
              else at[0] = (uint16_t)lo, at[1] = (uint16_t)(lo >> 16), at[2] = (uint16_t)hi, at[3] = (uint16_t)(hi >> 16);
            }
      }
    }
  }
}

// The pieces of a row put together by a workgroup: every wavefront weighs them all, then groups of dim / 4 lanes add four dimensions each of several pieces at a time.
// Bound by their bytes: 2048 rows of 128 in 33 pieces: 35 MB in 8.5 us, 4.1 TB/s.
__global__ __launch_bounds__(256) void attention_join_kernel(AttentionArgs a) {
  __shared__ float s_w[2 * kMostParts];
  __shared__ f32x4_t s_o[256];
  const int row = (int)blockIdx.x, lane = threadIdx.x & 63, all = a.own.parts + a.prefix.parts, dim = a.c.dim, lanes = dim / 4, groups = 256 / lanes;
  const float2* ml = (const float2*)a.part_ml + (long long)row * all;
  const int query = row / a.heads, h = row - query * a.heads;
  // (a row that no sequence has: its pieces are the prefix's, which come first; nobody wrote others)
  const int slots = !a.starts || (query >= a.starts[0] && query < a.starts[a.n_seqs]) ? all : a.prefix.parts;
  float m[2], l[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int s = lane + 64 * i;
    const float2 v = s < slots ? ml[s] : make_float2(-INFINITY, 0.f);
    m[i] = v.x, l[i] = v.y;
  }
  float top = fmaxf(m[0], m[1]);
#pragma unroll
  for (int x = 32; x; x >>= 1) top = fmaxf(top, __shfl_xor(top, x));
  const float base = top == -INFINITY ? 0.f : top;
  float total = 0.f;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const bool seen = m[i] != -INFINITY || l[i] != 0.f;       // (l alone: a row that saw what is no number)
    const float w = seen ? __builtin_amdgcn_exp2f(m[i] - base) : 0.f;
    if (threadIdx.x < 64 && lane + 64 * i < slots) s_w[lane + 64 * i] = seen && m[i] == -INFINITY ? l[i] : w;
    total += seen && m[i] == -INFINITY ? l[i] : w * l[i];
  }
  total = wave_sum(total);
  __syncthreads();
  const int group = (int)threadIdx.x / lanes, d = ((int)threadIdx.x - group * lanes) * 4;
  f32x4_t o = {0.f, 0.f, 0.f, 0.f};
  const float* from = a.part + (long long)row * all * dim + d;
  if (group < groups)
    for (int s0 = group; s0 < slots; s0 += 4 * groups) {
      float w[4];
      f32x4_t v[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int s = s0 + u * groups;
        w[u] = s < slots ? s_w[s] : 0.f;
        v[u] = w[u] != 0.f ? *(const f32x4_t*)(from + (long long)s * dim) : f32x4_t{0.f, 0.f, 0.f, 0.f};
      }
#pragma unroll
      for (int u = 0; u < 4; ++u) o += w[u] * v[u];
    }
  s_o[threadIdx.x] = o;
  __syncthreads();
  if ((int)threadIdx.x >= lanes) return;
  for (int g = 1; g < groups; ++g) o += s_o[threadIdx.x + g * lanes];
  const float inv = total == 0.f ? 0.f : 1.f / total;
  uint16_t* to = a.out + (long long)query * a.out_token + h * a.out_head + d;
  const uint32_t lo = f2bf2(o[0] * inv, o[1] * inv), hi = f2bf2(o[2] * inv, o[3] * inv);
  if (a.vec_out) *(uint2*)to = make_uint2(lo, hi);
  else to[0] = (uint16_t)lo, to[1] = (uint16_t)(lo >> 16), to[2] = (uint16_t)hi, to[3] = (uint16_t)(hi >> 16);
}

// One launch over the segments whose kernel is the same.
template <int NB>
int attention_rows(const AttentionArgs& a, bool many, int grid, hipStream_t st) {
  if (!many) attention_kernel<NB><<<grid, 64 * kWaves, 0, st>>>(a);
  else {
    static PerDevice raised;
    const hipError_t e = raise_lds_limit(attention_tile_kernel<NB>, raised);
    if (e != hipSuccess) return (int)e;
    constexpr int lds = 2 * (kKeys * (128 * NB + 16) + 64 * NB * (2 * kKeys + 16) + 4 * kKeys) + 16 + kWaves * 2 * kKeys;
    attention_tile_kernel<NB><<<grid, 64 * kWaves, lds, st>>>(a);
  }
  return (int)hipGetLastError();
}
template <int NB>
int attention(AttentionArgs a, hipStream_t st) {
  const int front = a.prefix.parts * a.prefix.tiles * a.c.heads, own = a.n_seqs * a.own.tiles * a.own.parts * a.c.heads;
  if (front && a.prefix.many == a.own.many) {
    if (const int e = attention_rows<NB>(a, a.own.many, front + own, st)) return e;
  } else {
    if (front)
      if (const int e = attention_rows<NB>(a, a.prefix.many, front, st)) return e;
    a.skip_prefix = 1;
    if (const int e = attention_rows<NB>(a, a.own.many, own, st)) return e;
  }
  if (attention_slots(a) > 1) attention_join_kernel<<<a.n_queries * a.heads, 256, 0, st>>>(a);
  return (int)hipGetLastError();
}

// Which kernel a segment has.  More than 32 rows, and rows x keys x dimensions of 1.6e9 at the least: many rows; below, its few workgroups and its way into LDS cost more than it saves.
// us for 16 rows a workgroup, for many rows (8 heads of 128, keys x sequences x rows): 8192 x 1 x 128: 33, 36; 5869 x 1 x 128 (dim 64): 17, 21; 8192 x 4 x 64: 54, 39; 8192 x 1 x 512: 79,
// 49; 2048 x 8 x 1024: 176, 99; 4 heads, 4097 x 1 x 20485, each row up to its own: 264, 147.
// The keys are cut in pieces until there are `want` workgroups, none shorter than two steps of every wavefront that takes turns with it: 16 rows, heads up to 128, 2048 (16 sequences of 100 to
// 32768 tokens, 8 heads of 128: in 512 140 us, in 2048 122; where all have 32768, 203 and 210); longer heads, of which a unit holds a workgroup or two, and many rows: 512 (32 sequences of 4042,
// 16 heads of 256: 190 us, in 2048 235; 8 sequences of 2048 with 1024 rows: 98, in 1024 175).
void share_out(AttentionShare& s, int dim, long long rows, long long times, long long tokens) {
  s.many = rows > 32 && (double)(rows * times) * (double)tokens * dim >= 1.6e9;
  const long long tile = s.many ? 32 * kWaves : 16, step = kKeys * (s.many ? 1 : kWaves), want = s.many || dim > 128 ? 512 : 2048;
  s.tiles = (int)std::max(1ll, (rows + tile - 1) / tile);
  const long long most = std::max(1ll, std::min<long long>(kMostParts, tokens / (2 * step)));
  const long long parts = std::min(std::max(1ll, want / std::max(1ll, s.tiles * times)), most);
  s.part_len = (int)(std::max(1ll, (tokens + parts * step - 1) / (parts * step)) * step);
  s.parts = (int)std::max(1ll, (tokens + s.part_len - 1) / s.part_len);
}

}  // namespace

void attention_split(AttentionArgs& a, int max_queries, int max_length) {
  share_out(a.own, a.c.dim, (long long)max_queries * a.group, (long long)std::max(1, a.n_seqs) * a.c.heads, max_length);
  if (a.prefix_len > 0) share_out(a.prefix, a.c.dim, (long long)a.n_queries * a.group, a.c.heads, a.prefix_len);
  else a.prefix = AttentionShare{1, 0, kKeys, false};
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
