// C-ABI entry points of the operators of a token model's serving step: what a caller hands over is checked here, then launched.
#include <algorithm>
#include <utility>
#include <hip/hip_runtime.h>

#include "status.h"
#include "token_kernels.h"

using namespace xenos;

namespace {

// The launch geometry has fewer than 2^32 threads.
constexpr long long kMostGroups = 1ll << 22;

bool aligned(const void* p, size_t to) { return (uintptr_t)p % to == 0; }
size_t size_of(xenos_dtype t) { return t == XENOS_BF16 ? 2 : 4; }
bool known(xenos_dtype t) { return t == XENOS_F32 || t == XENOS_BF16; }

xenos_status launched(int err, const char* what) {
  return err ? fail(XENOS_EDEVICE, "%s: %s", what, hipGetErrorString((hipError_t)err)) : XENOS_OK;
}

xenos_status rows_of(const char* who, const void* d_x, xenos_dtype dtype, int rows, int cols, long long row_stride, const float* d_gamma, float eps, void* d_q, float* d_scale,
                     QuantRowsArgs& a) {
  if (rows < 0 || cols <= 0 || !known(dtype)) return fail(XENOS_EINVAL, "%s: %d rows of %d columns, type %d", who, rows, cols, (int)dtype);
  if (cols > XENOS_QUANT_MAX_COLS) return fail(XENOS_EUNSUPPORTED, "%s: %d columns, at most %d", who, cols, XENOS_QUANT_MAX_COLS);
  // (a workgroup's row counter goes beyond the last row by less than the launch's workgroups)
  if (rows > (1 << 30)) return fail(XENOS_EUNSUPPORTED, "%s: %d rows, at most %d", who, rows, 1 << 30);
  if (rows == 0) return XENOS_OK;
  if (!d_x || !d_q || !d_scale) return fail(XENOS_EINVAL, "%s: NULL argument", who);
  if (rows > 1 && row_stride < cols) return fail(XENOS_ESHAPE, "%s: rows of %d elements, %lld apart", who, cols, row_stride);
  if (!aligned(d_x, size_of(dtype)) || !aligned(d_gamma, 4) || !aligned(d_q, 16) || !aligned(d_scale, 4))
    return fail(XENOS_EINVAL, "%s: a buffer is not aligned (the quantised rows, or the workspace: to 16 bytes)", who);
  if (d_gamma && !(eps >= 0.f)) return fail(XENOS_EINVAL, "%s: eps %g", who, (double)eps);
  a = QuantRowsArgs{d_x, d_gamma, (int8_t*)d_q, d_scale, rows > 1 ? row_stride : 0, quant_pitch(cols), rows, cols, eps, 0, aligned(d_gamma, 16)};
  a.vec = aligned(d_x, 16) && a.stride * size_of(dtype) % 16 == 0;
  return XENOS_OK;
}

xenos_status matmul_of(const char* who, const xenos_quant_matmul_args* p, QuantMatmulArgs& a) {
  if (!p || p->rows < 0 || p->cols <= 0 || p->out_c < 0 || !known(p->dtype)) return fail(XENOS_EINVAL, "%s: bad argument", who);
  if (p->cols > XENOS_QUANT_MAX_COLS) return fail(XENOS_EUNSUPPORTED, "%s: %d columns, at most %d", who, p->cols, XENOS_QUANT_MAX_COLS);
  if (p->rows == 0 || p->out_c == 0) return XENOS_OK;
  if (!p->d_q || !p->d_scale || !p->d_w || !p->d_w_scale || !p->d_out) return fail(XENOS_EINVAL, "%s: NULL argument", who);
  if (p->rows > 1 && (p->out_stride < p->out_c || (p->d_residual && p->residual_stride < p->out_c)))
    return fail(XENOS_ESHAPE, "%s: rows of %d elements, %lld (out) and %lld (residual) apart", who, p->out_c, p->out_stride, p->residual_stride);
  const size_t esz = size_of(p->dtype);
  if (!aligned(p->d_q, 16) || !aligned(p->d_w, 16) || !aligned(p->d_scale, 4) || !aligned(p->d_w_scale, 4) || !aligned(p->d_bias, 4) || !aligned(p->d_out, esz) ||
      !aligned(p->d_residual, esz))
    return fail(XENOS_EINVAL, "%s: a buffer is not aligned (quantised rows: to 16 bytes)", who);
  if (((p->rows + 63ll) / 64) * ((p->out_c + 15ll) / 16) > kMostGroups)
    return fail(XENOS_EUNSUPPORTED, "%s: %d x %d results are more than one launch holds", who, p->rows, p->out_c);
  a = QuantMatmulArgs{(const int8_t*)p->d_q, (const int8_t*)p->d_w, p->d_scale, p->d_w_scale, p->d_bias, p->d_residual, p->d_out, quant_pitch(p->cols),
                      p->rows > 1 ? p->residual_stride : 0, p->rows > 1 ? p->out_stride : 0, p->rows, p->out_c, p->relu ? 1 : 0, nullptr, (p->out_c + 7) / 8 * 8, 0};
  a.vec_out = a.out_stride * esz % 16 == 0 && aligned(a.out, 16) && (!a.res || (a.res_stride * esz % 16 == 0 && aligned(a.res, 16)));
  return XENOS_OK;
}

// A layer's workspace: quantised rows, their scales, and the sums of K's shares.
struct LinearSpace {
  size_t scale, part, bytes;
  int splits;
};
LinearSpace linear_space(int rows, int cols, int out_c) {
  const long long pitch = quant_pitch(cols);
  LinearSpace s{};
  if (rows == 0 || linear_in_one(rows, pitch, out_c)) return s;
  s.scale = (size_t)rows * pitch;
  s.part = (s.scale + (size_t)rows * 4 + 15) / 16 * 16;
  s.splits = quant_splits(rows, out_c, pitch);
  s.bytes = s.part + (s.splits > 1 ? (size_t)s.splits * rows * ((out_c + 7ll) / 8 * 8) * 4 : 0);
  return s;
}

xenos_status cache_of(const xenos_cache* c, const char* who, CacheArgs& a) {
  if (!c || c->n_pages < 0 || c->page_tokens <= 0 || c->heads <= 0 || c->head_dim <= 0) return fail(XENOS_EINVAL, "%s: bad cache description", who);
  if (c->page_tokens % 16 || c->head_dim % 16 || c->head_dim > 256)
    return fail(XENOS_EUNSUPPORTED, "%s: pages of %d tokens, heads of %d values (multiples of 16, at most 256 values)", who, c->page_tokens, c->head_dim);
  if (c->n_pages > 0 && (!c->d_k || !c->d_v || !c->d_k_scale || !c->d_v_scale)) return fail(XENOS_EINVAL, "%s: NULL cache buffer", who);
  if (!aligned(c->d_k, 16) || !aligned(c->d_v, 16) || !aligned(c->d_k_scale, 16) || !aligned(c->d_v_scale, 16))
    return fail(XENOS_EINVAL, "%s: a cache buffer is not aligned to 16 bytes", who);
  a = CacheArgs{(int8_t*)c->d_k, (int8_t*)c->d_v, c->d_k_scale, c->d_v_scale, c->n_pages, c->page_tokens, c->heads, c->head_dim};
  return XENOS_OK;
}

// Do any two of tokens x heads rows of `dim` elements, so many elements apart, share one?  (Nested as they are nearly always, the larger stride steps over all rows of the smaller
// one; else each token is held against those heads of the first one that lie around it.)
bool rows_overlap(long long tokens, long long heads, long long token_stride, long long head_stride, int dim) {
  if ((tokens > 1 && token_stride < dim) || (heads > 1 && head_stride < dim)) return true;
  if (tokens <= 1 || heads <= 1) return false;
  const auto span = [&](long long n, long long stride) { return (__int128)stride * (n - 1) + dim; };
  if (head_stride >= span(tokens, token_stride) || token_stride >= span(heads, head_stride)) return false;
  if (tokens > heads) std::swap(tokens, heads), std::swap(token_stride, head_stride);   // (the loop over the fewer)
  for (long long t = 1; t < tokens; ++t) {
    const __int128 at = (__int128)t * token_stride;
    for (__int128 h = at / head_stride, last = h + 1; h <= last && h < heads; ++h) {
      const __int128 off = at - h * head_stride;
      if (off < dim && -off < dim) return true;
    }
  }
  return false;
}

// Everything of the arguments that can be told without the device's memory.
xenos_status attention_of(const xenos_cache* cache, const xenos_attention_args* p, const char* who, AttentionArgs& a, size_t* bytes) {
  const xenos_status rc = cache_of(cache, who, a.c);
  if (rc != XENOS_OK) return rc;
  if (!p || p->n_seqs < 0 || p->n_queries < 0 || p->heads <= 0 || !known(p->dtype) || p->table_stride < 0 || p->max_queries < 0 || p->max_length < 0 || p->prefix_length < 0)
    return fail(XENOS_EINVAL, "%s: bad argument", who);
  if (p->dtype != XENOS_BF16) return fail(XENOS_EUNSUPPORTED, "%s: queries are bf16", who);
  if (p->heads % cache->heads) return fail(XENOS_ESHAPE, "%s: %d heads over %d heads of the cache", who, p->heads, cache->heads);
  if (p->max_length > (1 << 30) || p->prefix_length > (1 << 30) || (long long)p->n_queries * p->heads > (1 << 28))
    return fail(XENOS_EUNSUPPORTED, "%s: %d queries of %d heads, %d and %d tokens", who, p->n_queries, p->heads, p->max_length, p->prefix_length);
  // (the kernels count positions in 32 bits, to a few steps behind the end of what a table holds)
  if ((long long)p->table_stride * cache->page_tokens > (1 << 30)) return fail(XENOS_EUNSUPPORTED, "%s: tables of %d pages of %d tokens", who, p->table_stride, cache->page_tokens);
  if (p->n_queries > 0 && p->n_seqs == 0) return fail(XENOS_ESHAPE, "%s: %d queries of no sequence", who, p->n_queries);
  if (!p->d_starts && p->n_queries != p->n_seqs) return fail(XENOS_ESHAPE, "%s: %d queries of %d sequences, and no starts", who, p->n_queries, p->n_seqs);
  a.n_seqs = p->n_seqs, a.n_queries = p->n_queries, a.heads = p->heads, a.group = p->heads / cache->heads, a.table_stride = p->table_stride;
  a.prefix_len = p->prefix_length;
  attention_split(a, std::min(p->max_queries, p->n_queries), std::min(p->max_length, p->table_stride * cache->page_tokens));
  const long long own = (long long)a.n_seqs * a.own.tiles * a.own.parts, front = (long long)a.prefix.tiles * a.prefix.parts;
  if ((own + front) * cache->heads > kMostGroups || (long long)p->n_queries * p->heads > 2 * kMostGroups)
    return fail(XENOS_EUNSUPPORTED, "%s: %d queries of %d sequences are more than one launch holds", who, p->n_queries, p->n_seqs);
  *bytes = attention_slots(a) > 1 ? (size_t)p->n_queries * p->heads * attention_slots(a) * (cache->head_dim + 2) * 4 : 0;
  return XENOS_OK;
}

}  // namespace

extern "C" {

xenos_status xenos_quant_rows(const void* d_x, xenos_dtype dtype, int rows, int cols, long long row_stride, const float* d_gamma, float eps,
                              void* d_q, float* d_scale, void* hip_stream) {
  QuantRowsArgs a{};
  const xenos_status rc = rows_of("xenos_quant_rows", d_x, dtype, rows, cols, row_stride, d_gamma, eps, d_q, d_scale, a);
  if (rc != XENOS_OK || rows == 0) return rc;
  return launched(launch_quant_rows(a, dtype, hip_stream), "xenos_quant_rows");
}

xenos_status xenos_quant_matmul(const xenos_quant_matmul_args* p, void* hip_stream) {
  QuantMatmulArgs a{};
  const xenos_status rc = matmul_of("xenos_quant_matmul", p, a);
  if (rc != XENOS_OK || p->rows == 0 || p->out_c == 0) return rc;
  return launched(launch_quant_matmul(a, p->dtype, hip_stream), "xenos_quant_matmul");
}

xenos_status xenos_linear_workspace(int rows, int cols, int out_c, size_t* bytes) {
  if (rows < 0 || cols <= 0 || cols > XENOS_QUANT_MAX_COLS || out_c < 0 || !bytes) return fail(XENOS_EINVAL, "xenos_linear_workspace: %d rows of %d columns, %d results", rows, cols, out_c);
  *bytes = linear_space(rows, cols, out_c).bytes;
  return XENOS_OK;
}

xenos_status xenos_linear(const xenos_linear_args* p, void* d_workspace, size_t workspace_bytes, void* hip_stream) {
  if (!p) return fail(XENOS_EINVAL, "xenos_linear: NULL argument");
  LinearSpace space{};
  if (p->rows >= 0 && p->cols > 0 && p->cols <= XENOS_QUANT_MAX_COLS && p->out_c >= 0) space = linear_space(p->rows, p->cols, p->out_c);
  if (space.bytes && (!d_workspace || workspace_bytes < space.bytes)) return fail(XENOS_EINVAL, "xenos_linear: a workspace of %zu bytes, %zu are needed", workspace_bytes, space.bytes);
  // (where nothing is stored there, any aligned address will do)
  int8_t* q = space.bytes ? (int8_t*)d_workspace : (int8_t*)16;
  float* scale = space.bytes ? (float*)(q + space.scale) : (float*)16;
  QuantRowsArgs r{};
  xenos_status rc = rows_of("xenos_linear", p->d_x, p->dtype, p->rows, p->cols, p->x_stride, p->d_gamma, p->eps, q, scale, r);
  if (rc != XENOS_OK) return rc;
  const xenos_quant_matmul_args m{p->rows, p->cols, p->out_c, q, scale, p->d_w, p->d_w_scale, p->d_bias, p->d_residual, p->residual_stride, p->relu, p->dtype, p->d_out, p->out_stride};
  QuantMatmulArgs a{};
  rc = matmul_of("xenos_linear", &m, a);
  if (rc != XENOS_OK || p->rows == 0 || p->out_c == 0) return rc;
  if (space.splits > 1) a.part = (int*)(q + space.part);
  return launched(launch_linear(r, a, p->dtype, hip_stream), "xenos_linear");
}

xenos_status xenos_cache_write(const xenos_cache* cache, int n_tokens, const void* d_k, long long k_token_stride, long long k_head_stride,
                               const void* d_v, long long v_token_stride, long long v_head_stride, xenos_dtype dtype, const long long* d_slots, void* hip_stream) {
  CacheWriteArgs a{};
  const xenos_status rc = cache_of(cache, "xenos_cache_write", a.c);
  if (rc != XENOS_OK) return rc;
  if (n_tokens < 0 || !known(dtype)) return fail(XENOS_EINVAL, "xenos_cache_write: %d tokens, type %d", n_tokens, (int)dtype);
  if (n_tokens == 0) return XENOS_OK;
  if (!d_k || !d_v || !d_slots) return fail(XENOS_EINVAL, "xenos_cache_write: NULL argument");
  if (!aligned(d_k, size_of(dtype)) || !aligned(d_v, size_of(dtype)) || !aligned(d_slots, 8)) return fail(XENOS_EINVAL, "xenos_cache_write: a buffer is not aligned");
  if (k_token_stride < 0 || k_head_stride < 0 || v_token_stride < 0 || v_head_stride < 0) return fail(XENOS_ESHAPE, "xenos_cache_write: negative stride");
  if ((n_tokens + 127ll) / 128 * 8 * cache->heads > 2 * kMostGroups || n_tokens > (1 << 30)) return fail(XENOS_EUNSUPPORTED, "xenos_cache_write: %d tokens of %d heads are more than one launch holds", n_tokens, cache->heads);
  a.k = d_k, a.v = d_v, a.k_token = k_token_stride, a.k_head = k_head_stride, a.v_token = v_token_stride, a.v_head = v_head_stride, a.slots = d_slots, a.tokens = n_tokens;
  a.vec = aligned(d_k, 4 * size_of(dtype)) && aligned(d_v, 4 * size_of(dtype)) && (k_token_stride | k_head_stride | v_token_stride | v_head_stride) % 4 == 0;
  return launched(launch_cache_write(a, dtype, hip_stream), "xenos_cache_write");
}

xenos_status xenos_cache_read(const xenos_cache* cache, int n_tokens, const long long* d_slots, void* d_k, void* d_v, xenos_dtype dtype, void* hip_stream) {
  CacheReadArgs a{};
  const xenos_status rc = cache_of(cache, "xenos_cache_read", a.c);
  if (rc != XENOS_OK) return rc;
  if (n_tokens < 0 || !known(dtype)) return fail(XENOS_EINVAL, "xenos_cache_read: %d tokens, type %d", n_tokens, (int)dtype);
  if (n_tokens == 0) return XENOS_OK;
  if (!d_k || !d_v || !d_slots) return fail(XENOS_EINVAL, "xenos_cache_read: NULL argument");
  if (!aligned(d_k, 16) || !aligned(d_v, 16) || !aligned(d_slots, 8)) return fail(XENOS_EINVAL, "xenos_cache_read: a buffer is not aligned (k and v: to 16 bytes)");
  if ((n_tokens + 127ll) / 128 * 8 * cache->heads > 2 * kMostGroups || n_tokens > (1 << 30)) return fail(XENOS_EUNSUPPORTED, "xenos_cache_read: %d tokens of %d heads are more than one launch holds", n_tokens, cache->heads);
  a.slots = d_slots, a.k = d_k, a.v = d_v, a.tokens = n_tokens;
  return launched(launch_cache_read(a, dtype, hip_stream), "xenos_cache_read");
}

xenos_status xenos_attention_workspace(const xenos_cache* cache, const xenos_attention_args* args, size_t* bytes) {
  AttentionArgs a{};
  size_t need;
  if (!bytes) return fail(XENOS_EINVAL, "xenos_attention_workspace: NULL argument");
  const xenos_status rc = attention_of(cache, args, "xenos_attention_workspace", a, &need);
  if (rc == XENOS_OK) *bytes = need;
  return rc;
}

xenos_status xenos_attention(const xenos_cache* cache, const xenos_attention_args* p, void* d_workspace, size_t workspace_bytes, void* hip_stream) {
  AttentionArgs a{};
  size_t need = 0;
  const xenos_status rc = attention_of(cache, p, "xenos_attention", a, &need);
  if (rc != XENOS_OK) return rc;
  if (p->n_queries == 0 || p->n_seqs == 0) return XENOS_OK;
  if (!p->d_q || !p->d_out || !p->d_lengths || (p->table_stride > 0 && !p->d_tables) || (p->prefix_length > 0 && !p->d_prefix_table))
    return fail(XENOS_EINVAL, "xenos_attention: NULL argument");
  if (!aligned(p->d_q, 2) || !aligned(p->d_out, 2) || !aligned(p->d_starts, 4) || !aligned(p->d_lengths, 4) || !aligned(p->d_tables, 4) || !aligned(p->d_prefix_table, 4) ||
      !aligned(d_workspace, 16))
    return fail(XENOS_EINVAL, "xenos_attention: a buffer is not aligned (the workspace: to 16 bytes)");
  if (p->q_token_stride < 0 || p->q_head_stride < 0 || p->out_token_stride < 0 || p->out_head_stride < 0) return fail(XENOS_ESHAPE, "xenos_attention: negative stride");
  if (rows_overlap(p->n_queries, p->heads, p->out_token_stride, p->out_head_stride, cache->head_dim))
    return fail(XENOS_ESHAPE, "xenos_attention: rows of out overlap (%d values, %lld and %lld apart)", cache->head_dim, p->out_token_stride, p->out_head_stride);
  if (need && (!d_workspace || workspace_bytes < need)) return fail(XENOS_EINVAL, "xenos_attention: a workspace of %zu bytes, %zu are needed", workspace_bytes, need);
  a.q = (const uint16_t*)p->d_q, a.out = (uint16_t*)p->d_out;
  a.q_token = p->q_token_stride, a.q_head = p->q_head_stride, a.out_token = p->out_token_stride, a.out_head = p->out_head_stride;
  a.starts = p->d_starts, a.lengths = p->d_lengths, a.tables = p->d_tables, a.prefix_table = p->d_prefix_table, a.part = (float*)d_workspace;
  a.part_ml = a.part + (size_t)p->n_queries * p->heads * attention_slots(a) * cache->head_dim;
  a.vec_q = aligned(a.q, 16) && a.q_token % 8 == 0 && a.q_head % 8 == 0;
  a.vec_out = aligned(a.out, 8) && a.out_token % 4 == 0 && a.out_head % 4 == 0;
  a.scale2 = p->scale * 1.44269504088896340736f;
  return launched(launch_attention(a, hip_stream), "xenos_attention");
}

xenos_status xenos_logprobs_workspace(int rows, int vocab, int top, size_t* bytes) {
  if (rows < 0 || vocab <= 0 || top < 0 || top > XENOS_TOP_MAX || top > vocab || !bytes)
    return fail(XENOS_EINVAL, "xenos_logprobs_workspace: %d rows of %d tokens, the best %d", rows, vocab, top);
  int parts, len;
  logprobs_split(rows, vocab, &parts, &len);
  *bytes = parts > 1 ? (size_t)rows * parts * logprobs_part_words(top) * 4 : 0;
  return XENOS_OK;
}

xenos_status xenos_logprobs(const void* d_logits, xenos_dtype dtype, int rows, int vocab, long long row_stride, const long long* d_targets, int top,
                            float* d_logprob, float* d_entropy, float* d_top_logprob, int* d_top_token, void* d_workspace, size_t workspace_bytes, void* hip_stream) {
  if (rows < 0 || vocab <= 0 || top < 0 || top > XENOS_TOP_MAX || !known(dtype)) return fail(XENOS_EINVAL, "xenos_logprobs: %d rows of %d tokens, the best %d, type %d", rows, vocab, top, (int)dtype);
  if (top > vocab) return fail(XENOS_ESHAPE, "xenos_logprobs: the best %d of %d tokens", top, vocab);
  if (vocab > (1 << 30)) return fail(XENOS_EUNSUPPORTED, "xenos_logprobs: %d tokens", vocab);
  if (rows == 0) return XENOS_OK;
  if (!d_logits || !d_targets != !d_logprob || (top && (!d_top_logprob || !d_top_token))) return fail(XENOS_EINVAL, "xenos_logprobs: NULL argument");
  if (rows > 1 && row_stride < vocab) return fail(XENOS_ESHAPE, "xenos_logprobs: rows of %d elements, %lld apart", vocab, row_stride);
  if (!aligned(d_logits, size_of(dtype)) || !aligned(d_targets, 8) || !aligned(d_logprob, 4) || !aligned(d_entropy, 4) || !aligned(d_top_logprob, 4) || !aligned(d_top_token, 4) || !aligned(d_workspace, 4))
    return fail(XENOS_EINVAL, "xenos_logprobs: a buffer is not aligned");
  LogprobsArgs a{d_logits, d_targets, d_logprob, d_entropy, d_top_logprob, d_top_token, (uint32_t*)d_workspace, rows > 1 ? row_stride : 0, rows, vocab, top, 1, vocab};
  logprobs_split(rows, vocab, &a.parts, &a.part_len);
  if ((long long)rows * a.parts > kMostGroups) return fail(XENOS_EUNSUPPORTED, "xenos_logprobs: %d rows are more than one launch holds", rows);
  const size_t need = a.parts > 1 ? (size_t)rows * a.parts * logprobs_part_words(top) * 4 : 0;
  if (need && (!d_workspace || workspace_bytes < need)) return fail(XENOS_EINVAL, "xenos_logprobs: a workspace of %zu bytes, %zu are needed", workspace_bytes, need);
  return launched(launch_logprobs(a, dtype, hip_stream), "xenos_logprobs");
}

}  // extern "C"
