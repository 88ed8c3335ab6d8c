// Arguments and launchers of the kernels of a token model's serving step (8-bit linear layers, quantised cache, attention,
// log probabilities).  The entry points in xenos_tokens.cpp have checked everything that is said here of sizes and alignment.
#pragma once
#include <stddef.h>
#include <stdint.h>

namespace xenos {

constexpr float kTinyAmplitude = 7.888609052210118e-31f;     // 2^-100: 127 / it is finite, and so is every quantised row
constexpr int kQuantPitch = 128;                             // bytes: a quantised row's own, rounded up, zeros behind them
inline long long quant_pitch(long long cols) { return (cols + kQuantPitch - 1) / kQuantPitch * kQuantPitch; }

struct QuantRowsArgs {
  const void* x;                                             // [rows][stride], `cols` of each row
  const float* gamma;                                        // [cols] or null
  int8_t* q;                                                 // [rows][pitch]
  float* scale;                                              // [rows]
  long long stride, pitch;
  int rows, cols;
  float eps;
  int vec, vec_gamma;                                        // rows of x, and gamma, start at 16-byte boundaries
};
int launch_quant_rows(const QuantRowsArgs& a, int dtype, void* stream);

struct QuantMatmulArgs {
  const int8_t *x, *w;                                       // [M][pitch], [N][pitch]: K bytes and zeros
  const float *xs, *ws, *bias;                               // [M], [N], [N] or null
  const void* res;                                           // [M][res_stride] or null, of out's type
  void* out;                                                 // [M][out_stride]
  long long pitch, res_stride, out_stride;
  int M, N;
  int relu;
  int* part;                                                 // [quant_splits][M][part_pitch], 16-byte aligned, or null: K is not split
  int part_pitch;                                            // N rounded up to eight
  int vec_out;                                               // rows of out and res start at multiples of 16 bytes
};
int quant_splits(int rows, int out_c, long long pitch);
int launch_quant_matmul(const QuantMatmulArgs& a, int dtype, void* stream);
// Both for one layer.  A few short rows are quantised by every workgroup of the product for itself, which saves a launch; r.q and r.scale are not used then.
// (us in two launches, in one, among others in a graph: 1 x 512 x 2048: 5.5, 4.8; 1 x 4096 x 4096: 7.8, 6.2; 8 x 1024 x 4096: 7.0, 5.8; 16 x 512 x 2048: 6.0, 6.2; 8 x 2048 x 2048, beyond: 7.6, 7.1;
// 16 x 1024 x 4096: 7.3, 7.6.  8192 bytes are also what the one turn of weights covers that is under way meanwhile.)  Each 16 outputs quantise the rows once more: where there
// are 256 tiles of 64 outputs, which the product alone reads in tiles, that is worth it only beside the weights of one long row.  (In two launches, in one: 16 x 512 x 8192: 7.9, 8.7;
// x 16384: 8.1, 15.3; x 131072: 30, 108; 4 x 2048 x 16320: 17.9, 16.5; x 16384: 11.6, 16.5; 1 x 2048 x 32000: 18, 27; 2 x 4096 x 32000: 33, 37; 1 x 4096 x 16384: 20.4, 19.5;
// x 32000: 31.8, 33.5; x 131072: 139, 121; 1 x 8192 x 65536: 134, 100.)
inline bool linear_in_one(int rows, long long pitch, int out_c) {
  return rows <= 16 && rows * pitch <= 8192 && (out_c <= 255 * 64 || (rows == 1 && pitch >= 4096));
}
int launch_linear(const QuantRowsArgs& r, const QuantMatmulArgs& a, int dtype, void* stream);

struct CacheArgs {
  int8_t *k, *v;                                             // 16-byte aligned, as the scales are; the layouts of xenos.h
  float *k_scale, *v_scale;
  int n_pages, page, heads, dim;                             // page and dim are multiples of 16, dim <= 256
};
struct CacheWriteArgs {
  CacheArgs c;
  const void *k, *v;                                         // element (t, h, d) at t * token + h * head + d
  long long k_token, k_head, v_token, v_head;
  const long long* slots;
  int tokens;
  int vec;                                                   // fours of elements are aligned as such
};
struct CacheReadArgs {
  CacheArgs c;
  const long long* slots;
  void *k, *v;                                               // [tokens][heads][dim], 16-byte aligned
  int tokens;
};
// A segment of keys that the row tiles of an attention call pass over: the shared prefix, or the sequences' own tokens.
struct AttentionShare {
  int tiles;                                                 // of rows
  int parts, part_len;                                       // pieces of the keys, of part_len (a multiple of 64) tokens each, the last one to the end
  bool many;                                                 // rows: 32 for each wavefront of a workgroup, not the same 16 for all, which take turns with the keys
};
struct AttentionArgs {
  CacheArgs c;
  const uint16_t* q;
  uint16_t* out;
  long long q_token, q_head, out_token, out_head;
  const int *starts, *lengths, *tables, *prefix_table;
  float *part, *part_ml;                                     // [row][slot][dim] sums and [row][slot][2] maxima and normalisers, 16-byte aligned: unless there is one slot
  int n_seqs, n_queries, heads, group, table_stride, prefix_len;
  int vec_q, vec_out;                                        // rows of q are 16-byte, of out 8-byte aligned
  float scale2;                                              // scale log2 e
  int skip_prefix;                                           // this launch is the sequences' own keys alone
  AttentionShare own, prefix;
};
inline int attention_slots(const AttentionArgs& a) { return a.own.parts + a.prefix.parts; }
void attention_split(AttentionArgs& a, int max_queries, int max_length);
int launch_attention(const AttentionArgs& a, void* stream);

struct LogprobsArgs {
  const void* x;                                             // [rows][stride], `vocab` of each row
  const long long* targets;                                  // [rows] or null
  float *logprob, *entropy;                                  // [rows] or null
  float* top_logprob;                                        // [rows][top]
  int* top_token;
  uint32_t* part;                                            // [rows][parts][logprobs_part_words(top)], unless parts = 1
  long long stride;
  int rows, vocab, top;
  int parts, part_len;                                       // a row is read in `parts` pieces of part_len
};
constexpr int kTopMost = 64;
inline int logprobs_part_words(int top) { return 3 + 2 * top; }
void logprobs_split(int rows, int vocab, int* parts, int* part_len);
int launch_logprobs(const LogprobsArgs& a, int dtype, void* stream);

int launch_cache_write(const CacheWriteArgs& a, int dtype, void* stream);
int launch_cache_read(const CacheReadArgs& a, int dtype, void* stream);

}  // namespace xenos
