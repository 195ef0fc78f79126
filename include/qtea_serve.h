/*
 * qtea_serve.h - C ABI of the operators that stand around the compressed
 * products in a decoder's serving step, for MI355X (gfx950): a paged
 * key/value cache in 16, 8 or 4 bits with the rotation of keys and queries by
 * their positions, causal attention of a batch's newest tokens over it, and the
 * verification of drafted tokens.
 *
 * Conventions as in qtea.h: plain C, device pointers owned by the caller,
 * nothing is allocated, device work is enqueued on `stream` and never
 * synchronized, every call returns a qtea_status code and enqueues nothing
 * on an argument error.  All calls can be captured into a HIP graph: what
 * changes from step to step (lengths, page tables, probabilities) is read
 * from device memory by the kernels.
 */
#ifndef QTEA_SERVE_H_
#define QTEA_SERVE_H_

#include <stdint.h>

#include "qtea.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Element types of dense operands. */
enum qtea_type { QTEA_F16 = 0, QTEA_BF16 = 1, QTEA_F32 = 2 };

/* Storage of cached keys and values. */
enum qtea_kv_format {
  QTEA_KV_F16 = 0,
  QTEA_KV_BF16 = 1,
  QTEA_KV_E4M3 = 2, /* 8-bit codes, blocks of 32 channels share a scale */
  QTEA_KV_E2M1 = 3  /* 4-bit codes, the same blocks                     */
};

#define QTEA_KV_BLOCK 32       /* channels per scale                       */
#define QTEA_KV_MAX_DIM 256    /* largest head dimension                   */
#define QTEA_KV_MAX_PAGE 4096  /* largest page size in tokens              */
#define QTEA_KV_MAX_LEN (INT32_MAX - 2 * QTEA_KV_MAX_PAGE) /* positions of a page table */

/*
 * A cache: pools of pages, each page page_size tokens of every head.
 *
 *   k, v              device codes [n_pages][n_heads][page_size][head_dim]:
 *                     16-bit values, E4M3 bytes, or E2M1 pairs (channel 2i
 *                     in the low half of byte i); 16-byte aligned
 *   k_scale, v_scale  device uint8 [n_pages][n_heads][page_size][head_dim/32]
 *                     (quantized formats; NULL otherwise); 16-byte aligned
 *   head_dim          a multiple of 32, 32..256
 *   page_size         a power of two, 16..4096
 *
 * Quantized formats are microscaled: the block of channels 32b..32b+31 of a
 * token and head stands for code * 2^(scale[b] - 127).  E4M3: sign, four
 * exponent bits (bias 7), three mantissa bits, largest value 448.  E2M1:
 * 0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives.  A scale of 255 makes the
 * whole block NaN.  qtea_kv_append only writes scales for which every value
 * of the block is an fp16 (and a bf16) value: reading loses nothing.
 */
typedef struct qtea_kv_cache {
  void* k;
  void* v;
  uint8_t* k_scale;
  uint8_t* v_scale;
  int64_t n_pages;
  int32_t format;   /* enum qtea_kv_format */
  int32_t n_heads;  /* key/value heads     */
  int32_t head_dim;
  int32_t page_size;
} qtea_kv_cache;

/*
 * A step's sequences and its new tokens.  Sequence s has the dense rows
 * q_start[s] .. q_start[s+1]-1 (its n_s newest tokens, possibly none) and
 * kv_len[s] cached tokens including those: row q_start[s] + i is position
 * kv_len[s] - n_s + i, and position p is row p % page_size of page
 * page_table[s][p / page_size].
 *
 *   q_start     device int32 [n_seq + 1], not decreasing, in [0, n_tokens]
 *   kv_len      device int32 [n_seq], in [0, max_pages * page_size]
 *   page_table  device int32 [n_seq][max_pages]; entries that hold no
 *               position below kv_len are not read as pages
 *               max_pages * page_size is at most QTEA_KV_MAX_LEN: what the
 *               kernels add to a position stays an int32
 *   n_tokens    rows of the dense operands; rows outside every sequence
 *               are left as they are
 *
 * The kernels check what they read from these arrays and stay inside the
 * operands: q_start is taken within [0, n_tokens]; a kv_len outside its
 * range, or a page outside [0, n_pages) among a sequence's visible ones,
 * gives NaN outputs (qtea_kv_append writes nothing there).
 */
typedef struct qtea_kv_batch {
  const int32_t* q_start;
  const int32_t* kv_len;
  const int32_t* page_table;
  int64_t n_tokens;
  int32_t n_seq;
  int32_t max_pages;
} qtea_kv_batch;

/*
 * Write the batch's new keys and values into the cache.
 *   k, v      device [n_tokens][n_heads][head_dim] of `type` (enum
 *             qtea_type), `k_stride` / `v_stride` elements from one token
 *             to the next (>= n_heads * head_dim): columns of a fused
 *             projection's output can be passed in place.  16-byte aligned,
 *             strides a multiple of 16 bytes, below 2^29 elements.
 * 16-bit formats: rounded to nearest.  Quantized formats, per block of 32
 * channels: the scale is the smallest power of two 2^e with
 * max|x| <= 448 * 2^e, -15 <= e <= 7 (E4M3) or max|x| <= 6 * 2^e,
 * -23 <= e <= 13 (E2M1); the codes are x / 2^e to nearest, ties to even,
 * saturating.  A block that holds a NaN or an infinity becomes NaN.  A row
 * whose position is negative (n_s > kv_len[s]) is not written.
 * Errors: QTEA_ERR_INVALID_ARG, QTEA_ERR_HIP.
 */
int qtea_kv_append(const qtea_kv_cache* cache, const qtea_kv_batch* batch, const void* k, const void* v, int type,
                   int64_t k_stride, int64_t v_stride, void* stream);

/*
 * qtea_kv_append with the rotation by position: query and key heads are
 * rotated by their tokens' positions, the queries go to q_out, the keys and
 * (as they are) the values into the cache.  For a token at position p, pair i
 * of a head's first rot_dim channels (i < rot_dim / 2) turns by p * freq[i]:
 *
 *   (a, b) <- (a cos - b sin, b cos + a sin),
 *
 * pair i being channels i and i + rot_dim / 2, or, interleaved, 2i and 2i + 1.
 * The angle, its sine and its cosine are taken in 64 bits (off by at most 2^-36 at
 * angles up to 2^46, 2^-28 up to 2^51) and rounded to 32, the products are taken
 * in 32; then one rounding, to q_out_type or the cache's format.
 *
 *   q, k, v     device [n_tokens][n_q_heads (q) or n_heads][head_dim] of
 *               `type`, strides and alignment as qtea_kv_append's: the three
 *               parts of a fused projection's output can be passed in place
 *   q_out       device [n_tokens][n_q_heads][head_dim] of q_out_type (enum
 *               qtea_type), q_out_stride elements from token to token; 16-byte
 *               aligned, stride a multiple of 16 bytes.  It may be q itself
 *               (same type and stride); other operands must not overlap it
 *   n_q_heads   0 .. 65535; 0: keys and values only (q and q_out NULL)
 *   freq        device fp32 [rot_dim / 2], of magnitude up to 2^20
 *   rot_dim     a multiple of 16, 16 .. head_dim; channels past it are
 *               not turned
 * A token whose position is negative (n_s > kv_len[s]) gets a q_out of zeros, one
 * of a sequence whose kv_len is out of range NaN; rows of no sequence are
 * left as they are.
 * Errors: QTEA_ERR_INVALID_ARG, QTEA_ERR_HIP.
 */
int qtea_kv_append_rotated(const qtea_kv_cache* cache, const qtea_kv_batch* batch, const void* q, const void* k, const void* v,
                           int type, int64_t q_stride, int64_t k_stride, int64_t v_stride, int n_q_heads, const float* freq,
                           int rot_dim, int interleaved, void* q_out, int q_out_type, int64_t q_out_stride, void* stream);

/*
 * Read the batch's rows back: the inverse of qtea_kv_append, with the same
 * operands as outputs.  (All of a sequence: n_s = kv_len[s].)  Values of
 * quantized formats are exact in every type; 16-bit ones are rounded to
 * nearest where the types differ.  Rows of negative position become zero.
 */
int qtea_kv_read(const qtea_kv_cache* cache, const qtea_kv_batch* batch, void* k, void* v, int type, int64_t k_stride,
                 int64_t v_stride, void* stream);

/*
 * Workspace bytes of qtea_paged_attention for n_q_heads query heads of
 * head_dim channels, for any cache and any batch on the current device.
 * It holds arrival counters and partial rows, and must be zero-filled once
 * before its first use (qtea_workspace_init); every call that runs to
 * completion leaves the counters at zero.  Calls that may overlap in time
 * must not share one, and no other entry point may use it.
 */
int qtea_attention_workspace_bytes(int n_q_heads, int head_dim, int64_t* out_bytes);

/*
 * Causal attention of the batch's new tokens over the cache (which already
 * holds them).  For the row of sequence s at position p, query head a and
 * its key/value head h = a / (n_q_heads / n_heads):
 *
 *   out = sum_j w_j v[j][h] / sum_j w_j,   w_j = exp(scale * q . k[j][h]),
 *
 * over the positions j <= p, with window > 0 also j > p - window.  A row
 * that sees no position (p < 0) becomes zero.  What a row does not see does
 * not reach it, NaN and infinities included.
 *
 *   q, out     device [n_tokens][n_q_heads][head_dim] of `type` (QTEA_F16 or
 *              QTEA_BF16; a 16-bit cache's own type), q_stride / out_stride
 *              elements from one token to the next (>= n_q_heads *
 *              head_dim); 16-byte aligned, strides a multiple of 8
 *   scale      > 0, and scale log2(e) an fp32 number (up to 2.3e38)
 *   window     0 (none) or the number of positions a row sees
 *   workspace  device, >= qtea_attention_workspace_bytes
 *
 * Sequences may have any mix of lengths: one token each (decoding), a few
 * (drafts), chunks of a prompt.  The products run on the matrix cores in
 * `type` with fp32 sums; the softmax is fp32, its weights are rounded to
 * `type` for the second product.  Run-to-run deterministic.
 * Errors: QTEA_ERR_INVALID_ARG (also where n_tokens and the page table
 * together would make more than 2^31 pieces of work), QTEA_ERR_WORKSPACE,
 * QTEA_ERR_HIP.
 */
int qtea_paged_attention(const qtea_kv_cache* cache, const qtea_kv_batch* batch, const void* q, void* out, int type,
                         int n_q_heads, int64_t q_stride, int64_t out_stride, float scale, int window, void* workspace,
                         int64_t workspace_bytes, void* stream);

/*
 * Workspace bytes of qtea_verify_draft for n_seq sequences.  As the
 * attention's it holds arrival counters, is zero-filled once, and must not be
 * shared by calls that may overlap in time, nor with another entry point.  One
 * made for n_seq sequences serves every smaller call too, in any order.
 */
int qtea_verify_workspace_bytes(int n_seq, int64_t* out_bytes);

/*
 * Verification of drafted tokens: which of them a sequence keeps, and its
 * next token, distributed as the target's own samples would be.
 *
 * Sequence s has the target rows q_start[s] .. q_start[s+1]-1 (as in the
 * batch that computed them): n_s = their number - 1 drafted tokens and the
 * distribution after the last of them.  The sequences' drafts follow each
 * other in `tokens` and `u_accept` and as rows of `draft`, n_drafts in all.
 *
 * Probabilities are taken in whole units of 2^-38, floor(2^38 p) with p
 * limited to [0, 1] (NaN: 0), the given random numbers in units of 2^-24,
 * so that every decision is exact and no order of summation changes a token:
 *   draft i is accepted when U_i Q_i(x_i) < 2^24 P_i(x_i) (u < p / q), and
 *   all before it are;
 *   at the first rejected draft r, W = max(P_r - Q_r, 0) (if that is zero
 *   everywhere: P_r); with all accepted, W = P_{n_s};
 *   the next token is the lowest v with sum_{w <= v} W(w) >
 *   floor(U sum(W) / 2^24), U the sequence's u_sample; -1 where W has no
 *   mass at all.
 *
 *   target      device [rows][vocab] of `type`, target_stride elements apart
 *               (not read, and possibly NULL, where n_rows is 0)
 *   draft       the same for the drafts, draft_stride apart; NULL: every
 *               drafted token had probability 1 (a deterministic draft)
 *   tokens      device int32 [drafts]; one outside [0, vocab) is rejected
 *   q_start     device int32 [n_seq + 1], not decreasing, in [0, n_rows]
 *   u_accept    device fp32 [drafts], u_sample  device fp32 [n_seq], in [0, 1)
 *   n_accepted  device int32 [n_seq]
 *   out_tokens  device int32 [n_seq][max_draft + 1]: the accepted tokens,
 *               the next token, then -1.  A sequence with more than
 *               max_draft drafts has the rest of them ignored (its row
 *               max_draft is then the distribution after the last kept).
 *               A sequence without rows gets 0 and -1s.
 *   vocab       1 .. 2^24; max_draft 0 .. 1023
 * Errors: QTEA_ERR_INVALID_ARG, QTEA_ERR_WORKSPACE, QTEA_ERR_HIP.
 */
int qtea_verify_draft(const void* target, const void* draft, int type, int64_t vocab, int64_t target_stride,
                      int64_t draft_stride, const int32_t* tokens, const int32_t* q_start, const float* u_accept,
                      const float* u_sample, int n_seq, int64_t n_rows, int64_t n_drafts, int max_draft, int32_t* n_accepted,
                      int32_t* out_tokens, void* workspace, int64_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* QTEA_SERVE_H_ */
