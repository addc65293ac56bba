/*
 * nightjar_serve.h -- what lies between a prompt and its first token on MI355X:
 * chunks of new tokens written to the paged KV cache (in 32, 16 or 8 bits) and
 * read back, the attention of such a chunk over the cache, and sampling with
 * temperature, top-k, top-p and min-p.  Part of libnightjar.so; conventions
 * (return codes, nightjar_last_error, streams, workspaces, device errors, page
 * layouts) as in nightjar.h.
 *
 * The verify step (nightjar.h) scores windows of up to 16 tokens whose keys and
 * values are committed only after acceptance.  A chunk is the other way round:
 * its tokens are known (a prompt, or the one token a decoding step has just
 * drawn), so their keys and values go to the pages first and the attention reads
 * everything from there.  fp32 and bf16 pages are the verify step's own.
 */
#ifndef NIGHTJAR_SERVE_H
#define NIGHTJAR_SERVE_H

#include <stddef.h>
#include <stdint.h>

#include "nightjar.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * Element type of a cache's pages, beside NJ_F32 and NJ_BF16: 8-bit e4m3 (the
 * OCP format without infinities), with one power-of-two scale per (token, KV
 * head) of K and of V.
 */
enum { NJ_E4M3 = 2 };

/* Device error bits, beside those of nightjar.h. */
enum {
  NJ_DEV_BAD_SAMPLING = 32 /* a row that cannot be sampled: a setting out of range, a NaN or +inf
                              logit, or no finite logit at all (its token is -1)            */
};

/*
 * One layer's paged cache.
 *   k        device [num_blocks][Hkv][16][D]
 *   v        device [num_blocks][Hkv][D][16]   (dim-major inside a block)
 *   k_scale, v_scale
 *            NJ_E4M3: device uint8 [num_blocks][Hkv][16], the scale of token
 *            slot t of a block and head as a biased power of two: an element's
 *            value is code * 2^(byte - 127).  Otherwise NULL.
 * NJ_F32 pages go with NJ_F32 descriptors; NJ_BF16 and NJ_E4M3 pages with
 * NJ_BF16 descriptors.
 */
typedef struct nj_kv_layer {
  void* k;
  void* v;
  void* k_scale;
  void* v_scale;
  int32_t num_blocks;
  int32_t dtype;
} nj_kv_layer;

/*
 * A ragged batch of chunks: sequence b's n_b = starts[b+1] - starts[b] new
 * tokens are rows starts[b] .. starts[b+1]-1 of the row arrays and sit at
 * positions context_lens[b] + i (context_lens: tokens cached before the chunk).
 * n_b may be 0.  Rows behind starts[B] belong to nobody: they are neither read
 * nor written.  The struct is host memory, read during the call.
 *
 *   starts        device int32 [B+1], not decreasing, 0 <= starts[0], starts[B] <= rows
 *   context_lens  device int32 [B], not modified
 *   block_table   device int32 [B][max_blocks], max_blocks <= 2^21
 *   B, rows       1 <= B <= 2^20, 1 <= rows <= 2^24: rows of the row arrays
 *   max_chunk     no sequence has more new tokens than this (1 <= max_chunk <= rows)
 *
 * A sequence that breaks these rules, or whose positions do not fit the block
 * table, is skipped whole (NJ_DEV_BAD_CONTEXT; where starts decrease, rows of other
 * sequences may be skipped with it); a token whose block id is
 * outside [0, num_blocks) is skipped (NJ_DEV_BAD_BLOCK; an attention row that
 * needs such a block is undefined).
 */
typedef struct nj_chunk_batch {
  const int32_t* starts;
  const int32_t* context_lens;
  const int32_t* block_table;
  int32_t max_blocks;
  int32_t B;
  int32_t rows;
  int32_t max_chunk;
} nj_chunk_batch;

/*
 * Workspace of the three chunk calls: device memory, 256-byte aligned, prepared
 * once with nightjar_workspace_init.  nightjar_chunk_store and
 * nightjar_chunk_load need 256 bytes (the device error word);
 * nightjar_chunk_attn the bytes returned here (0 if an argument is invalid).
 * A workspace for (B, rows, max_chunk) serves every smaller batch.
 * Calls that overlap in time need workspaces of their own.
 */
size_t nightjar_chunk_attn_workspace_bytes(const nj_model_desc* desc, int32_t B, int32_t rows, int32_t max_chunk);

/*
 * nightjar_chunk_store -- RoPE on a chunk's queries and keys, and its keys and
 * values into the pages, quantised as they are written.
 *
 *   qkv         device fp32, row r at qkv + r * qkv_stride: [q | k | v] of
 *               (H + 2 Hkv) * D values, as the QKV projection gives them
 *               (nightjar_gemm); 16-byte aligned, qkv_stride % 4 == 0
 *   q_out       device [rows][H][D] (desc dtype), 16-byte aligned: rotated queries, apart from qkv;
 *               NULL: not wanted
 * Rotation as in nightjar_rmsnorm_rope (rotate-half, pair (j, j + D/2) turns by
 * position * rope_theta^(-2j/D)), angle and products in 64 bits, rounded once.
 * NJ_E4M3: a head row's scale is the smallest power of two 2^e with
 * max |x| <= 448 * 2^e over its finite values, e in [-112, 119] (so that every
 * stored value is exact in bf16); codes are round-to-nearest-even of x * 2^-e,
 * saturated at 448; NaN and infinities become NaN codes.  Slots of other tokens
 * in the same blocks are left as they are.  Only the tokens' own slots are
 * written; where two rows of one call share a slot (two sequences that share a
 * block), what it holds afterwards is undefined.
 */
int nightjar_chunk_store(const nj_model_desc* desc, const nj_kv_layer* kv, const nj_chunk_batch* batch,
                         const float* qkv, int64_t qkv_stride, void* q_out, void* workspace, size_t workspace_bytes,
                         void* stream);

/*
 * nightjar_chunk_load -- reads the chunk's positions back from the pages:
 *   k_out, v_out   device [rows][Hkv][D] (desc dtype), 16-byte aligned, apart from each other;
 *                  8-bit values are exact in bf16
 * With context_lens 0 and n_b the cached lengths it reads whole contexts.
 */
int nightjar_chunk_load(const nj_model_desc* desc, const nj_kv_layer* kv, const nj_chunk_batch* batch, void* k_out,
                        void* v_out, void* workspace, size_t workspace_bytes, void* stream);

/*
 * nightjar_chunk_attn -- attention of the chunk's rows over the paged cache:
 * row i of sequence b attends to its cached positions 0 .. context_lens[b] + i
 * (the chunk's own keys and values included, stored before); query head h reads
 * KV head h / (H / Hkv); scores q.k / sqrt(D), softmax, weighted sum of values.
 *
 *   q     device [rows][H][D] (desc dtype), 16-byte aligned
 *   out   device [rows][H*D] (desc dtype), 16-byte aligned; may not overlap q
 */
int nightjar_chunk_attn(const nj_model_desc* desc, const nj_kv_layer* kv, const nj_chunk_batch* batch, const void* q,
                        void* out, void* workspace, size_t workspace_bytes, void* stream);

/*
 * nightjar_sample -- one token per row of logits, from given uniforms.
 *
 * Tokens are ordered by logit, largest first, ties to the lowest index.  With
 * weights w_j = exp((l_j - max l) / temperature):
 *   top-k   keeps the first top_k tokens (top_k <= 0: all);
 *   top-p   of these, the shortest prefix whose weights sum to at least top_p
 *           times theirs (never less than one token; top_p >= 1: all);
 *   min-p   of these, the tokens with w_j >= min_p (min_p == 0: all).
 * The token is the smallest kept index whose running sum of kept weights (index
 * order) exceeds uniforms[r] times their total.  temperature 0 is greedy: the
 * largest logit, lowest index.  A logit of -inf is never drawn.  Weights are
 * computed and summed in 64 bits, in an order that depends on vocab alone.
 *
 *   logits       device fp32, row r at logits + r * logits_stride (>= vocab)
 *   temperature, top_p, min_p   device fp32 [rows], top_k device int32 [rows];
 *                each may be NULL: 1, 1, 0, 0.  temperature finite and >= 0, top_p >= 0,
 *                0 <= min_p <= 1, uniforms in [0, 1), else NJ_DEV_BAD_SAMPLING
 *   uniforms     device fp32 [rows]
 *   tokens       device int32 [rows], out (-1 where a row cannot be sampled)
 *   probs        device fp32, row r at probs + r * probs_stride (>= vocab), out: the
 *                distribution the token was drawn from, w_j / total for kept tokens, else 0
 *                (all 0 where a row cannot be sampled); may not overlap logits; NULL: not
 *                wanted.  With stride k*V this is column i of a draft's
 *                draft_probs [B][k][V] (nightjar_verify_step); log(probs) is a valid
 *                logits input of nightjar_accept, which then tests against the truncated
 *                target distribution.
 *   vocab        1 .. 524288
 *   workspace    device, 256-byte aligned, >= nightjar_sample_workspace_bytes(rows, vocab),
 *                prepared once with nightjar_workspace_init
 */
size_t nightjar_sample_workspace_bytes(int32_t rows, int32_t vocab);
int nightjar_sample(const float* logits, int64_t logits_stride, int32_t rows, int32_t vocab, const float* temperature,
                    const int32_t* top_k, const float* top_p, const float* min_p, const float* uniforms,
                    int32_t* tokens, float* probs, int64_t probs_stride, void* workspace, size_t workspace_bytes,
                    void* stream);

#ifdef __cplusplus
}
#endif

#endif /* NIGHTJAR_SERVE_H */
