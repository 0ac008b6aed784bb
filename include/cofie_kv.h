/*
 * cofie_kv.h -- the part of libcofie_ngff.so that answers from the selected
 * frames: rotary positions, a paged key/value cache of 16-bit values or 4-bit
 * codes, and attention over that cache. It follows the selection of evidence
 * (CoFiE Sec. 3.3: once the frames are ranked, the positional embeddings and
 * the keys and values of the kept ones go on, those of the others do not).
 *
 * Conventions are those of cofie_ngff.h (return codes, streams, handles).
 * Every pointer below named "device memory" must be readable or writable by
 * the GPU of the call; data that a kernel reads there (page tables, lengths,
 * offsets) is checked on the device: an entry out of range is left out, and
 * cofie_kv_status reports it.
 *
 * One batch of sequences. Sequence s owns the rows offsets[s] ..
 * offsets[s + 1] - 1 of every per-token argument (its new tokens), and holds
 * lengths[s] cached tokens, its new ones among them as the last. Cached token
 * i of sequence s lies in page table[s * table_stride + i / page_size], at
 * place i % page_size.
 *
 * Pages: [n_pages][n_kv_heads][page_size][row], keys and values apart.
 *   bits = 16  a row is head_dim values of the cache's type.
 *   bits = 4   a row is head_dim codes, two to a byte (the even dimension in
 *              the low four bits), and beside the pages lie the scale words,
 *              [n_pages][n_kv_heads][page_size][head_dim / 64] uint16. A word
 *              serves 64 consecutive codes: with its low four bits cleared it
 *              is the bf16 scale s (4 significant bits), its low four bits are
 *              the zero point z. Code n stands for (n - z) s, which bf16 holds
 *              exactly (fp16 too, for s from 2^-21 and as long as it does not
 *              pass 65504: cofie_kv_read, and attention of more than 32 rows of a
 *              sequence and key head, see it as a number of the cache's type).
 *   Codes of x (64 values, rotated keys as fp32 numbers; hi - lo is formed in
 *   fp32, all else exactly): lo = min(0, min x), hi = max(0, max x),
 *   s = (hi - lo) / 15 rounded up to 4 significant bits (0 below 2^-100),
 *   z = min(15, [-lo / s]), n = min(15, max(0, [x / s] + z)), [] to the
 *   nearest, halves away from zero. A group that holds a NaN or an infinity,
 *   or whose hi - lo passes fp32's range, reads as NaN.
 */
#ifndef COFIE_KV_H
#define COFIE_KV_H

#include <stddef.h>
#include <stdint.h>

#include "cofie_ngff.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Element types. */
#define COFIE_BF16 0
#define COFIE_FP16 1
#define COFIE_FP32 2 /* cofie_rotary_run only */

/* ------------------------------------------------------------------------
 * Rotary positions. Pair i (0 <= i < rotary_dim / 2) of a head turns by
 * a = pos[axis_i] f_i:  y1 = m (x1 cos a - x2 sin a), y2 = m (x2 cos a + x1 sin a);
 * the head's other head_dim - rotary_dim values pass through.
 *   layout HALF         pair i is (x[i], x[i + rotary_dim / 2])
 *   layout INTERLEAVED  pair i is (x[2 i], x[2 i + 1])
 * f_i = base^(-2 i / rotary_dim), m = 1, changed by the scaling:
 *   LINEAR  f_i / factor
 *   BASE    base times factor^(rotary_dim / (rotary_dim - 2))
 *   YARN    (1 - g) f_i / factor + g f_i, g = (r - slow) / (fast - slow) cut to
 *           [0, 1], r = original_len f_i / (2 pi) the pair's turns over the
 *           trained length; m = 0.1 ln(factor) + 1 (Peng et al. 2023, "YaRN").
 *           This is the paper's g, linear in the turns; programs that make g
 *           linear in i between two whole numbers get other frequencies.
 * Angles are formed as 64-bit fractions of a turn, so that a position up to
 * 2^31 costs no accuracy.
 * ------------------------------------------------------------------------ */
#define COFIE_ROTARY_HALF 0
#define COFIE_ROTARY_INTERLEAVED 1
#define COFIE_ROTARY_NONE 0
#define COFIE_ROTARY_LINEAR 1
#define COFIE_ROTARY_BASE 2
#define COFIE_ROTARY_YARN 3

typedef struct cofie_rotary cofie_rotary_t;

typedef struct {
  uint32_t head_dim;     /* even, 2..256 */
  uint32_t rotary_dim;   /* even, 2..head_dim */
  uint32_t layout;       /* COFIE_ROTARY_HALF or COFIE_ROTARY_INTERLEAVED */
  uint32_t scaling;      /* COFIE_ROTARY_NONE .. COFIE_ROTARY_YARN */
  double base;           /* > 1 */
  double factor;         /* >= 1; 1 without scaling */
  double original_len;   /* YARN: the trained length, >= 1 */
  double beta_fast;      /* YARN: turns from which a pair is left as it is (32) */
  double beta_slow;      /* YARN: turns up to which it is stretched in full (1) */
  uint32_t n_axes;       /* position axes, 1..4 */
  const uint8_t* axes;   /* rotary_dim / 2 axis numbers in host memory, or NULL: all 0 */
} cofie_rotary_params;

/* Rows of one tensor: value d of head h of token t is at in[t in_token + h in_head + d]
 * (strides in elements, any sign and size; the head's values are contiguous). */
typedef struct {
  const void* in; /* device memory */
  void* out;      /* device memory; may be `in` itself with the same strides, else must not overlap it */
  uint32_t heads; /* 1..4096 */
  int64_t in_token, in_head, out_token, out_head;
} cofie_rows;

/* Host-only work. Errors: COFIE_EINVAL, COFIE_ENOMEM. */
int cofie_rotary_create(const cofie_rotary_params* p, cofie_rotary_t** out);
void cofie_rotary_destroy(cofie_rotary_t* h);

/*
 * Rotates n_rows (1..4) tensors of the same n_tokens tokens in one launch.
 *   positions  int32 [n_axes][n_tokens], device memory.
 *   dtype      COFIE_BF16, COFIE_FP16 or COFIE_FP32; sums in fp32, one rounding.
 *   transpose  nonzero: the transposed rotation (angle -a, the same m), which
 *              turns a gradient of the outputs into that of the inputs.
 * n_tokens = 0 is a no-op. May be captured. Errors: COFIE_EINVAL, COFIE_ECUDA.
 */
int cofie_rotary_run(cofie_rotary_t* h, const cofie_rows* rows, uint32_t n_rows, uint32_t n_tokens,
                     const int32_t* positions, uint32_t dtype, int transpose, void* cuda_stream);

/* Last error of h, or of the last failed cofie_rotary_create on this thread when h is NULL. Never NULL. */
const char* cofie_rotary_last_error(const cofie_rotary_t* h);

/* ------------------------------------------------------------------------ */
typedef struct cofie_kv cofie_kv_t;

typedef struct {
  uint32_t n_pages;    /* 1..2^31 - 1 */
  uint32_t page_size;  /* tokens: 16, 32, 64, 128 or 256 */
  uint32_t n_heads;    /* query heads */
  uint32_t n_kv_heads; /* divides n_heads; query head h reads head h / (n_heads / n_kv_heads) */
  uint32_t head_dim;   /* 64 or 128 */
  uint32_t dtype;      /* COFIE_BF16 or COFIE_FP16: queries, keys, values, outputs and 16-bit pages */
  uint32_t bits;       /* 16 or 4 */
  int32_t device;      /* CUDA device ordinal, or -1 for the current device */
  void* k_pages;       /* the caller's device memory, 16-byte aligned, for the handle's lifetime */
  void* v_pages;
  uint16_t* k_scales;  /* bits = 4 only */
  uint16_t* v_scales;
} cofie_kv_params;

typedef struct {
  uint32_t n_seqs;
  uint32_t n_tokens;       /* rows of the per-token arguments; offsets[n_seqs] at most (rows past it are left alone) */
  uint32_t max_new;        /* cofie_kv_attend: at least the largest count of new tokens (0: n_tokens) */
  uint32_t table_stride;   /* entries of one sequence */
  const int32_t* table;    /* [n_seqs][table_stride], device memory */
  const int32_t* lengths;  /* [n_seqs], device memory */
  const int32_t* offsets;  /* [n_seqs + 1], device memory, or NULL: one token each (n_tokens = n_seqs) */
} cofie_kv_batch;

/* Validates *p and allocates the handle's scratch (about 40 MB of device memory at head_dim 128, 20 MB at 64).
 * Synchronous: it waits for the default stream. Errors: COFIE_EINVAL, COFIE_ENOMEM, COFIE_ECUDA. */
int cofie_kv_create(const cofie_kv_params* p, cofie_kv_t** out);
void cofie_kv_destroy(cofie_kv_t* h);

/*
 * Puts the batch's new tokens into the cache, keys rotated on the way. One launch.
 *   k, v       n_kv_heads rows a token (their `out` fields are not used).
 *   q          NULL, or n_heads rows a token, rotated into its `out` by the same launch (needs rotary).
 *   rotary     NULL: keys are stored as they are. Its head_dim is the cache's.
 *   positions  int32 [n_axes][n_tokens], device memory (with rotary).
 * 16-bit pages take the rotated keys rounded once; 4-bit codes are formed from
 * the rotated keys in fp32. Tokens whose page is out of range are left out.
 */
int cofie_kv_append(cofie_kv_t* h, const cofie_kv_batch* b, const cofie_rows* k, const cofie_rows* v,
                    const cofie_rows* q, const cofie_rotary_t* rotary, const int32_t* positions, void* cuda_stream);

/* What the cache holds at the batch's new tokens, as numbers of the cache's
 * type: k_out, v_out [n_tokens][n_kv_heads][head_dim] contiguous, device
 * memory. With lengths[s] new tokens of every sequence this is the whole cache.
 * Rows of tokens whose page is out of range are zero. */
int cofie_kv_read(cofie_kv_t* h, const cofie_kv_batch* b, void* k_out, void* v_out, void* cuda_stream);

/*
 * Attention of the batch's new tokens over their sequences' cached tokens.
 * Query token i of n new ones sees cached token j of m when j <= m - n + i
 * (causal; every j < m otherwise) and mask[s mask_stride + j] is nonzero:
 *   out = sum_j p_j v_j, p = softmax_j(scale <q, k_j>), lse = ln sum_j exp(scale <q, k_j>)
 * Products are of 16-bit numbers, sums in fp32. The weights exp(scale <q, k_j>)
 * are rounded to 16 bits for their product with the values (to the cache's type,
 * of up to 2^8 or 2^11 for fp16; for at most 32 rows over 4-bit pages to fp16,
 * times the values' scale) and not for lse; over 4-bit pages such rows' queries
 * are taken to fp16 with a power of two for each row, which is meant for queries
 * below 2^110. out is rounded to the cache's type. A row that sees nothing gets
 * out = 0, lse = -infinity; what a masked or unwritten place holds (NaN too)
 * never matters. (A NaN or an infinity among a call's own new values may reach
 * all new rows of its sequence, those before it too.)
 *   q     n_heads rows a token; `out` is the output.
 *   lse   NULL, or fp32 [n_tokens][n_heads], device memory.
 *   mask  NULL, or uint8 [n_seqs][mask_stride], device memory, mask_stride >= the longest sequence
 *         (a cached token past mask_stride counts as masked).
 *   scale 0: 1 / sqrt(head_dim).
 * May be captured, except for the first masked call of a larger n_seqs x
 * table_stride, which grows the handle's scratch. Calls captured before it are
 * launched as before (what they use stays until cofie_kv_destroy).
 */
int cofie_kv_attend(cofie_kv_t* h, const cofie_kv_batch* b, const cofie_rows* q, float* lse, const uint8_t* mask,
                    uint64_t mask_stride, int causal, float scale, void* cuda_stream);

/* Synchronises cuda_stream; COFIE_EDEVICE if a kernel met a page number, a length or an offset out of range since the
 * last call, COFIE_ETIMEOUT if a bounded device wait ran out. */
int cofie_kv_status(cofie_kv_t* h, void* cuda_stream);

/* Last error of h, or of the last failed cofie_kv_create on this thread when h is NULL. Never NULL. */
const char* cofie_kv_last_error(const cofie_kv_t* h);

#ifdef __cplusplus
}
#endif

#endif /* COFIE_KV_H */
