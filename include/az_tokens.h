/*
 * az_tokens -- the output end of a language model on one NVIDIA B200 (sm_100a), from hidden states to the
 * probabilities of the next token.  It takes the steps that az_evaluate's policy head takes for the moves of a
 * position (features -> matrix product -> logits -> softmax over the entries a bit mask allows) with kernels of
 * its own, for vocabularies of 10^5 entries and operands of 8 bits; az_evaluate does not call it:
 *
 *   hidden states   --az_quantise_blocks-->  e4m3 codes with one scale for each block of 128
 *   codes, weights  --az_block_matmul----->  logits
 *   logits, rules   --az_token_probs------>  probabilities, best token, its log-probability
 *                     az_adjust_logits       or the logits under the same rules, for a sampler of the caller's
 *
 * Each call is useful by itself: az_block_matmul serves every linear layer, az_token_probs takes the masks of
 * az_legal_masks as they are.  There are no backward passes (the library evaluates, it does not train).
 *
 * Conventions (as in az_eval.h)
 *   - Every function returns AZ_OK (0) or a negative AZ_ERR_* code; nothing throws or aborts.  Arguments are
 *     checked before any CUDA call; a refused call has queued nothing.
 *   - "_dev" pointers are memory of the current device; the stream is one of the current device's.  The caller
 *     owns every buffer.  Calls are asynchronous on the stream, allocate nothing, keep nothing from one call to
 *     the next and share no workspace, so calls on different streams may overlap and each can be captured in a
 *     CUDA graph.
 *   - An output shares no memory with another output or an input, except where a call says so.
 *   - Strides count elements from one row to the next.  A matrix's rows are contiguous in themselves.  Rows of
 *     an output must not overlap.  What lies beyond the stated rows and columns is not written, and not used.
 *   - Zero rows are a no-op.
 */
#ifndef AZ_TOKENS_H
#define AZ_TOKENS_H

#include "az_eval.h"

#ifdef __cplusplus
extern "C" {
#endif

enum { AZ_TYPE_F32 = 0, AZ_TYPE_BF16 = 1, AZ_TYPE_F16 = 2 };

#define AZ_QUANT_BLOCK 128       /* columns (and, for weights, rows) that share a scale */
#define AZ_MAX_VOCAB 262144      /* entries of a row of logits */

/*
 * Numbers -> e4m3 codes with a scale for each block.
 * x_dev: [rows][cols] of x_type.  block_rows 1 (tokens: a block is 128 columns of one row) or 128 (weights: 128 rows
 * x 128 columns).  The last blocks may be partial.
 *   a = max |x| over the block;  s = max(a / 448, 2^-126) in float32;  code = x / s rounded to e4m3
 * where x / s is the real quotient, rounded ONCE to the nearest e4m3 number (ties to the even one), so that the
 * codes do not depend on how a division was carried out.  (A code of zero may carry either sign.)  A block of
 * zeros has s = 2^-126.  A block that holds an infinity or a NaN has that as its scale, so every value that its
 * codes stand for is NaN.
 * codes_dev: [rows][cols] bytes, row stride codes_stride.  scales_dev: [ceil(rows / block_rows)][ceil(cols / 128)]
 * float32, row stride scales_stride.
 * No alignment is asked for beyond the element's own; 16-byte aligned rows are read and written fastest.
 * Errors: BAD_ARG (null pointer, negative size, unknown type, block_rows, a stride smaller than a row, misaligned
 * element), UNSUPPORTED (more than about 2^44 elements), CUDA.  rows == 0 or cols == 0 is a no-op.
 */
int az_quantise_blocks(const void *x_dev, int x_type, int rows, int cols, int64_t x_stride, int block_rows,
                       void *codes_dev, int64_t codes_stride, float *scales_dev, int64_t scales_stride, void *cuda_stream);

/*
 * out[i][j] = sum over blocks c of  a_scales[i][c] * b_scales[j / 128][c] * sum over the block's k of a[i][k] * b[j][k]
 *             (+ bias[j])
 * a_dev: [m][k] e4m3 codes with a scale for 128 columns of a row (az_quantise_blocks, block_rows 1); b_dev: [n][k] e4m3
 * codes with a scale for 128 x 128 (block_rows 128), i.e. a linear layer's weight as [out][in].  bias_dev: [n] float32
 * or NULL.  out_dev: [m][n] of out_type.  Sums are held in float32 and rounded once, when they are stored.  The order of
 * a sum depends on m, n and k only: equal calls give equal bits.
 * A block's two scales are multiplied with each other first, in float32.  Where that product overflows (the largest values of the two
 * blocks have a product above 448^2 x 2^128), the outputs of that row and those 128 columns are infinite or NaN, even where the
 * block's sum is 0; a product below 2^-126 is rounded as a subnormal number, which moves the block's term by up to 2^-125.
 * k need not be a multiple of 128 (the last block is short); rows of a and b start on 16-byte boundaries, i.e. both
 * base addresses and both strides are multiples of 16.  A code of NaN (0x7f, 0xff) makes its outputs NaN.
 * A wait inside the kernel that runs out (none does, short of a fault) is reported by az_tokens_status.
 * Errors: BAD_ARG (null pointer, negative size, k == 0, unknown type, a stride smaller than a row, misaligned operand), UNSUPPORTED (a
 * size above 2^31 - 256, 2^46 outputs or more), CUDA.  m == 0 or n == 0 is a no-op.
 */
int az_block_matmul(const void *a_dev, int64_t a_stride, const float *a_scales_dev, int64_t a_scales_stride,
                    const void *b_dev, int64_t b_stride, const float *b_scales_dev, int64_t b_scales_stride,
                    const float *bias_dev, int m, int n, int k, void *out_dev, int out_type, int64_t out_stride,
                    void *cuda_stream);

/*
 * What changes a row of logits before the choice of a token.  Every part may be absent (NULL).  For token t of row r,
 * in this order, each step rounded to float32:
 *   t in the history:            l = l > 0 ? l / repetition[r] : l * repetition[r]
 *   t n > 0 times in the answer: l = (l - frequency[r] * n) - presence[r]
 *   t in the row's bias list:    l = l + bias (a token listed twice: one after the other, in the list's order)
 *   temperature:                 l = l * (1 / temperature[r])
 *   t not allowed:               l = -infinity, whatever it was
 * The history of row r is tokens[r][0 .. lengths[r]), the first prompt_lengths[r] of it the prompt and the rest the answer
 * so far.  Lengths are clamped to [0, token_room] and prompt lengths to [0, length]; ids outside [0, vocab) are skipped, so a
 * history may hold padding.
 * Bias lists are bias_tokens / bias_values[bias_offsets[r] .. bias_offsets[r + 1]), offsets clamped to [0, bias_count].
 * Allowed tokens: bit (t & 31) of word t >> 5 of the row's mask; bits beyond the vocabulary are ignored.  allowed_stride 0:
 * all rows share one mask.  The 64-bit masks of az_legal_masks are such masks with twice the words (a stride of 60 for the
 * flat head).  repetition and temperature are positive, finite and no subnormal numbers (at least 2^-126: the reciprocal of a smaller
 * temperature is infinite); a row where they are not has unspecified values (what is not allowed stays so).
 */
typedef struct {
    const int32_t *tokens;           /* [rows][token_room], row stride token_stride */
    int64_t token_stride;
    int64_t token_room;              /* at most 2^31 - 1 */
    const int32_t *lengths;          /* [rows]; needed with tokens */
    const int32_t *prompt_lengths;   /* [rows]; NULL: no prompt, all of it is the answer */
    const float *repetition;         /* [rows] */
    const float *presence;           /* [rows] */
    const float *frequency;          /* [rows] */
    const int32_t *bias_offsets;     /* [rows + 1] */
    const int32_t *bias_tokens;      /* [bias_count] */
    const float *bias_values;        /* [bias_count] */
    int64_t bias_count;              /* at most 2^31 - 1 */
    const float *temperature;        /* [rows] */
    const uint32_t *allowed;         /* [rows][allowed_stride] */
    int64_t allowed_stride;          /* in 32-bit words; 0: one mask for all rows */
} az_logit_rules;

/*
 * The logits under the rules: out_dev [rows][vocab] of the same type as logits_dev, rounded once.  out_dev may be logits_dev with
 * the same stride (in place); any other overlap is refused.  rules: a struct in host memory, read during the call; NULL: none.
 * Errors: BAD_ARG (null pointer, negative size, unknown type, a stride smaller than a row, misaligned element, an
 * incomplete rule, overlap), UNSUPPORTED (vocab > AZ_MAX_VOCAB), CUDA.  rows == 0 or vocab == 0 is a no-op.
 */
int az_adjust_logits(const void *logits_dev, int type, int rows, int vocab, int64_t logits_stride,
                     const az_logit_rules *rules, void *out_dev, int64_t out_stride, void *cuda_stream);

/*
 * Probabilities and the best token under the rules.  With l as above BEFORE the division by the temperature T and m its
 * largest value over the allowed tokens of the row:
 *   probs[r][t] = exp((l - m) / T) / sum over allowed u of exp((l_u - m) / T);  exactly 0 where t is not allowed
 *   best[r]     = the lowest t with l = m;     best_logprob[r] = -log(the sum)
 * A row that allows nothing, or only -infinity, has probabilities 0, best -1, best_logprob -infinity.  A NaN among the allowed
 * makes the row's probabilities NaN and is its best token; +infinity gives NaN as the formula does.
 * probs_dev: [rows][vocab] of probs_type, which is AZ_TYPE_F32 or the logits' type, or NULL; it may be logits_dev in place as
 * above.  best_dev: [rows] int32 or NULL; best_logprob_dev: [rows] float32 or NULL; not all three NULL.
 * Errors: as az_adjust_logits.
 */
int az_token_probs(const void *logits_dev, int type, int rows, int vocab, int64_t logits_stride, const az_logit_rules *rules,
                   void *probs_dev, int probs_type, int64_t probs_stride, int32_t *best_dev, float *best_logprob_dev,
                   void *cuda_stream);

/*
 * Status word of the current device's calls of this header (0 = clean).  Synchronises the given stream, so calls queued there or
 * finished elsewhere are covered; what a call still running on another stream raises is left for a later read.  The bits that are
 * returned are cleared, others are not touched.  AZ_ERR_DEVICE_TIMEOUT if a bounded wait ran out: outputs of the calls since the
 * last read are then incomplete.
 */
int az_tokens_status(void *cuda_stream, uint32_t *status_out);

/*
 * Self-test of that report: queues a one-CTA kernel whose wait runs out (after a millisecond) and raises the status bit, as a
 * wait would in the product's kernels (part 0) or in the logit calls' (part 1).  The next az_tokens_status returns
 * AZ_ERR_DEVICE_TIMEOUT, the one after it is clean.  Nothing hangs or traps.  Errors: BAD_ARG (part), CUDA.
 */
int az_selftest_tokens_timeout(int part, void *cuda_stream);

#ifdef __cplusplus
}
#endif
#endif /* AZ_TOKENS_H */
