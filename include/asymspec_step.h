/*
 * asymspec_step.h -- the operators around the decision step, for MI355X
 * (gfx950), in the same library as asymspec.h.
 *
 * Around each call of asymspec_fuse_verify a serving program has work on the
 * same tensors, which these entry points do on the device, so that a step
 * needs no copy to the host:
 *
 *   asymspec_shape_logits   penalties for repeated tokens, biases and grammar
 *                           masks on the logit rows, drafts counted
 *   asymspec_draw_tokens    the drafter's own choice from a row: a token and
 *                           its probability q(d)
 *   asymspec_commit_tokens  the accepted drafts and the emitted token joined
 *                           to the requests' histories, with stop tokens
 *                           and length limits
 *   asymspec_plan_slots     block tables grown from and trimmed to a ring of
 *                           free blocks, and the cache slot of every new
 *                           token, from the requests' lengths
 *
 * Conventions: those of asymspec.h (caller-owned device pointers, nothing
 * allocated or retained, asynchronous on `stream`, negative status codes with
 * nothing enqueued, host checks first).  Unlike the decision step these calls
 * may be captured into a HIP graph and replayed.  No workgroup waits for
 * another one.  Values that the host cannot see (token ids, lengths, block
 * counts, mask rows) may hold anything: what is out of range is left out as
 * stated below, and never read or written out of bounds.
 */
#ifndef ASYMSPEC_STEP_H
#define ASYMSPEC_STEP_H

#include "asymspec.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ---- penalties, biases and masks ---------------------------------------- */

#define ASYMSPEC_SHAPE_MAX_ROWS 64        /* R                              */
#define ASYMSPEC_SHAPE_MAX_BIAS 1023      /* bias entries of a request      */
#define ASYMSPEC_SHAPE_MAX_HISTORY 1048575 /* tokens of a history            */

/*
 * Row r of request b holds the logits behind the request's history h and its
 * first D - (R - 1) + r drafts.  With, for a token x,
 *   c      how often x stands in h[prompt_length .. length) and those drafts,
 *   seen   whether c > 0 or x stands in h[0 .. prompt_length),
 * its logit v becomes, in fp32, each step rounded and rounded once more to the
 * storage type at the end:
 *   seen:           v = v > 0 ? v / repetition : v * repetition
 *   c > 0:          v = (v - frequency * c) - presence
 *   x has a bias:   v = v + bias
 *   x is masked:    v = -inf
 * A logit with none of these keeps its bits.
 */
typedef struct asymspec_shape {
  const void* logits;            /* [B][R][V] (dtype); a row is contiguous, rows and requests
                                    are row_stride and request_stride elements apart        */
  void* out;                     /* the same for out_row_stride, out_request_stride.  Either
                                    `logits` itself with the same strides (in place: only
                                    16-byte pieces that change are read or written), or
                                    memory that begins behind its end or ends ahead of it
                                    (all rows are written).  Rows of `out` lie apart         */
  int64_t request_stride, row_stride;
  int64_t out_request_stride, out_row_stride;
  const int32_t* history;        /* [B][max_history], or NULL: no history                    */
  const int32_t* lengths;        /* [B] tokens of each history (clamped to [0, max_history])  */
  const int32_t* prompt_lengths; /* [B], or NULL: 0.  Tokens ahead of it are seen, not counted */
  const int32_t* draft_tokens;   /* [B][D], requests draft_stride elements apart, or NULL: D = 0 */
  int64_t draft_stride;
  const int32_t* id_map;         /* [n_ids], or NULL: history and draft tokens are ids of another
                                    vocabulary; id_map[x] is the id here (out of range: none)  */
  const float* repetition;       /* [B], or NULL: 1; positive                                 */
  const float* frequency;        /* [B], or NULL: 0                                           */
  const float* presence;         /* [B], or NULL: 0                                           */
  const int32_t* bias_ids;       /* [B][n_bias], ids out of range are unused entries; of several
                                    entries with one id the last counts; or NULL: n_bias = 0   */
  const float* bias_values;      /* [B][n_bias]                                               */
  const uint32_t* mask;          /* [n_masks][ceil(V / 32)]: bit x % 32 of word x / 32 is set where
                                    token x is allowed; or NULL                               */
  const int32_t* mask_index;     /* [B][R]: the row of `mask`; out of range: no mask          */
  int32_t dtype;                 /* ASYMSPEC_BF16 or ASYMSPEC_FP32                            */
  int32_t B, R, V;               /* B >= 1, R in [1, 64], V in [1, 2^30); B * ceil(V / 8192)
                                    below 2^23 - 1                                            */
  int32_t max_history;           /* row length of `history`; at most 1048575                  */
  int32_t D;                     /* 0, or in [R - 1, 64]                                       */
  int32_t n_ids;                 /* length of id_map                                          */
  int32_t n_bias;                /* at most 1023                                              */
  int32_t n_masks;
} asymspec_shape;

/* Token ids outside [0, V) (after id_map) are left out.  Arrays are 4-byte
 * aligned, bf16 logits 2-byte.  A row whose mask allows nothing becomes -inf
 * throughout.  Returns ASYMSPEC_OK or a negative status. */
int asymspec_shape_logits(const asymspec_shape* shape, void* stream);

/* ---- a draw from each row ----------------------------------------------- */

/*
 * token and prob of N rows of V logits, rows row_stride elements apart.
 *   temperature[n] <= 0 (or not a number): the lowest index of the row's
 *     largest logit, prob 1;
 *   temperature[n] > 0: with w(x) = exp((l(x) - max l) / temperature) in fp64,
 *     the first token whose inclusive sum of w exceeds uniforms[n] times the
 *     row's sum, and prob = w(token) / sum: an inverse-CDF draw from
 *     softmax(l / temperature), as the drafter makes it for fuse_verify.
 * Logits of -inf or not a number have no weight, as has one whose w(x) would be
 * below fp64's smallest number, 2^-1074; logits of +inf share all of it.  A row
 * without any weight gives token 0 with prob 0.  Uniforms are in [0, 1); below
 * (or not a number) count as 0, at or above 1 give the last token with weight.
 * The same inputs give the same outputs, bit for bit.
 *   logits       (dtype), aligned to an element
 *   uniforms     [N], entries uniform_stride elements apart (may be NULL when
 *                no temperature is positive: then a draw takes 0)
 *   token        [N] out, token_stride elements apart
 *   prob         [N] out, prob_stride elements apart; or NULL
 *   workspace    >= asymspec_draw_workspace_size bytes, 16-byte aligned;
 *                needs no initialisation; calls that may run at the same time
 *                (replays of a captured one among them) need distinct ones.  A
 *                draw leaves anything there, so memory that asymspec_fuse_verify
 *                works in is cleared in between (asymspec_workspace_clear)
 * The outputs and the workspace overlap no other array.  N >= 1, 1 <= V < 2^30,
 * N * ceil(V / 1024) below 2^26 - 4 (a size of 0 bytes says that a shape is not
 * valid).
 */
size_t asymspec_draw_workspace_size(int N, int V, int dtype);
int asymspec_draw_tokens(const void* logits, int dtype, int N, int V, int64_t row_stride,
                         const float* temperature, const float* uniforms, int64_t uniform_stride,
                         int32_t* token, int64_t token_stride, float* prob, int64_t prob_stride,
                         void* workspace, size_t workspace_bytes, void* stream);

/* ---- committed tokens ---------------------------------------------------- */

/*
 * Joins to each history what a step committed: draft_tokens[b][0 .. accept_len)
 * and next_token[b], cut behind the first stop token and at the request's
 * limit.  A request that is finished, or whose accept_len is not in [0, K]
 * (-1: its decision did not complete), commits nothing.
 *   draft_tokens   [B][K], requests draft_stride elements apart (NULL when K = 0)
 *   history        [B][max_history], in place: the committed tokens are written
 *                  at lengths[b], nothing else changes
 *   lengths        [B] (a length outside [0, max_history] commits nothing)
 *   finished       [B], nonzero: finished; or NULL: none
 *   stop_tokens    [n_stop], or NULL when n_stop = 0
 *   max_lengths    [B] limit of each history's length, or NULL: max_history
 *                  (limits are clamped to [0, max_history])
 *   lengths_out    [B] out: the new lengths
 *   finished_out   [B] out: 1 where the request was finished, committed a stop
 *                  token, or (with accept_len in [0, K]) is at its limit; else 0
 *   tokens_out     [B][K + 1] out: the committed tokens, then -1
 *   counts_out     [B] out: how many
 * The outputs overlap one another and the inputs nowhere, except that
 * lengths_out may be lengths and finished_out finished.  1 <= B < 2^26 - 4,
 * 0 <= K <= 63.
 */
int asymspec_commit_tokens(const int32_t* accept_len, const int32_t* next_token,
                           const int32_t* draft_tokens, int64_t draft_stride,
                           int32_t* history, int max_history, const int32_t* lengths,
                           const int32_t* finished, const int32_t* stop_tokens, int n_stop,
                           const int32_t* max_lengths, int B, int K,
                           int32_t* lengths_out, int32_t* finished_out,
                           int32_t* tokens_out, int32_t* counts_out, void* stream);

/* ---- cache slots ---------------------------------------------------------- */

#define ASYMSPEC_SLOTS_MAX_REQUESTS 4096

/*
 * A paged cache keeps position p of request b in slot
 *   block_table[b][p / block_size] * block_size + p % block_size.
 * The call makes room for each request's next tokens: request b has
 * lengths[b] positions and gets new_tokens[b] more, so it needs
 * ceil((lengths[b] + new_tokens[b]) / block_size) blocks (none with
 * release[b], which also has no new tokens).
 *   - Missing blocks are taken from the free ring in the order of the
 *     requests, blocks beyond the need go back behind its end in the order of
 *     the requests and of their tables (those beyond the ring's size are
 *     dropped).  Blocks given back in a call are not taken in the same call.
 *   - A request that needs more than max_blocks, or whose blocks together with
 *     those of the requests before it are more than are free, is short: its
 *     table and count stay as they are and it gets no slots.
 *   lengths        [B]; negative counts as 0
 *   new_tokens     [B], or NULL: `width` for every request; negative counts as
 *                  0, and with width > 0 more than `width` counts as `width`
 *   release        [B], nonzero: give all blocks back; or NULL
 *   block_table    [B][max_blocks] in place: entries taken are written, entries
 *                  given back become -1, all others stay
 *   n_blocks       [B]: blocks that each request holds (clamped to [0, max_blocks])
 *   free_ring      [ring_size] in place; free_state [2]: the ring's first free
 *                  entry (modulo ring_size) and how many there are (clamped to
 *                  [0, ring_size]).  A ring as large as the pool never overflows
 *   width, total   width > 0: slots is [B][width], request b's j-th new token in
 *                  row b; width = 0: slots is [total], the requests' tokens one
 *                  behind the other.  Places with no token hold -1
 *   slots          out
 *   starts         [B + 1] out or NULL: where each request's tokens begin when
 *                  they lie one behind the other, and their number (at most
 *                  2^31 - 1)
 *   short_out      [B] out: 1 where the request is short, else 0
 *   n_blocks_out   [B] out; free_state_out [2] out.  Neither is its input
 * What the call writes (block_table and free_ring among it) overlaps no other of
 * its arrays (checked: ASYMSPEC_E_ARG).  1 <= B <= 4096, block_size >= 1,
 * max_blocks >= 1, ring_size >= 1, B * max_blocks, B * width and ring_size below
 * 2^31; with width = 0, total >= 1 and new_tokens is given.
 */
int asymspec_plan_slots(const int32_t* lengths, const int32_t* new_tokens, const int32_t* release,
                        int32_t* block_table, int max_blocks, const int32_t* n_blocks,
                        int32_t* free_ring, int ring_size, const int32_t* free_state,
                        int block_size, int B, int width, int total,
                        int64_t* slots, int32_t* starts, int32_t* short_out,
                        int32_t* n_blocks_out, int32_t* free_state_out, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* ASYMSPEC_STEP_H */
