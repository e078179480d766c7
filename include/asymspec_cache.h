/*
 * asymspec_cache.h -- a paged cache of keys and values in 8 or 4 bits, for
 * MI355X (gfx950), in the same library as asymspec.h.
 *
 * asymspec_plan_slots (asymspec_step.h) says where a step's tokens go in a paged
 * cache; these entry points fill the slots and answer from them:
 *
 *   asymspec_rotate_heads   rotary positions on the queries and keys of a
 *                           step's tokens
 *   asymspec_write_cache    their keys and values into the slots, quantised
 *   asymspec_read_cache     positions of each request back as dense tensors
 *   asymspec_attend_cache   attention of a step's rows over the cache
 *
 * Conventions: those of asymspec_step.h (caller-owned device pointers, nothing
 * allocated or retained, asynchronous on `stream`, negative status codes with
 * nothing enqueued, host checks first; calls may be captured into a HIP graph).
 * No workgroup waits for another one.  Values that the host cannot see (slots,
 * block tables, lengths) may hold anything: what is out of range is left out as
 * stated below, and never read or written out of bounds.
 */
#ifndef ASYMSPEC_CACHE_H
#define ASYMSPEC_CACHE_H

#include "asymspec.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ---- the cache ----------------------------------------------------------- */

#define ASYMSPEC_CACHE_MAX_DIM 256

/*
 * Slot s of a head is row ((s / block_size) * heads + head) * block_size +
 * s % block_size of four arrays, 16-byte aligned: `dim` values of a key (and of a
 * value) in 8 or 4 bits each, and a scale byte for each 32 of them.  With 8 bits
 * a code is an e4m3 number, with 4 an e2m1 number (sign, two bits of exponent,
 * one of mantissa: 0 0.5 1 1.5 2 3 4 6), the even channel in the low half of its
 * byte.  A scale byte s stands for 2^(s - 127); one above 246 (8 bits) or 252 (4
 * bits), 255 where it is written here, says that the 32 values are not all finite:
 * each of them reads as not a number.
 */
typedef struct asymspec_cache {
  void* keys;          /* [blocks][heads][block_size][dim * bits / 8]            */
  void* key_scales;    /* [blocks][heads][block_size][dim / 32]                  */
  void* values;        /* as keys                                                */
  void* value_scales;  /* as key_scales                                          */
  int32_t blocks;      /* >= 1; blocks * heads * block_size below 2^31            */
  int32_t heads;       /* >= 1                                                   */
  int32_t block_size;  /* >= 1                                                   */
  int32_t dim;         /* a multiple of 32, at most 256                          */
  int32_t bits;        /* 8 or 4                                                 */
} asymspec_cache;

/* A tensor [B][R][heads][dim]: a head's channels are contiguous, the others lie
 * `request`, `row` and `head` elements apart (none negative). */
typedef struct asymspec_heads {
  void* at;
  int64_t request, row, head;
} asymspec_heads;

/* ---- rotary positions ------------------------------------------------------ */

/*
 * Turns pairs of channels of each head by their token's position.  With
 * p the position, f_i = frequencies[i] (radians a position) and the pair (x, y) of
 * channels (i, i + n), or (2i, 2i + 1) where interleaved:
 *   x' = magnitude * (x cos(p f_i) - y sin(p f_i))
 *   y' = magnitude * (x sin(p f_i) + y cos(p f_i))
 * Angles are fp64; sines and cosines are fp32 numbers, two units off at most (small
 * ones too); the products and sums are fp32 and rounded once to the storage type.
 * Channels from 2n on stay as they are.
 *   q, k         [B][R][q_heads][dim] and [B][R][k_heads][dim] (dtype, aligned to
 *                an element); k_heads = 0: no k
 *   q_out, k_out the same shapes; each either its input with the same strides, or
 *                memory apart from all others.  Rows of an output lie apart
 *   positions    [B]: token r of request b stands at positions[b] + r; or, with
 *                every_row, [B][R].  Any value; a negative one turns back
 *   frequencies  [n] fp64, 8-byte aligned; n in [1, dim / 2]
 * dim in [2, 1024], B, R, q_heads >= 1, q_heads + k_heads at most 4096, B * R below
 * 2^24.
 */
typedef struct asymspec_rotate {
  asymspec_heads q, k, q_out, k_out;
  const int32_t* positions;
  const double* frequencies;
  float magnitude;
  int32_t every_row, interleaved;
  int32_t dtype;                 /* ASYMSPEC_BF16 or ASYMSPEC_FP32 */
  int32_t B, R, q_heads, k_heads, dim, n;
} asymspec_rotate;

int asymspec_rotate_heads(const asymspec_rotate* rotate, void* stream);

/* ---- keys and values into their slots -------------------------------------- */

/*
 * Writes the key and the value of token r of request b to slots[b][r].  For each
 * 32 channels with a largest magnitude m, the scale is the smallest power of
 * two, 2^-100 at least, with m <= 448 * scale (8 bits) or m <= 6 * scale (4 bits),
 * and each code the nearest to x / scale, ties to the even code: a result that
 * does not depend on how it is computed.  Where one of the 32 is not finite, or
 * of a magnitude beyond 1.75 * 2^127 (8 bits) or 1.5 * 2^127 (4 bits), the scale byte
 * is 255 and the codes are 0.
 *   k, v    [B][R][heads][dim] (dtype, aligned to an element)
 *   slots   [B][R]; out of [0, blocks * block_size): the token is left out.
 *           The slots of a call are distinct (one given twice holds a mix)
 * Nothing else in the cache changes.  B, R >= 1; heads at most 4096;
 * ceil(B * R / floor(2048 / dim)) * heads below 2^24.
 */
int asymspec_write_cache(const asymspec_cache* cache, const asymspec_heads* k, const asymspec_heads* v, int dtype,
                         const int64_t* slots, int B, int R, void* stream);

/* ---- positions as dense tensors --------------------------------------------- */

/*
 * Position p of request b is in slot block_table[b][p / block_size] * block_size +
 * p % block_size.  Gives each request's positions first[b] .. first[b] + width as
 * [B][width][heads][dim] (dtype; a code times its scale is exact in both).  A
 * position outside [0, lengths[b]), outside the table or in a block outside
 * [0, blocks) gives zeros.
 *   first   [B] or NULL: 0
 *   k, v    out, contiguous, 16-byte aligned; either may be NULL
 * B, width, max_blocks >= 1; heads at most 4096; B * ceil(width /
 * floor(2048 / dim)) * heads below 2^24.
 */
int asymspec_read_cache(const asymspec_cache* cache, const int32_t* block_table, int max_blocks, const int32_t* lengths,
                        const int32_t* first, int dtype, int B, int width, void* k, void* v, void* stream);

/* ---- attention over the cache ------------------------------------------------ */

#define ASYMSPEC_ATTEND_MAX_REQUESTS 4096
#define ASYMSPEC_ATTEND_MAX_ROWS 64
#define ASYMSPEC_ATTEND_COUNTERS 524288   /* bytes at a workspace's start  */

/*
 * Row r of request b stands at position p = lengths[b] + r (the lengths and
 * new_tokens that plan_slots takes), and sees the positions in (p - window, p] (with
 * window 0: up to p) that lie in its table and in a block of the cache.  Query head
 * h reads head h / (q_heads / heads) of the cache.  With t = scale * (q . key) over
 * the positions seen:
 *   out = sum(exp(t) value) / sum(exp(t)),   lse = log(sum(exp(t)))
 * A row that sees nothing, and a row r >= new_tokens[b], is 0 with lse -inf.
 * Scores, statistics and sums are fp32; a probability is split into bf16 parts
 * whose sum is within 2^-17 of it (bf16) or 2^-24 (fp32), an fp32 query likewise.
 * Sums hold up to 2^8 times each value, and overflow where that is beyond fp32.
 * A position that is not seen has no effect, whatever it holds.  The same inputs
 * give the same outputs, bit for bit.
 *   q            [B][R][q_heads][dim] (dtype, aligned to an element)
 *   out          [B][R][q_heads][dim] contiguous, 16-byte aligned
 *   lse          [B][R][q_heads] contiguous, or NULL
 *   block_table  [B][max_blocks]; lengths [B] (negative counts as 0, more than
 *                2^31 - 256 as that); new_tokens [B] (clamped to [0, R]), or NULL: R
 *   window       0 or more
 *   workspace    >= asymspec_attend_workspace_size bytes, 16-byte aligned.  Its
 *                first ASYMSPEC_ATTEND_COUNTERS bytes are zero before its first use
 *                (for a single call the first 128 * max(2048, B * heads * ceil(R *
 *                q_heads / heads / 16)) of them are enough), and each call leaves them so
 *                for the next one, of any shape.  Calls that may run at the same time
 *                (replays of captured ones among them) need distinct ones.  (What
 *                workgroups leave for each other lies on whole lines of 128 bytes in
 *                it, wherever it begins: the size has room for that)
 * The outputs and the workspace overlap no other array.  dim is 64, 96, 128, 192
 * or 256; 1 <= B <= 4096, 1 <= R <= 64; q_heads is a multiple of the cache's
 * heads, at most 64 times as many; max_blocks >= 1, max_blocks * block_size below
 * 2^31 - 256, and n = B * heads * ceil(R * q_heads / heads / 16) at most
 * 2^17, n * (max_blocks * block_size / 128 + 2) below 2^31.
 */
typedef struct asymspec_attend {
  asymspec_cache cache;
  asymspec_heads q;
  void* out;
  float* lse;
  const int32_t* block_table;
  const int32_t* lengths;
  const int32_t* new_tokens;
  float scale;
  int32_t window;
  int32_t dtype;
  int32_t B, R, q_heads, max_blocks;
} asymspec_attend;

/* 0 for sizes that are not valid; of `attend` only sizes and types are read. */
size_t asymspec_attend_workspace_size(const asymspec_attend* attend);
int asymspec_attend_cache(const asymspec_attend* attend, void* workspace, size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* ASYMSPEC_CACHE_H */
