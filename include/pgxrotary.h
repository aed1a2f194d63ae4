/*
 * pgxrotary.h -- C ABI of rotary positions for policies that read a game as its sequence of moves (gfx950).
 *
 * Before queries and keys go into attention (pgxcache.h) they are turned by their token's position, so that their product depends on how far apart
 * two moves are.  Conventions are those of pgxgo.h: pointers named *_dev are device pointers owned by the caller, work is enqueued on the given
 * stream and is asynchronous, every function returns PGXROTARY_OK or a negative code, nothing throws, aborts, allocates or synchronises.  Nothing is
 * kept between calls.
 */
#ifndef PGXROTARY_H_
#define PGXROTARY_H_

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define PGXROTARY_OK 0
#define PGXROTARY_EINVAL (-1) /* null or misaligned pointer, size out of range, unknown type, output rows that overlap each other or other tensors' rows */
#define PGXROTARY_EHIP (-2)   /* a HIP runtime call failed; see pgxrotary_last_hip_error() */

#define PGXROTARY_F32 0
#define PGXROTARY_F16 1
#define PGXROTARY_BF16 2

#define PGXROTARY_MAX_HEAD_DIM 1024
#define PGXROTARY_MAX_PARTS 2

/* One tensor, such as the queries or the keys: element [i][t][head][.] at i * entry_stride + t * token_stride + head * head_stride, in elements.
 * out_dev may be in_dev with the same strides.  Otherwise no output shares memory with an input or an output of either tensor (rows that lie between each other's, as views of one
 * product do, are apart), and rows of an output may not overlap each other: such calls are refused. */
typedef struct {
  const void* in_dev;
  int64_t in_entry_stride, in_token_stride, in_head_stride;
  void* out_dev;
  int64_t out_entry_stride, out_token_stride, out_head_stride;
  int32_t heads;
} pgxrotary_part;

/* For every entry i, token t and head, with p = positions[i][t], the first rotary_dim = R elements x of the head become
 *     a = p * frequencies_dev[j],  c = magnitude cos a,  s = magnitude sin a  (inverse != 0: s = -magnitude sin a),   0 <= j < R / 2
 *     x'[u] = x[u] c - x[w] s,   x'[w] = x[w] c + x[u] s,       u, w = j, j + R / 2,  or with interleaved != 0  2 j, 2 j + 1
 * and the others are copied.  inverse gives the gradient: d loss / d x from d loss / d x'.  The angle is formed and reduced as two 64-bit numbers (every
 * position keeps its own to 2^-23 in 32 bits, while it turns less than 2^51 times), its cosine and sine and the products are in 32, rounded once to the type.
 * positions_dev: int32, element [i][t] at i * entry_stride + t * token_stride; they may repeat (stride 0).  frequencies_dev: float64 [R / 2], radians per position. */
int pgxrotary_turn(int32_t entries, int32_t tokens, int32_t head_dim, int32_t rotary_dim, int32_t type, const int32_t* positions_dev, int64_t positions_entry_stride,
                   int64_t positions_token_stride, const double* frequencies_dev, float magnitude, int32_t interleaved, int32_t inverse, int32_t parts,
                   const pgxrotary_part* part, void* stream);

const char* pgxrotary_strerror(int code);
int pgxrotary_last_hip_error(void); /* hipError_t of the most recent PGXROTARY_EHIP on this thread, else 0 */

#ifdef __cplusplus
}
#endif
#endif /* PGXROTARY_H_ */
