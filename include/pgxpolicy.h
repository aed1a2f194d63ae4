/*
 * pgxpolicy.h -- C ABI of the step between a policy's logits and the actions of the games (gfx950).
 *
 * The environments of this library (pgxgo.h, pgxhex.h) give a legal mask and take actions; these entry points turn the
 * logits that a model has for the actions into adjusted logits (pgxpolicy_logits), into moves (pgxpolicy_sample), and into
 * the loss and gradient that a learner of recorded moves needs (pgxpolicy_loss).
 *
 * Conventions are those of pgxgo.h: pointers named *_dev are device pointers owned by the caller, work is enqueued on
 * the given stream and is asynchronous, every function returns PGXPOLICY_OK or a negative code, nothing throws, aborts,
 * allocates or synchronises.  Nothing is kept between calls.  Rows of inputs may overlap (pitch 0: one row for all games),
 * rows of outputs may not.  Adjusted logits and gradients may take the place of logits of their type and pitch.
 *
 * Adjusted logits.  For row b (a game) and action a, in 32-bit floating point, every operation rounded by itself (a quotient
 * below 2^-100 may differ in its last bit):
 *     z = logits[b][a]
 *     c = how often a occurs among record[b][t], max(begin[b], 0) <= t < min(end[b], record_len)      (0 without a record)
 *     if c > 0:  z = z > 0 ? z / repetition : z * repetition
 *     z = z - frequency * c;   if c > 0:  z = z - presence
 *     z = z + bias[b][a]
 *     z = z / T,  T = temperature[b], or 1 where that is not above 0
 *     z = -infinity where mask[b][a] == 0, whatever the logit, bias and record hold there
 * An action is possible where z > -infinity (so neither masked nor NaN).  Entries of the record outside [0, actions), such
 * as the -1 of a game that did not move, count for nothing.  A temperature that is not above 0 means greedy play: no noise
 * in pgxpolicy_sample, and T = 1.  +infinity in a possible place makes the row's probabilities NaN.
 */
#ifndef PGXPOLICY_H_
#define PGXPOLICY_H_

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define PGXPOLICY_OK 0
#define PGXPOLICY_EINVAL (-1) /* null pointer, size or pitch out of range (also rows of 2^32 threads: 16 to a row of up to 384 actions, 64 up to 2048, then 256), unknown type, repetition not above 0 */
#define PGXPOLICY_EHIP (-2)   /* a HIP runtime call failed; see pgxpolicy_last_hip_error() */

#define PGXPOLICY_F32 0
#define PGXPOLICY_F16 1
#define PGXPOLICY_BF16 2

#define PGXPOLICY_MAX_ACTIONS 8192
#define PGXPOLICY_MAX_RECORD 65535

/* What is done to the logits.  All zero means nothing (repetition and temperature 0 stand for 1). */
typedef struct {
  const uint8_t* mask_dev;     /* [rows][mask_pitch] bytes, non-zero = legal (what pgxgo_legal_mask writes); NULL: all legal */
  int64_t mask_pitch;
  const float* bias_dev;       /* [rows][bias_pitch], in elements; NULL: none */
  int64_t bias_pitch;
  const int32_t* record_dev;   /* move t of row b at [b * record_row_stride + t * record_ply_stride]; NULL: none */
  int64_t record_row_stride, record_ply_stride;   /* a recorded trajectory [plies][games] has strides 1 and games */
  int32_t record_len;          /* plies in the record, at most PGXPOLICY_MAX_RECORD */
  float repetition, frequency, presence;
  const int32_t* begin_dev;    /* [rows]; NULL: 0 */
  const int32_t* end_dev;      /* [rows]; NULL: record_len */
  const float* temperature_dev; /* [rows]; NULL: `temperature` for all rows */
  float temperature;           /* above 0, or 0 for 1 */
} pgxpolicy_adjust;

/* out_dev[b][a] = z (float32, pitch in elements), or with normalize != 0 its log-probability z - log sum exp z over the
 * possible actions, -infinity elsewhere.  logits_dev: `type`, pitch in elements.  adjust may be NULL. */
int pgxpolicy_logits(int32_t rows, int32_t actions, const void* logits_dev, int32_t type, int64_t logits_pitch, const pgxpolicy_adjust* adjust,
                     int32_t normalize, float* out_dev, int64_t out_pitch, void* stream);

/* actions_dev[b] = the possible action with the largest z + noise[b][a] (in 32 bits; the lowest index among equals), and
 * logp_dev[b] (may be NULL) its log-probability under softmax(z).  noise_dev: float32, pitch in elements, NULL: none; with
 * Gumbel noise, -log(-log u), the action is a draw from softmax(z).  Noise that is NaN counts as -infinity.
 * A row without possible actions gets action -1, which the environments' step calls leave untouched, and log-probability 0. */
int pgxpolicy_sample(int32_t rows, int32_t actions, const void* logits_dev, int32_t type, int64_t logits_pitch, const pgxpolicy_adjust* adjust,
                     const float* noise_dev, int64_t noise_pitch, int32_t* actions_dev, float* logp_dev, void* stream);

/* With p = softmax(z) over the possible actions and y the target:
 *     entropy[b] = -sum p log p
 *     loss[b]    = -weight[b] * sum y log p - entropy_bonus * entropy[b]
 *     grad[b][a] = grad_scale * d loss[b] / d logits[b][a]       (type and rounding of the logits; 0 where not possible)
 * The target is either target_dev, float32 [rows][target_pitch] (a search's visit shares; need not add up to one), or
 * taken_dev, int32 [rows]: one move each (a played move; weight is then its advantage).  Target shares of impossible actions, and a
 * move outside [0, actions), count for nothing.  weight_dev NULL: 1.  loss_dev and entropy_dev may be NULL.  A row without
 * possible actions has loss, entropy and gradient 0.  The gradient takes record, bias, mask and temperature as constants. */
int pgxpolicy_loss(int32_t rows, int32_t actions, const void* logits_dev, int32_t type, int64_t logits_pitch, const pgxpolicy_adjust* adjust,
                   const float* target_dev, int64_t target_pitch, const int32_t* taken_dev, const float* weight_dev, float entropy_bonus, float grad_scale,
                   float* loss_dev, float* entropy_dev, void* grad_dev, int64_t grad_pitch, void* stream);

const char* pgxpolicy_strerror(int code);
int pgxpolicy_last_hip_error(void); /* hipError_t of the most recent PGXPOLICY_EHIP on this thread, else 0 */

#ifdef __cplusplus
}
#endif
#endif /* PGXPOLICY_H_ */
