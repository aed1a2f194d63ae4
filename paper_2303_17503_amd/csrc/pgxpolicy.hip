// pgxpolicy.hip -- from a policy's logits to actions, and the learner's loss with its gradient (include/pgxpolicy.h), gfx950.
//
// A row (a game's logits) is held in the registers of G lanes, 8 consecutive actions per lane and chunk, so that every input is
// read once and everything that needs the row's maximum and sum follows without a second pass.  All three calls are bound by the
// bytes they move; 16 lanes per row (rather than the wavefront) let a row's reductions run on four rows at once by DPP rotations
// inside the 16-lane rows, and 3 chunks x 16 lanes x 8 hold the 362 actions of 19x19 with 6 % of the lanes' slots idle.
//
// Measured: the loss of 65536 x 362 logits in bfloat16 26.0 us, 4.6 TB/s of what it has to move; 16384 x 122 log-probabilities 5.3 us; sampling of
// 65536 x 362 with records of up to 361 plies, [plies][games], 75 us, 3.3 TB/s (vector instructions keep 60 % of the time busy, and waves
// that wait for moves the rest: blocks of 8, 32 and 64 rows instead of 16 take 82, 85 and 104 us).
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>
#include <stdlib.h>

#include <type_traits>

#include "pgxpolicy.h"

namespace {

thread_local int g_last_hip = 0;

#define HIPCHK(expr)                                   \
  do {                                                 \
    hipError_t e_ = (expr);                            \
    if (e_ != hipSuccess) {                            \
      g_last_hip = (int)e_;                            \
      return PGXPOLICY_EHIP;                           \
    }                                                  \
  } while (0)

constexpr float kNone = -INFINITY;
constexpr int kThreads = 256;

enum Op { kLogits, kSample, kLossShares, kLossMoves };

struct Args {
  const void* logits;
  int64_t logits_pitch;
  const uint8_t* mask;
  int64_t mask_pitch;
  const float* bias;
  int64_t bias_pitch;
  const int32_t* record;
  int64_t record_row, record_ply;
  const int32_t *begin, *end;
  const float* temperature_row;
  const float* second;      // noise, or the target shares
  int64_t second_pitch;
  const int32_t* taken;
  const float* weight;
  void* out;                // adjusted logits, actions, or the gradient
  int64_t out_pitch;
  float *row_out, *row_out2;   // log-probability; loss, entropy
  int32_t rows, actions, record_len, normalize, record_by_row, record_near, by_die;
  float repetition, frequency, presence, temperature, entropy_bonus, grad_scale;
};

// ---- loads and stores of 8 consecutive elements at any alignment the element type has ----------------------------------------
// (rows of 82 or 362 elements start on no particular boundary; the target takes vector accesses at any address)
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef u32x4 u32x4_2 __attribute__((aligned(2)));
typedef u32x2 u32x2_1 __attribute__((aligned(1)));
typedef f32x4 f32x4_4 __attribute__((aligned(4)));

struct F32 {
  typedef float type;
  static __device__ __forceinline__ void load8(const type* p, float* x) {
    const f32x4 a = *(const f32x4_4*)p, b = *(const f32x4_4*)(p + 4);
#pragma unroll
    for (int j = 0; j < 4; ++j) { x[j] = a[j]; x[4 + j] = b[j]; }
  }
  static __device__ __forceinline__ void store8(type* p, const float* x) {
    *(f32x4_4*)p = f32x4{x[0], x[1], x[2], x[3]};
    *(f32x4_4*)(p + 4) = f32x4{x[4], x[5], x[6], x[7]};
  }
};
template <class H>
struct Half {
  typedef H type;
  typedef H h8 __attribute__((ext_vector_type(8)));
  static __device__ __forceinline__ void load8(const type* p, float* x) {
    const u32x4 w = *(const u32x4_2*)p;
    const h8 h = __builtin_bit_cast(h8, w);
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = (float)h[j];
  }
  static __device__ __forceinline__ void store8(type* p, const float* x) {   // to nearest, ties to even
    h8 h;
#pragma unroll
    for (int j = 0; j < 8; ++j) h[j] = (H)x[j];
    *(u32x4_2*)p = __builtin_bit_cast(u32x4, h);
  }
};
typedef Half<_Float16> F16;
typedef Half<__bf16> BF16;

// The chunk of 8 actions that begins at action `at` of a row of `actions` >= 8: read 8 from `base`, of which those from `skip` on count.
// The row's last chunk is moved back so that it ends with the row; what it shares with the chunk before it is computed alike in
// both, counts once in sums, and is written twice with the same value.
struct Chunk {
  int at, base, skip;
  __device__ __forceinline__ Chunk(int index, int actions) {
    at = index * 8;
    base = min(at, max(actions - 8, 0));
    skip = at - base;
  }
};
template <class T>
__device__ __forceinline__ void load_chunk(const typename T::type* row, const Chunk& k, int actions, float* x) {
  if (actions >= 8) {
    T::load8(row + k.base, x);
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = (float)row[min(j, actions - 1)];
  }
}
template <class T>
__device__ __forceinline__ void store_chunk(typename T::type* row, const Chunk& k, int actions, const float* x) {
  if (actions >= 8) {
    if (k.at < actions) T::store8(row + k.base, x);
  } else if (k.at == 0) {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (j < actions) row[j] = (typename T::type)x[j];
  }
}
__device__ __forceinline__ void load_mask(const uint8_t* row, const Chunk& k, int actions, uint32_t* m) {   // m[0], m[1]: bytes
  if (actions >= 8) {
    const u32x2 w = *(const u32x2_1*)(row + k.base);
    m[0] = w[0];
    m[1] = w[1];
  } else {
    m[0] = m[1] = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) m[j >> 2] |= (uint32_t)row[min(j, actions - 1)] << (8 * (j & 3));
  }
}

// ---- reductions over the G lanes of a row; every lane gets the result -----------------------------------------------------------
template <int ROT>
__device__ __forceinline__ uint32_t rotated(uint32_t x) {   // within each 16 lanes
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x120 + ROT, 0xF, 0xF, false);
}
template <int ROT>
__device__ __forceinline__ float rotated(float x) { return __uint_as_float(rotated<ROT>(__float_as_uint(x))); }

struct Sum { static __device__ __forceinline__ float of(float a, float b) { return a + b; } };
struct Max { static __device__ __forceinline__ float of(float a, float b) { return fmaxf(a, b); } };

template <class F, int G>
__device__ __forceinline__ float reduced(float x, float* shared) {
  x = F::of(x, rotated<8>(x));
  x = F::of(x, rotated<4>(x));
  x = F::of(x, rotated<2>(x));
  x = F::of(x, rotated<1>(x));
  if (G >= 64) {
    x = F::of(x, __shfl_xor(x, 16));
    x = F::of(x, __shfl_xor(x, 32));
  }
  if (G > 64) {   // the block has one row
    if ((threadIdx.x & 63) == 0) shared[threadIdx.x >> 6] = x;
    __syncthreads();
    x = shared[0];
#pragma unroll
    for (int w = 1; w < G / 64; ++w) x = F::of(x, shared[w]);
    __syncthreads();
  }
  return x;
}
// the larger score; among equals the lower index
__device__ __forceinline__ void better(float& score, int& index, float s, int i) {
  const bool take = s > score || (s == score && i < index);
  score = take ? s : score;
  index = take ? i : index;
}
template <int G>
__device__ __forceinline__ void reduce_best(float& score, int& index, float* shared) {
  better(score, index, rotated<8>(score), (int)rotated<8>((uint32_t)index));
  better(score, index, rotated<4>(score), (int)rotated<4>((uint32_t)index));
  better(score, index, rotated<2>(score), (int)rotated<2>((uint32_t)index));
  better(score, index, rotated<1>(score), (int)rotated<1>((uint32_t)index));
  if (G >= 64) {
    better(score, index, __shfl_xor(score, 16), __shfl_xor(index, 16));
    better(score, index, __shfl_xor(score, 32), __shfl_xor(index, 32));
  }
  if (G > 64) {
    int* where = (int*)(shared + 8);
    if ((threadIdx.x & 63) == 0) { shared[threadIdx.x >> 6] = score; where[threadIdx.x >> 6] = index; }
    __syncthreads();
#pragma unroll
    for (int w = 0; w < G / 64; ++w) better(score, index, shared[w], where[w]);
    __syncthreads();
  }
}

// The part of the rows' records that this thread looks at, asked for ahead of everything else.
template <int G>
struct RecordPart {
  int row, row_index;     // of the block; of the call
  int first;              // this thread's first ply after the record's begin, then every G-th
  int from, to;           // as the caller has them
  __device__ __forceinline__ void begin(const Args& a, int first_row) {
    // neighbouring threads read what is next to each other in memory: the plies of a row, or the rows of a ply
    const int rows = (int)blockDim.x / G, tid = (int)threadIdx.x;
    row = a.record_by_row ? tid / G : tid % rows;
    first = a.record_by_row ? tid % G : tid / rows;
    const int b = min(first_row + row, a.rows - 1);
    from = a.begin ? a.begin[b] : 0;
    to = first_row + row >= a.rows ? 0 : a.end ? a.end[b] : a.record_len;
    row_index = b;
  }
  // How often each action occurs: 16-bit counters in LDS, two to a word, `words` words per row.
  __device__ __forceinline__ void count(const Args& a, uint32_t* counts, int words) {
    const int threads = (int)blockDim.x;
    for (int i = (int)threadIdx.x; i < threads / G * words; i += threads) counts[i] = 0;
    __syncthreads();
    uint32_t* mine = counts + row * words;
    int t = min(max(from, 0), a.record_len) + first;   // (a begin of the largest int32 is "no ply": the sum must not wrap)
    const int end = min(to, a.record_len);
    auto add = [&](int move, bool there) {
      if (there && (uint32_t)move < (uint32_t)a.actions) atomicAdd(&mine[move >> 1], 1u << (16 * (move & 1)));
    };
    constexpr int kAhead = 24;   // loads under way at once (65536 rows of up to 361 plies: 81 us with 8 and 64-bit addresses, 76 with 24 and 32-bit ones)
    if (a.record_near) {   // every move within 32 bits of the first: loads without a condition, those behind the end repeat the last
      const uint32_t row_at = (uint32_t)row_index * (uint32_t)a.record_row, ply = (uint32_t)a.record_ply, last = row_at + (uint32_t)max(end - 1, 0) * ply;
      for (; t < end; t += G * kAhead) {
        const uint32_t p = row_at + (uint32_t)t * ply;
        int move[kAhead];
#pragma unroll
        for (int j = 0; j < kAhead; ++j) move[j] = a.record[min(p + (uint32_t)(j * G) * ply, last)];
#pragma unroll
        for (int j = 0; j < kAhead; ++j) add(move[j], t + j * G < end);
      }
    } else {
      const int64_t step = (int64_t)G * a.record_ply;
      const int32_t* p = a.record + (int64_t)row_index * a.record_row + (int64_t)t * a.record_ply;
      for (; t < end; t += G, p += step) add(*p, true);
    }
    __syncthreads();
  }
};

// x / d, rounded to nearest, for a d whose reciprocal y is: the product's error is found exactly and taken off (P. Markstein, 1990: with y
// correctly rounded is).  3 instructions instead of 11; quotients below 2^-100 may differ in the last bit.  For |x| up to 2^100 and d from 2^-20 to 2^20.
__device__ __forceinline__ float divided(float x, float d, float y) {
  const float q = x * y;
  return __builtin_fmaf(-__builtin_fmaf(q, d, -x), y, q);   // (the error's negative, so that -0 stays -0)
}
__device__ __forceinline__ bool plain_divisor(float d) { return d >= 0x1p-20f && d <= 0x1p20f; }
template <int NC>
__device__ __forceinline__ bool plain_dividends(const float (&z)[NC][8]) {   // (false for infinities; NaN stays NaN either way)
  float most = 0.0f;
#pragma unroll
  for (int c = 0; c < NC; ++c)
#pragma unroll
    for (int j = 0; j < 8; ++j) most = fmaxf(most, fabsf(z[c][j]));
  return most <= 0x1p100f;
}

// G lanes and NC chunks per row: up to G * NC * 8 actions, and with FULL more than G * (NC - 1) * 8, so that only the last chunk can pass the row's end
template <class T, int G, int NC, bool FULL, bool RECORD, int OP>
__global__ void __launch_bounds__(kThreads) policy_kernel(Args a) {
#pragma clang fp contract(off)   // every operation of the adjustment is rounded by itself, as the header defines it
  extern __shared__ uint32_t counts[];
  __shared__ float shared[16];
  typedef typename T::type Elem;
  constexpr bool kLoss = OP == kLossShares || OP == kLossMoves;
  const int rows_per_block = (int)blockDim.x / G, words = (a.actions + 1) / 2 | 1;
  // blocks go to the eight dies in turn: each die takes a stretch of rows, so that rows that share a line of memory meet in its L2
  const uint32_t eighth = gridDim.x >> 3, piece = a.by_die ? (blockIdx.x & 7u) * eighth + (blockIdx.x >> 3) : blockIdx.x;
  const int first_row = (int)piece * rows_per_block, lane = (int)threadIdx.x % G, slot = (int)threadIdx.x / G;
  const int A = a.actions;
  if (first_row >= a.rows) return;
  const int b = min(first_row + slot, a.rows - 1);   // lanes beyond the last row repeat it and write nothing
  const bool mine = first_row + slot < a.rows;

  RecordPart<G> part;
  if (RECORD) part.begin(a, first_row);
  const Elem* logits = (const Elem*)a.logits + (int64_t)b * a.logits_pitch;
  float z[NC][8], other[NC][8];   // other: noise, or target shares
  uint32_t mask[NC][2];
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    const Chunk k(c * G + lane, A);
    load_chunk<T>(logits, k, A, z[c]);
    if (a.mask) load_mask(a.mask + (int64_t)b * a.mask_pitch, k, A, mask[c]);
    if (OP == kLossShares || (OP == kSample && a.second)) load_chunk<F32>(a.second + (int64_t)b * a.second_pitch, k, A, other[c]);
  }
  const float own_temperature = a.temperature_row ? a.temperature_row[b] : a.temperature;
  const bool greedy = !(own_temperature > 0.0f);
  const float temperature = greedy ? 1.0f : own_temperature;
  const float weight = kLoss && a.weight ? a.weight[b] : 1.0f;
  int taken = OP == kLossMoves ? a.taken[b] : -1;
  if ((uint32_t)taken >= (uint32_t)A) taken = -1;
  if (RECORD) part.count(a, counts, words);

  // the adjustment, a step at a time over all of the lane's actions
  uint32_t seen[NC], positive[NC];   // bits: the action occurs in the record; its logit is above 0 (for the gradient)
  if (RECORD) {
    const uint16_t* n_of = (const uint16_t*)(counts + slot * words);
    const float inverse = 1.0f / a.repetition;
    auto punish = [&](auto quick) {
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        const Chunk k(c * G + lane, A);
        seen[c] = positive[c] = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          float x = z[c][j];
          const uint32_t n = n_of[k.base + (A >= 8 ? j : min(j, A - 1))];
          if (kLoss) {
            seen[c] |= (uint32_t)(n > 0) << j;
            positive[c] |= (uint32_t)(x > 0.0f) << j;
          }
          const float less = quick.value ? divided(x, a.repetition, inverse) : x / a.repetition;
          const float punished = x > 0.0f ? less : x * a.repetition;
          x = n > 0 ? punished : x;
          x = x - a.frequency * (float)n;
          z[c][j] = x - (n > 0 ? a.presence : 0.0f);
        }
      }
    };
    if (__all(plain_divisor(a.repetition) && plain_dividends(z))) punish(std::true_type{});
    else punish(std::false_type{});
  }
  if (a.bias) {
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      float bias[8];
      load_chunk<F32>(a.bias + (int64_t)b * a.bias_pitch, Chunk(c * G + lane, A), A, bias);
#pragma unroll
      for (int j = 0; j < 8; ++j) z[c][j] = z[c][j] + bias[j];
    }
  }
  if (__any(temperature != 1.0f)) {
    if (__all(plain_divisor(temperature) && plain_dividends(z))) {
      const float inverse = 1.0f / temperature;
#pragma unroll
      for (int c = 0; c < NC; ++c)
#pragma unroll
        for (int j = 0; j < 8; ++j) z[c][j] = divided(z[c][j], temperature, inverse);
    } else {
#pragma unroll
      for (int c = 0; c < NC; ++c)
#pragma unroll
        for (int j = 0; j < 8; ++j) z[c][j] = z[c][j] / temperature;
    }
  }
  if (a.mask) {
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
      for (int j = 0; j < 8; ++j) z[c][j] = (mask[c][j >> 2] >> (8 * (j & 3)) & 0xFFu) != 0 ? z[c][j] : kNone;
  }
  if (OP == kLogits && !a.normalize) {
    if (G > 64) __syncthreads();   // out may be the logits: a row's last chunk reads what another wavefront's chunk before it writes
    if (mine) {
#pragma unroll
      for (int c = 0; c < NC; ++c) store_chunk<F32>((float*)a.out + (int64_t)b * a.out_pitch, Chunk(c * G + lane, A), A, z[c]);
    }
    return;
  }
  float top = kNone;   // (NaN, which is not possible, is left out; what a last chunk shares with the one before it may count twice here)
#pragma unroll
  for (int c = 0; c < NC; ++c)
#pragma unroll
    for (int j = 0; j < 8; ++j) top = fmaxf(top, z[c][j]);
  top = reduced<Max, G>(top, shared);
  const bool some = top > kNone;
  constexpr float kLowest = -0x1.fffffep127f;   // the lowest finite number
  // (the loss: beside a logit of +infinity, which makes the row NaN, z - from is at least 0 for every possible action, so that these are told from the others)
  const float from = !some ? 0.0f : !kLoss || top < INFINITY ? top : kLowest;

  if (OP == kSample && a.second && __any(greedy)) {
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
      for (int j = 0; j < 8; ++j) other[c][j] = greedy ? 0.0f : other[c][j];
  }

  // Sums over the possible actions: of e = exp(d), d = z - top, and for the loss of e d, y and y d.  d is kept at or above kFar, where e is 0
  // already (below -104 it is in 32 bits), so that an action that is not possible adds 0 to each of them.
  constexpr float kFar = -256.0f;
  float total = 0.0f, moment = 0.0f, share = 0.0f, cross = 0.0f, found = kNone;   // found: z, later z - top, of the move that was taken
  float best = kNone, best_z = kNone;
  int best_at = 0x7FFFFFFF;
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    const Chunk k(c * G + lane, A);
    const bool check = !FULL || c == NC - 1;
    const int rel = taken - k.base;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const bool counts_here = !check || (j >= k.skip && k.base + j < A);   // an action counts once
      const float raw = z[c][j] - from, d = fmaxf(raw, kFar), e = __expf(d), counted = counts_here ? e : 0.0f;
      total += counted;
      if (OP == kSample) {
        const float score = a.second ? z[c][j] + other[c][j] : z[c][j];
        const bool take = score > best;   // ascending within the lane: the lowest index among equals
        best = take ? score : best;
        best_z = take ? z[c][j] : best_z;
        best_at = take ? k.base + j : best_at;
      }
      if (kLoss) {
        moment = __builtin_fmaf(counted, d, moment);
        if (OP == kLossShares) {
          const float y = z[c][j] > kNone ? other[c][j] : 0.0f, y_counted = counts_here ? y : 0.0f;
          other[c][j] = y;
          share += y_counted;
          cross = __builtin_fmaf(y_counted, fmaxf(raw, kLowest), cross);   // (a finite number: y is 0 where the action is not possible)
        } else {
          found = rel == j ? z[c][j] : found;
        }
        z[c][j] = d;
      }
    }
  }
  total = reduced<Sum, G>(total, shared);
  const float log_total = __logf(total);

  if (OP == kLogits && mine) {
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      float out[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) out[j] = z[c][j] > kNone ? z[c][j] - from - log_total : kNone;
      store_chunk<F32>((float*)a.out + (int64_t)b * a.out_pitch, Chunk(c * G + lane, A), A, out);
    }
  }
  if (OP == kSample) {
    if (some && best_at == 0x7FFFFFFF) {   // this lane's scores are all -infinity or NaN: its lowest possible action
#pragma unroll
      for (int c = NC - 1; c >= 0; --c) {
        const Chunk k(c * G + lane, A);
#pragma unroll
        for (int j = 7; j >= 0; --j) {
          const bool take = z[c][j] > kNone && k.base + j < A;
          best_z = take ? z[c][j] : best_z;
          best_at = take ? k.base + j : best_at;
        }
      }
    }
    const int own = best_at;
    reduce_best<G>(best, best_at, shared);
    // the lane that holds the action writes (two if the row's last chunks share it: the same); a row without one is written by its first lane
    if (mine && own == best_at && (some || lane == 0)) {
      ((int32_t*)a.out)[b] = some ? best_at : -1;
      if (a.row_out) a.row_out[b] = some ? best_z - from - log_total : 0.0f;
    }
  }
  if (kLoss) {
    moment = reduced<Sum, G>(moment, shared);
    if (OP == kLossShares) {
      share = reduced<Sum, G>(share, shared);
      cross = reduced<Sum, G>(cross, shared);
    } else {
      found = reduced<Max, G>(fmaxf(found, kNone), shared);
      found = found > kNone ? fmaxf(found - from, kLowest) : kNone;
      share = found > kNone ? 1.0f : 0.0f;
      cross = found > kNone ? found : 0.0f;
    }
    const float inverse = some ? 1.0f / total : 0.0f;
    const float entropy = some ? log_total - moment * inverse : 0.0f;
    if (mine && lane == 0) {
      if (a.row_out) a.row_out[b] = some ? weight * (share * log_total - cross) - a.entropy_bonus * entropy : 0.0f;
      if (a.row_out2) a.row_out2[b] = entropy;
    }
    // with p = e / total:  weight (share p - y) + bonus p (d - log_total + entropy)  =  e (bend d + level) - pull y
    const float slope = a.grad_scale / temperature, pull = weight * slope, each = inverse * slope, bend = a.entropy_bonus * each;
    const float level = some ? (weight * share + a.entropy_bonus * (entropy - log_total)) * each : 0.0f;
    if (mine) {
      Elem* row = (Elem*)a.out + (int64_t)b * a.out_pitch;
      auto through = [&](int c, int j, float g) {   // back through the penalty for repeated moves
        return RECORD && (seen[c] >> j & 1u) ? (positive[c] >> j & 1u ? g / a.repetition : g * a.repetition) : g;
      };
      // Where all factors are finite, e = 0 makes the gradient of what is not possible 0.  Where they are not (the scale over a small temperature, a
      // logit of +infinity) it is chosen, not multiplied: choosing everywhere takes 2 us more for 65536 x 362.
      auto write = [&](auto finite) {
#pragma unroll
        for (int c = 0; c < NC; ++c) {
          const Chunk k(c * G + lane, A);
          float out[8];
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const float y = OP == kLossShares ? other[c][j] : 0.0f;
            float g = __expf(z[c][j]) * __builtin_fmaf(bend, z[c][j], level);
            if (!finite.value) g = z[c][j] > kFar ? g : 0.0f;   // (a possible action as far below has e = 0 too)
            if (OP == kLossShares) g = finite.value || y != 0.0f ? __builtin_fmaf(-pull, y, g) : g;   // (y is 0 where the action is not possible)
            out[j] = through(c, j, g);
          }
          store_chunk<T>(row, k, A, out);
          const int rel = taken - k.base;
          if (OP == kLossMoves && (uint32_t)rel < 8u && k.at < A && found > kNone)   // the move that was taken is written once more
            row[k.base + rel] = (Elem)through(c, rel, __expf(found) * __builtin_fmaf(bend, fmaxf(found, kFar), level) - pull);
        }
      };
      // (against a finite limit: the compiler takes "below infinity" for "not infinity" here, which NaN passes)
      if (__all(fabsf(bend) * -kFar + fabsf(level) + fabsf(pull) <= 0x1p127f)) write(std::true_type{});
      else write(std::false_type{});
    }
  }
}

template <class T, int G, int NC, bool FULL, int OP>
hipError_t launch(Args a, hipStream_t stream) {
  // a block of one wavefront while that leaves the machine's 256 compute units a block each at most; rows of a larger batch share blocks of four
  const int threads = G > 64 ? G : (int64_t)a.rows * G <= 64 * 1024 ? 64 : kThreads;
  const int rows_per_block = threads / G;
  const unsigned blocks = (unsigned)((a.rows + rows_per_block - 1) / rows_per_block);
  a.by_die = blocks >= 64;
  const dim3 grid(a.by_die ? (blocks + 7) / 8 * 8 : blocks), block((unsigned)threads);
  if (a.record) {
    const size_t lds = (size_t)rows_per_block * ((a.actions + 1) / 2 | 1) * 4;
    hipLaunchKernelGGL((policy_kernel<T, G, NC, FULL, true, OP>), grid, block, lds, stream, a);
  } else {
    hipLaunchKernelGGL((policy_kernel<T, G, NC, FULL, false, OP>), grid, block, 0, stream, a);
  }
  return hipGetLastError();
}
template <class T, int OP>
hipError_t launch_for_actions(const Args& a, hipStream_t stream) {
  if (a.actions <= 128) return launch<T, 16, 1, true, OP>(a, stream);
  if (a.actions <= 256) return launch<T, 16, 2, true, OP>(a, stream);
  if (a.actions <= 384) return launch<T, 16, 3, true, OP>(a, stream);
  if (a.actions <= 2048) return launch<T, 64, 4, false, OP>(a, stream);
  return launch<T, 256, 4, false, OP>(a, stream);
}
template <int OP>
int run(const Args& a, int32_t type, void* stream) {
  if (a.rows == 0) return PGXPOLICY_OK;
  switch (type) {
    case PGXPOLICY_F32: HIPCHK((launch_for_actions<F32, OP>(a, (hipStream_t)stream))); return PGXPOLICY_OK;
    case PGXPOLICY_F16: HIPCHK((launch_for_actions<F16, OP>(a, (hipStream_t)stream))); return PGXPOLICY_OK;
    case PGXPOLICY_BF16: HIPCHK((launch_for_actions<BF16, OP>(a, (hipStream_t)stream))); return PGXPOLICY_OK;
    default: return PGXPOLICY_EINVAL;
  }
}

// rows of an output must not overlap; an input's may (pitch 0: one row for all games)
bool pitch_ok(int64_t pitch, int32_t rows, int32_t actions) { return rows <= 1 || pitch >= actions; }
bool input_ok(const void* p, int64_t pitch) { return !p || pitch >= 0; }

// fills the arguments that all three calls share
bool common(Args& a, int32_t rows, int32_t actions, const void* logits, int32_t type, int64_t logits_pitch, const pgxpolicy_adjust* adjust) {
  a = Args{};
  if (rows < 0 || actions < 1 || actions > PGXPOLICY_MAX_ACTIONS || type < PGXPOLICY_F32 || type > PGXPOLICY_BF16) return false;
  if (rows > 0 && (!logits || ((uintptr_t)logits & (type == PGXPOLICY_F32 ? 3u : 1u)) != 0)) return false;
  if (!input_ok(logits, logits_pitch)) return false;
  a.rows = rows; a.actions = actions; a.logits = logits; a.logits_pitch = logits_pitch;
  a.repetition = a.temperature = 1.0f;
  if (!adjust) return true;
  a.mask = adjust->mask_dev; a.mask_pitch = adjust->mask_pitch;
  a.bias = adjust->bias_dev; a.bias_pitch = adjust->bias_pitch;
  if (!input_ok(a.mask, a.mask_pitch) || !input_ok(a.bias, a.bias_pitch)) return false;
  if (adjust->temperature_dev) a.temperature_row = adjust->temperature_dev;
  else if (adjust->temperature != 0.0f) a.temperature = adjust->temperature;
  if (!(a.temperature > 0.0f) || a.temperature > 3.402823e38f) return false;
  if (adjust->repetition != 0.0f) a.repetition = adjust->repetition;
  if (!(a.repetition > 0.0f) || a.repetition > 3.402823e38f) return false;
  a.frequency = adjust->frequency; a.presence = adjust->presence;
  if (adjust->record_len < 0 || adjust->record_len > PGXPOLICY_MAX_RECORD) return false;
  if (adjust->record_dev && adjust->record_len > 0) {
    a.record = adjust->record_dev; a.record_len = adjust->record_len;
    a.record_row = adjust->record_row_stride; a.record_ply = adjust->record_ply_stride;
    a.begin = adjust->begin_dev; a.end = adjust->end_dev;
    const int64_t most = (int64_t)1 << 29;   // elements
    a.record_near = a.record_row >= 0 && a.record_ply >= 0 && a.record_row < most && a.record_ply < most &&
                    (rows - 1) * a.record_row + (int64_t)(a.record_len - 1) * a.record_ply < most;
    a.record_by_row = llabs(a.record_ply) <= llabs(a.record_row);
  }
  return true;
}

}  // namespace

extern "C" {

int pgxpolicy_logits(int32_t rows, int32_t actions, const void* logits_dev, int32_t type, int64_t logits_pitch, const pgxpolicy_adjust* adjust,
                     int32_t normalize, float* out_dev, int64_t out_pitch, void* stream) {
  Args a;
  if (!common(a, rows, actions, logits_dev, type, logits_pitch, adjust)) return PGXPOLICY_EINVAL;
  if ((rows > 0 && !out_dev) || !pitch_ok(out_pitch, rows, actions)) return PGXPOLICY_EINVAL;
  a.out = out_dev; a.out_pitch = out_pitch; a.normalize = normalize;
  return run<kLogits>(a, type, stream);
}

int pgxpolicy_sample(int32_t rows, int32_t actions, const void* logits_dev, int32_t type, int64_t logits_pitch, const pgxpolicy_adjust* adjust,
                     const float* noise_dev, int64_t noise_pitch, int32_t* actions_dev, float* logp_dev, void* stream) {
  Args a;
  if (!common(a, rows, actions, logits_dev, type, logits_pitch, adjust)) return PGXPOLICY_EINVAL;
  if ((rows > 0 && !actions_dev) || !input_ok(noise_dev, noise_pitch)) return PGXPOLICY_EINVAL;
  a.second = noise_dev; a.second_pitch = noise_pitch; a.out = actions_dev; a.row_out = logp_dev;
  return run<kSample>(a, type, stream);
}

int pgxpolicy_loss(int32_t rows, int32_t actions, const void* logits_dev, int32_t type, int64_t logits_pitch, const pgxpolicy_adjust* adjust,
                   const float* target_dev, int64_t target_pitch, const int32_t* taken_dev, const float* weight_dev, float entropy_bonus, float grad_scale,
                   float* loss_dev, float* entropy_dev, void* grad_dev, int64_t grad_pitch, void* stream) {
  Args a;
  if (!common(a, rows, actions, logits_dev, type, logits_pitch, adjust)) return PGXPOLICY_EINVAL;
  if (rows > 0 && (!grad_dev || (target_dev != nullptr) == (taken_dev != nullptr))) return PGXPOLICY_EINVAL;
  if (!pitch_ok(grad_pitch, rows, actions) || !input_ok(target_dev, target_pitch)) return PGXPOLICY_EINVAL;
  a.second = target_dev; a.second_pitch = target_pitch; a.taken = taken_dev; a.weight = weight_dev;
  a.entropy_bonus = entropy_bonus; a.grad_scale = grad_scale;
  a.row_out = loss_dev; a.row_out2 = entropy_dev; a.out = grad_dev; a.out_pitch = grad_pitch;
  return target_dev ? run<kLossShares>(a, type, stream) : run<kLossMoves>(a, type, stream);
}

const char* pgxpolicy_strerror(int code) {
  switch (code) {
    case PGXPOLICY_OK: return "ok";
    case PGXPOLICY_EINVAL: return "invalid argument";
    case PGXPOLICY_EHIP: return "HIP runtime error";
    default: return "unknown error";
  }
}

int pgxpolicy_last_hip_error(void) { return g_last_hip; }

}  // extern "C"
