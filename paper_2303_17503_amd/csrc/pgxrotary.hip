// pgxrotary.hip -- queries and keys turned by their positions (include/pgxrotary.h), gfx950.
//
// A block has some tokens.  The cosines and sines of their positions are worked out once, in LDS, for all heads of both tensors (an angle takes 64-bit
// arithmetic and some 100 instructions, a pair of elements 4); then threads take the rows, 8 pairs each, so that neighbouring threads read neighbouring memory, with the next
// row on its way while one is turned.
//
// Bound by the bytes: 185000 tokens of 10 heads of 64 in bfloat16 94 to 97 us, 5.0 TB/s (vector instructions keep half of the time busy); 40001 of 16 heads of 128 in float32, half of each turned, 135 to 138 us,
// 4.8 TB/s.  One ply of 256 games 3.3 us: a launch, one round trip to memory and an angle.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>
#include <stdlib.h>

#include <utility>

#include "pgxrotary.h"
#include "rows_apart.hpp"

namespace {

thread_local int g_last_hip = 0;

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x8 __attribute__((ext_vector_type(8)));
typedef u32x4 u32x4_2 __attribute__((aligned(2)));
typedef f32x4 f32x4_4 __attribute__((aligned(4)));

// 8 neighbouring elements at any alignment that the element type has (the target takes vector accesses at any address)
struct F32 {
  typedef float type;
  static __device__ __forceinline__ f32x8 load8(const type* p) {
    const f32x4 a = *(const f32x4_4*)p, b = *(const f32x4_4*)(p + 4);
    return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
  }
  static __device__ __forceinline__ void store8(type* p, f32x8 x) {
    *(f32x4_4*)p = __builtin_shufflevector(x, x, 0, 1, 2, 3);
    *(f32x4_4*)(p + 4) = __builtin_shufflevector(x, x, 4, 5, 6, 7);
  }
};
template <class H>
struct Half {
  typedef H type;
  typedef H h8 __attribute__((ext_vector_type(8)));
  static __device__ __forceinline__ f32x8 load8(const type* p) {
    return __builtin_convertvector(__builtin_bit_cast(h8, (u32x4)*(const u32x4_2*)p), f32x8);
  }
  static __device__ __forceinline__ void store8(type* p, f32x8 x) {   // to nearest, ties to even
    *(u32x4_2*)p = __builtin_bit_cast(u32x4, __builtin_convertvector(x, h8));
  }
};

struct Args {
  pgxrotary_part part[PGXROTARY_MAX_PARTS];
  const int32_t* positions;
  const double* frequencies;
  int64_t positions_entry, positions_token;
  int32_t tokens, head_dim, pairs, heads, block_tokens, entry_blocks, pair_chunks, chunks;   // heads: of all parts; chunks: of a row, those with pairs first
  float magnitude;
  int32_t per_wave, lanes, t_step, h_step;          // rows that a wavefront, and the block, look at together; these as tokens and heads
  uint32_t chunks_inverse, heads_inverse, pairs_inverse;   // rounded up: over 2^16, quotients of threads; over 2^32, of angles
  int32_t entries, inverse, back;   // back: a run of pairs or elements that is not full begins earlier instead, so that it is, and shares some with the one before it
};

struct Row {   // where a row begins
  const char* in;
  char* out;
};

template <class T, bool INTERLEAVED>
__global__ void __launch_bounds__(256) turn_kernel(Args a) {
  typedef typename T::type E;
  extern __shared__ float2 turns[];   // [block_tokens][pairs]: cosine, sine
  const int threads = (int)blockDim.x, tid = (int)threadIdx.x, A = a.pairs;
  const int entry = a.entries == 1 ? 0 : (int)(blockIdx.x / (uint32_t)a.entry_blocks), token0 = (int)(blockIdx.x - (uint32_t)entry * (uint32_t)a.entry_blocks) * a.block_tokens;
  const int here = min(a.block_tokens, a.tokens - token0), rows = here * a.heads;
  // Rows that the block looks at together.  A row's chunks are in one wavefront where that holds them: it has loaded all of a row before it stores any, so chunks that share
  // elements may be turned in place.
  const bool whole = a.chunks <= 64;
  const int part = whole ? tid & 63 : tid, in_part = (int)((uint32_t)part * a.chunks_inverse >> 16), chunk = part - in_part * a.chunks;
  const int row0 = whole ? tid / 64 * a.per_wave + in_part : in_part, lanes = a.lanes;
  const bool busy = in_part < (whole ? a.per_wave : lanes);

  // both parts' addresses of the block's first token, and a row's from them
  const E *in0 = (const E*)a.part[0].in_dev + entry * a.part[0].in_entry_stride + token0 * a.part[0].in_token_stride;
  const E *in1 = (const E*)a.part[1].in_dev + entry * a.part[1].in_entry_stride + token0 * a.part[1].in_token_stride;
  E *out0 = (E*)a.part[0].out_dev + entry * a.part[0].out_entry_stride + token0 * a.part[0].out_token_stride;
  E *out1 = (E*)a.part[1].out_dev + entry * a.part[1].out_entry_stride + token0 * a.part[1].out_token_stride;
  const int heads0 = a.part[0].heads;
  auto row = [&](int t, int h) __attribute__((always_inline)) {
    const bool second = h >= heads0;
    const int64_t in_token = second ? a.part[1].in_token_stride : a.part[0].in_token_stride, in_head = second ? a.part[1].in_head_stride : a.part[0].in_head_stride;
    const int64_t out_token = second ? a.part[1].out_token_stride : a.part[0].out_token_stride, out_head = second ? a.part[1].out_head_stride : a.part[0].out_head_stride;
    const int head = second ? h - heads0 : h;
    return Row{(const char*)((second ? in1 : in0) + t * in_token + head * in_head), (char*)((second ? out1 : out0) + t * out_token + head * out_head)};
  };
  const bool turned = chunk < a.pair_chunks;
  const int low = turned ? 0 : 2 * A, high = turned ? A : a.head_dim, begin = low + (turned ? chunk : chunk - a.pair_chunks) * 8;
  const int at = a.back && high - low >= 8 ? min(begin, high - 8) : begin;              // first pair, or first element that is copied
  const int many = min(8, high - at);                                                   // pairs or elements
  const int u0 = !turned ? at : INTERLEAVED ? 2 * at : at, w0 = INTERLEAVED ? u0 + 8 : at + A;   // the two runs of elements; of a copied chunk the first
  struct Chunk {
    f32x8 x, y;   // the two runs
  };
  auto load = [&](const char* p) {
    const E* e = (const E*)p;
    Chunk c = {};
    if (many == 8) {
      c.x = T::load8(e + u0);
      if (turned) c.y = T::load8(e + w0);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int last = turned && INTERLEAVED ? 2 * many : many;
        if (j < last) c.x[j] = (float)e[u0 + j];
        if (turned && (INTERLEAVED ? j + 8 : j) < last) c.y[j] = (float)e[w0 + j];
      }
    }
    return c;
  };
  Chunk now_chunk = {};
  Row now{nullptr, nullptr};
  int t = (int)((uint32_t)row0 * a.heads_inverse >> 16), h = row0 - t * a.heads;
  if (busy && row0 < rows) {   // the first row is on its way while the angles are worked out
    now = row(t, h);
    now_chunk = load(now.in);
  }
  for (int k = tid; k < here * A; k += threads) {
    const int t = A == 1 ? k : (int)__umulhi((uint32_t)k, a.pairs_inverse), j = k - t * A;
    const int32_t position = a.positions[entry * a.positions_entry + (int64_t)(token0 + t) * a.positions_token];
    // Of a whole circle, to -1/2 .. 1/2: the turns of a position as two numbers, and the whole turns taken off before their product with the position is rounded, so that 2^-52 of a turn
    // is what is lost however far the position.
    constexpr double kTurn = 0x1.45f306dc9c883p-3, kTurnRest = -0x1.6b01ec5417056p-57;   // 1 / (2 pi) is their sum
    const double f = a.frequencies[j], far = (double)position, each = f * kTurn, each_rest = __builtin_fma(f, kTurnRest, __builtin_fma(f, kTurn, -each));
    const double part = __builtin_fma(far, each_rest, __builtin_fma(far, each, -rint(far * each)));
    float s, c;
    sincospif(2.0f * (float)part, &s, &c);
    turns[k] = make_float2(a.magnitude * c, a.inverse ? -a.magnitude * s : a.magnitude * s);
  }
  __syncthreads();
  if (!busy) return;
  for (int r = row0; r < rows; r += lanes) {
    Chunk next_chunk = {};
    Row next{nullptr, nullptr};
    const float2* turn = turns + t * A + at;
    t += a.t_step;
    h += a.h_step;
    if (h >= a.heads) {
      h -= a.heads;
      ++t;
    }
    if (r + lanes < rows) {
      next = row(t, h);
      next_chunk = load(next.in);
    }
    E* e = (E*)now.out;
    f32x8 x = now_chunk.x, y = now_chunk.y;
    if (turned) {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float2 cs = turn[j];   // (behind the last pair: what is there is not used)
        const int k = 2 * (j & 3);
        const float b = INTERLEAVED ? (j < 4 ? now_chunk.x[k] : now_chunk.y[k]) : now_chunk.x[j], d = INTERLEAVED ? (j < 4 ? now_chunk.x[k + 1] : now_chunk.y[k + 1]) : now_chunk.y[j];
        const float b1 = __builtin_fmaf(b, cs.x, -(d * cs.y)), d1 = __builtin_fmaf(d, cs.x, b * cs.y);
        if (!INTERLEAVED) { x[j] = b1; y[j] = d1; }
        else if (j < 4) { x[k] = b1; x[k + 1] = d1; }
        else { y[k] = b1; y[k + 1] = d1; }
      }
    }
    if (many == 8) {
      T::store8(e + u0, x);
      if (turned) T::store8(e + w0, y);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int last = turned && INTERLEAVED ? 2 * many : many;
        if (j < last) e[u0 + j] = (E)x[j];
        if (turned && (INTERLEAVED ? j + 8 : j) < last) e[w0 + j] = (E)y[j];
      }
    }
    now = next;
    now_chunk = next_chunk;
  }
}

template <class T>
hipError_t launch(Args& a, int32_t entries, bool interleaved, hipStream_t stream) {
  // Tokens of a block: as many as give each of 256 threads three chunks, two of 32-bit elements (185000 tokens of 10 heads of 64 in bfloat16 with one 98.6 us, two 93.1, three 93.9, eight 104; 192000 of
  // 3 heads of 256 146, 136, 126, 150; in float32 one and two are even: with one, two and three 65536 of 5 of 32 17.4, 16.4, -; 160000 of 10 of 130 336, 333.5, 345; 92000 of 16 of 128 270.5, 271.4, 280.9;
  // 40001 of 16 of 128, half of each turned, 133.7, 134.8, 137.8; 185000 of 10 of 64 168.5, 175.9, 182; 64000 of 3 of 256 76.8, 82.9, 76.8), fewer where that would
  // leave the machine's 256 compute units without four blocks each (16384 tokens of one ply: 9.7 us, with half and twice the blocks 11.0 and 9.8); an entry's tokens in equal shares.
  constexpr int kChunks = sizeof(typename T::type) == 4 ? 2 : 3;
  const int64_t per_token = (int64_t)a.heads * a.chunks, spread = ((int64_t)entries * a.tokens + 1023) / 1024, room = 4096 / a.pairs;
  int64_t tokens = (kChunks * 256 + per_token - 1) / per_token;
  tokens = tokens < spread ? tokens : spread;
  tokens = tokens < room ? tokens : room;
  if (tokens < 1) tokens = 1;
  a.entry_blocks = (int32_t)((a.tokens + tokens - 1) / tokens);
  a.block_tokens = (int32_t)(((int64_t)a.tokens + a.entry_blocks - 1) / a.entry_blocks);
  const int threads = a.chunks <= 64 && a.block_tokens * per_token <= 128 ? 64 : 256;
  if ((int64_t)entries * a.entry_blocks * threads >= (int64_t)1 << 32) return hipErrorInvalidConfiguration;   // (a launch of so many threads runs what is left of them beyond 2^32, without an error)
  a.entries = entries;
  a.per_wave = a.chunks <= 64 ? 64 / a.chunks : 0;
  a.lanes = a.chunks <= 64 ? threads / 64 * a.per_wave : threads / a.chunks;
  a.t_step = a.lanes / a.heads; a.h_step = a.lanes % a.heads;
  // (exact: thread * (what rounding up adds) is below the power of two for up to 256 threads and divisors, 4096 angles of up to 512 pairs; quotients by more heads are 0)
  a.chunks_inverse = (65536u + (uint32_t)a.chunks - 1) / (uint32_t)a.chunks;
  a.heads_inverse = (65536u + (uint32_t)a.heads - 1) / (uint32_t)a.heads;
  a.pairs_inverse = a.pairs == 1 ? 0 : (uint32_t)((((uint64_t)1 << 32) + (uint64_t)a.pairs - 1) / (uint64_t)a.pairs);
  const dim3 grid((unsigned)(entries * a.entry_blocks)), block((unsigned)threads);
  const size_t lds = ((size_t)a.block_tokens * a.pairs + 8) * sizeof(float2);
  if (interleaved) hipLaunchKernelGGL((turn_kernel<T, true>), grid, block, lds, stream, a);
  else hipLaunchKernelGGL((turn_kernel<T, false>), grid, block, lds, stream, a);
  return hipGetLastError();
}

}  // namespace

extern "C" {

int pgxrotary_turn(int32_t entries, int32_t tokens, int32_t head_dim, int32_t rotary_dim, int32_t type, const int32_t* positions_dev, int64_t positions_entry_stride,
                   int64_t positions_token_stride, const double* frequencies_dev, float magnitude, int32_t interleaved, int32_t inverse, int32_t parts,
                   const pgxrotary_part* part, void* stream) {
  if (entries < 0 || tokens < 0 || head_dim < 2 || head_dim > PGXROTARY_MAX_HEAD_DIM || rotary_dim < 2 || rotary_dim > head_dim || rotary_dim % 2 != 0) return PGXROTARY_EINVAL;
  if (type < PGXROTARY_F32 || type > PGXROTARY_BF16 || parts < 1 || parts > PGXROTARY_MAX_PARTS || !part || !(magnitude - magnitude == 0.0f)) return PGXROTARY_EINVAL;
  const int64_t total = (int64_t)entries * tokens;
  if (total > 0x7FFFFFFF) return PGXROTARY_EINVAL;
  Args a = {};
  bool in_place = true, any_in_place = false;
  for (int k = 0; k < parts; ++k) {
    const pgxrotary_part& p = part[k];
    if (p.heads < 0 || p.heads > 65536) return PGXROTARY_EINVAL;
    a.part[k] = p;
    a.heads += p.heads;
    if (p.heads == 0 || total == 0) continue;
    const uintptr_t either = (uintptr_t)p.in_dev | (uintptr_t)p.out_dev;
    const int64_t sizes[3] = {entries, tokens, p.heads}, out[3] = {p.out_entry_stride, p.out_token_stride, p.out_head_stride};
    if (!p.in_dev || !p.out_dev || (either & (type == PGXROTARY_F32 ? 3u : 1u)) != 0 || !rows_apart(sizes, out, head_dim)) return PGXROTARY_EINVAL;
    const bool same = p.in_dev == p.out_dev && (entries == 1 || p.in_entry_stride == p.out_entry_stride) && (tokens == 1 || p.in_token_stride == p.out_token_stride) &&
                      (p.heads == 1 || p.in_head_stride == p.out_head_stride);
    in_place = in_place && same;
    any_in_place = any_in_place || same;
    // Wavefronts store rows while others have yet to load theirs: beside an output that is its own input, no output may share memory with an input or another output.
    const int64_t bytes = type == PGXROTARY_F32 ? 4 : 2;
    const Rows output = {p.out_dev, {entries, tokens, p.heads}, {out[0], out[1], out[2]}};
    for (int j = 0; j < parts; ++j) {
      const pgxrotary_part& o = part[j];
      if (!(j == k && same) && rows_meet(Rows{o.in_dev, {entries, tokens, o.heads}, {o.in_entry_stride, o.in_token_stride, o.in_head_stride}}, output, head_dim, bytes)) return PGXROTARY_EINVAL;
      if (j > k && rows_meet(Rows{o.out_dev, {entries, tokens, o.heads}, {o.out_entry_stride, o.out_token_stride, o.out_head_stride}}, output, head_dim, bytes)) return PGXROTARY_EINVAL;
    }
  }
  if (total == 0 || a.heads == 0) return PGXROTARY_OK;
  if (!positions_dev || !frequencies_dev || ((uintptr_t)positions_dev & 3u) != 0 || ((uintptr_t)frequencies_dev & 7u) != 0) return PGXROTARY_EINVAL;
  a.positions = positions_dev; a.positions_entry = positions_entry_stride; a.positions_token = positions_token_stride;
  a.frequencies = frequencies_dev; a.magnitude = magnitude; a.inverse = inverse;
  a.tokens = tokens; a.head_dim = head_dim; a.pairs = rotary_dim / 2;
  a.pair_chunks = (a.pairs + 7) / 8;
  a.chunks = a.pair_chunks + (in_place ? 0 : (head_dim - rotary_dim + 7) / 8);
  a.back = a.chunks <= 64 || !any_in_place;
  // entries whose tokens follow each other's in every tensor are one long entry, and so are entries of one token
  bool follow = true;
  auto next = [&](int64_t& entry, int64_t& token) {
    if (tokens == 1) token = entry;
    else follow = follow && (entries == 1 || entry == token * tokens);
  };
  next(a.positions_entry, a.positions_token);
  for (int k = 0; k < parts; ++k) {
    if (a.part[k].heads == 0) continue;
    next(a.part[k].in_entry_stride, a.part[k].in_token_stride);
    next(a.part[k].out_entry_stride, a.part[k].out_token_stride);
  }
  if (follow) {
    a.tokens = (int32_t)total;
    entries = 1;
  } else if (entries > tokens && entries >= 1 << 24) {   // more entries than a launch has blocks: tokens of one place are the entries then
    std::swap(entries, a.tokens);
    std::swap(a.positions_entry, a.positions_token);
    for (pgxrotary_part& p : a.part) {
      std::swap(p.in_entry_stride, p.in_token_stride);
      std::swap(p.out_entry_stride, p.out_token_stride);
    }
  }
  const hipStream_t s = (hipStream_t)stream;
  const hipError_t e = type == PGXROTARY_F32 ? launch<F32>(a, entries, interleaved != 0, s) : type == PGXROTARY_F16 ? launch<Half<_Float16>>(a, entries, interleaved != 0, s) : launch<Half<__bf16>>(a, entries, interleaved != 0, s);
  if (e == hipErrorInvalidConfiguration) return PGXROTARY_EINVAL;
  if (e != hipSuccess) {
    g_last_hip = (int)e;
    return PGXROTARY_EHIP;
  }
  return PGXROTARY_OK;
}

const char* pgxrotary_strerror(int code) {
  switch (code) {
    case PGXROTARY_OK: return "ok";
    case PGXROTARY_EINVAL: return "invalid argument";
    case PGXROTARY_EHIP: return "HIP runtime error";
    default: return "unknown error";
  }
}

int pgxrotary_last_hip_error(void) { return g_last_hip; }

}  // extern "C"
