// cache_common.hpp -- what the kernels of the paged cache (include/pgxcache.h) share: the handle, the pages' layout, how a row of attention ends.
#ifndef CACHE_COMMON_HPP_
#define CACHE_COMMON_HPP_

#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>
#include <stdlib.h>

#include <type_traits>

#include "pgxcache.h"

constexpr int kNoTail = -1, kSkip = -2;
struct __attribute__((aligned(16))) pgxcache_fork_entry {   // an entry of a fork call as its plan leaves it, so that the copying starts after one look at memory
  int32_t tail;            // the page for the copy of the last page, kNoTail or kSkip
  int32_t src, dst, length;
  int32_t last;            // the source's partly filled last page
  int32_t old;             // pages of the destination
  int32_t unused[2];
};

struct pgxcache_ctx {
  pgxcache_opts o;
  void* kv;
  float* scales;           // null: keys and values are held in 16 bits
  int32_t *table, *lengths, *refs;
  uint64_t* free_bits;     // a bit per page: free; 0 behind the last page
  uint64_t* taken;         // the same shape: pages given out by a plan and still marked free; 0 between calls
  int32_t* grown;          // [slots] tokens that the slot's last advance made room for
  int32_t* plan;           // [slots] advance: whether the entry is done
  pgxcache_fork_entry* forks;   // [slots] what fork does with its entries
  int32_t* moved_to;       // [pages] compact: where a page at or above `used` goes
  int2* moves;             // [pages] compact: (from, to)
  int32_t* counts;         // compact: used, number of moves
  uint32_t* arrived;       // [kSplitBlocks] attend: blocks of a row that are done, 0 between calls
  float* partial;          // attend: what they found
};

namespace pgxcache_parts {

typedef pgxcache_fork_entry ForkEntry;
constexpr int kSplitBlocks = 512;    // most blocks of an attend call that splits rows
constexpr int kMostSplits = 128;     // most blocks of one row
constexpr int kHeads = 16;           // query heads of a matrix tile
constexpr int kBlockShift = 4;       // tokens that share a scale: 16

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef u32x4 u32x4_2 __attribute__((aligned(2)));

// what every kernel knows of the cache
struct Cache {
  char* kv;
  int32_t *table, *lengths, *refs;
  uint64_t *free_bits, *taken;
  int32_t* grown;
  int32_t slots, pages, width, page_shift, layers, kv_heads, head_dim;
  float* scales;           // [pages][layers][2][kv_heads][blocks of a page]; null where elements have 16 bits

  __device__ __forceinline__ int pages_of(int tokens) const { return (int)(((int64_t)tokens + (1 << page_shift) - 1) >> page_shift); }
  __device__ __forceinline__ int capacity() const { return (int)min((int64_t)width << page_shift, (int64_t)0x7FFFFFFF); }
  __device__ __forceinline__ int length(int slot) const { return min(max(lengths[slot], 0), capacity()); }
  __device__ __forceinline__ int32_t* row(int slot) const { return table + (int64_t)slot * width; }
  __device__ __forceinline__ bool is_page(int p) const { return (uint32_t)p < (uint32_t)pages; }
  __host__ __device__ __forceinline__ int element_bytes() const { return scales ? 1 : 2; }
  // (kernels that know how many bytes an element has say so)
  __host__ __device__ __forceinline__ int64_t head_bytes(int element) const { return ((int64_t)head_dim << page_shift) * element; }   // one head's keys or values of a page
  __host__ __device__ __forceinline__ int64_t page_bytes(int element) const { return head_bytes(element) * kv_heads * 2 * layers; }
  __host__ __device__ __forceinline__ int64_t head_bytes() const { return head_bytes(element_bytes()); }
  __host__ __device__ __forceinline__ int64_t page_bytes() const { return page_bytes(element_bytes()); }
  __host__ __device__ __forceinline__ int page_blocks() const { return 1 << (page_shift - kBlockShift); }
  __host__ __device__ __forceinline__ int64_t page_scales() const { return (int64_t)page_blocks() * kv_heads * 2 * layers; }
};

struct Tokens {   // keys or values of new tokens
  const char* p;
  int64_t entry, token, head;   // strides in bytes
};

struct AttendArgs {
  const char *q, *k, *v;
  char* out;
  float* lse;
  int64_t q_entry, q_head, k_entry, k_head, v_entry, v_head, out_entry, out_head;   // bytes
  const int32_t* slots;
  float* partial;
  uint32_t* arrived;
  int32_t n, layer, heads, group, head_tiles, splits;
  float scale;   // times log2 e
  int32_t by_die;   // 8 bits: whether heads of one part are launched eight blocks apart
};

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef f32x4 f32x4_4 __attribute__((aligned(4)));

// Probabilities go into the second product as two numbers of the type that add up to them, relative to an exponent that is moved only when a tile
// requires it, so that most tiles need no exchange between lanes.
//  * bfloat16 has the range of 32 bits: the sum is within 2^-17 of p whatever its size.  The exponent is the running maximum, raised when a score passes it by 2^8.
//  * float16 ends at 65504 and at steps of 2^-24: the sum is within 2^-22 of p or within 2^-25.  The exponent goes up and down with the tiles, so that the
//    largest p of a head in a tile is between 2^-3 and 2^15 (2^11 where it is moved), and the tile's 32 errors add up to 2^-17 of the tile's sum at most.  It goes no further down than 2^60
//    below the largest score, where nothing counts any more and the sums stay far from the end of 32 bits.  With the running maximum for exponent, p
//    below 2^-25 of it was lost (721 tokens at e^-15 beside one: 0.7 % of what they add), and the time is the same.
struct F16 {
  typedef _Float16 elem;
  static constexpr bool kNarrow = true;
  static constexpr float kLargest = 65504.0f;
  static constexpr float kRoom = 11.0f, kMost = 15.0f, kLeast = -3.0f, kDepth = 60.0f;
  typedef elem x8 __attribute__((ext_vector_type(8)));
  static __device__ __forceinline__ f32x4 mfma(x8 a, x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
};
struct BF16 {
  typedef __bf16 elem;
  static constexpr bool kNarrow = false;
  static constexpr float kLargest = 0x1.fep127f;
  static constexpr float kRoom = 0.0f, kMost = 8.0f, kLeast = 0.0f, kDepth = 0.0f;
  typedef elem x8 __attribute__((ext_vector_type(8)));
  static __device__ __forceinline__ f32x4 mfma(x8 a, x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
};

constexpr float kLn2 = 0.69314718055994530942f;

__device__ __forceinline__ float across_groups_max(float x) {
  x = fmaxf(x, __shfl_xor(x, 16));
  return fmaxf(x, __shfl_xor(x, 32));
}
__device__ __forceinline__ float across_groups_sum(float x) {
  x += __shfl_xor(x, 16);
  return x + __shfl_xor(x, 32);
}

// What one block leaves for another of the same launch goes through the dies' L2 caches, which do not know of each other, without
// writing back or dropping anything else in them: a device-wide fence per block instead cost 20 us each, 32 us with 3 sequences of 110000 tokens.
constexpr int kAcrossDies = 16;             // cache policy of a buffer instruction: as an atomic access of the whole device (sc1)
constexpr int kBufferFlags = 0x00027000;    // raw buffer of 32-bit words

// A launch of 2^32 threads or more runs what is left of them beyond 2^32 and reports no error: calls that would need one are refused.
inline bool launchable(int64_t blocks, int threads) { return blocks * threads < (int64_t)1 << 32; }

template <bool STREAM, class V>
__device__ __forceinline__ V read_once(const V* p) { return STREAM ? __builtin_nontemporal_load(p) : *p; }

// Where a wavefront stands in an attend call.
struct Spot {
  int wave, lane, col, g;            // col: head of the tile, g: group of 16 lanes
  int i, head0, heads_here;          // entry, first query head, query heads of the tile
  int split, active;                 // block of the row, blocks that it has
  uint32_t unit;                     // the row's number
  bool alone;                        // the row's first wavefront has all of it
};

// Elements of the output before they are rounded.  Over 8 bits a float16 value above 63488 is held as 65536, so that averages of such values may lie beyond the type's end by what
// held them and by the sums' errors, well below 2^-10; they become its largest number.  (One look for all of a wavefront's: two comparisons for each element take 0.2 us with 1024 rows.)
template <class T, bool EIGHT, int N>
__device__ __forceinline__ void within_type(float (&x)[N]) {
  if constexpr (EIGHT && T::kNarrow) {
    float most = 0.0f;
#pragma unroll
    for (int e = 0; e < N; ++e) most = fmaxf(most, fabsf(x[e]));
    if (__any(most > T::kLargest)) {
#pragma unroll
      for (int e = 0; e < N; ++e) x[e] = fabsf(x[e]) > T::kLargest && fabsf(x[e]) < 65536.0f * (1.0f + 0x1p-10f) ? copysignf(T::kLargest, x[e]) : x[e];
    }
  }
}

// The end of a row: the parts of W wavefronts, and of `active` blocks, are joined and written.  Lane 16 g + c has elements (4 g + r) D/16 + m of head c in
// acc[m][r], relative to the exponent `top` (of powers of two), and the sum of its group's probabilities.  EIGHT: keys and values are held in 8 bits.
template <class T, int NT, int W, bool SPLIT, bool EIGHT>
__device__ __forceinline__ void finish_row(const AttendArgs& a, const Spot& at_spot, float top, float sum, f32x4 (&acc)[2 * NT]) {
  typedef typename T::x8 x8;
  constexpr int D = NT * 32, kOut = 8 * NT;   // elements of the output per lane
  __shared__ float joined_m[W][kHeads], joined_l[W][kHeads];
  extern __shared__ float joined_o[];   // [W - 1][kHeads][D]
  const int wave = at_spot.wave, lane = at_spot.lane, col = at_spot.col, g = at_spot.g, i = at_spot.i, head0 = at_spot.head0, heads_here = at_spot.heads_here;
  const int split = at_spot.split, active = at_spot.active;
  const uint32_t unit = at_spot.unit;
  const bool alone = at_spot.alone;
  sum = across_groups_sum(sum);

  if (W > 1 && !alone) {   // the wavefronts' parts, into the first's registers
    if (g == 0) { joined_m[wave][col] = top; joined_l[wave][col] = sum; }
    __syncthreads();
    float now = -INFINITY;
#pragma unroll
    for (int w = 0; w < W; ++w) now = fmaxf(now, joined_m[w][col]);
    const float from = now > -INFINITY ? now : 0.0f, factor = __builtin_amdgcn_exp2f(top - from);
    sum = 0.0f;
#pragma unroll
    for (int w = 0; w < W; ++w) sum += joined_l[w][col] * __builtin_amdgcn_exp2f(joined_m[w][col] - from);
    top = now;
#pragma unroll
    for (int m = 0; m < 2 * NT; ++m) acc[m] *= factor;
    if (wave > 0) {
#pragma unroll
      for (int m = 0; m < 2 * NT; ++m)
#pragma unroll
        for (int r = 0; r < 4; ++r) joined_o[((wave - 1) * 8 * NT + m * 4 + r) * 64 + lane] = acc[m][r];
    }
    __syncthreads();
    if (wave == 0) {
#pragma unroll
      for (int w = 0; w < W - 1; ++w)
#pragma unroll
        for (int m = 0; m < 2 * NT; ++m)
#pragma unroll
          for (int r = 0; r < 4; ++r) acc[m][r] += joined_o[(w * 8 * NT + m * 4 + r) * 64 + lane];
    }
  }

  if (!SPLIT || active == 1) {
    if (wave > 0) return;
    if (col >= heads_here) return;
    const float inverse = 1.0f / sum;
    char* out = a.out + i * a.out_entry + (head0 + col) * a.out_head + g * kOut * 2;
    float y[kOut];
#pragma unroll
    for (int e = 0; e < kOut; ++e) y[e] = acc[e % (2 * NT)][e / (2 * NT)] * inverse;
    within_type<T, EIGHT>(y);
#pragma unroll
    for (int u = 0; u < NT; ++u) {
      x8 x;
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = (typename T::elem)y[u * 8 + e];
      *(u32x4_2*)(out + u * 16) = __builtin_bit_cast(u32x4, x);
    }
    if (a.lse && g == 0) a.lse[(int64_t)i * a.heads + head0 + col] = (top + __log2f(sum)) * kLn2;
    return;
  }

  // The row is split over `active` blocks: each leaves its part in memory, and the one that comes last joins them, in an order of its own.
  // All its loads are of 16 bytes and under way together: with 4-byte ones, one output each, joining 256 parts of 8 heads of 128 took 40 us.
  if constexpr (SPLIT) {
    constexpr int kPart = kHeads * (D + 2), kThreads = 64 * W, kPer = kMostSplits / (4 * W), kJoin = NT < 8 ? 16 : 8;
    const uint32_t part_bytes = kPart * 4;
    float* parts = a.partial + (int64_t)unit * a.splits * kPart;
    const auto memory = __builtin_amdgcn_make_buffer_rsrc(parts, 0, a.splits * part_bytes, kBufferFlags);
    if (wave == 0 && col < heads_here) {
      const uint32_t at = (uint32_t)split * part_bytes;
      if (g == 0) {
        __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(top), memory, at + col * 4, 0, kAcrossDies);
        __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(sum), memory, at + (kHeads + col) * 4, 0, kAcrossDies);
      }
#pragma unroll
      for (int u = 0; u < kOut / 4; ++u) {
        f32x4 x;
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = acc[(u * 4 + e) % (2 * NT)][(u * 4 + e) / (2 * NT)];
        __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, x), memory, at + (2 * kHeads + col * D + g * kOut + u * 4) * 4, 0, kAcrossDies);
      }
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // they are where every die sees them
    }
    __shared__ int is_last;
    __syncthreads();
    if (threadIdx.x == 0) is_last = atomicAdd(&a.arrived[unit], 1u) == (uint32_t)active - 1u;
    __syncthreads();
    if (!is_last) return;
    if (threadIdx.x == 0) a.arrived[unit] = 0;

    // lane 16 g + c of wavefront w: head c of parts 4 (w + W k) + g
    float tops[kPer], sums[kPer];
#pragma unroll
    for (int k = 0; k < kPer; ++k) {
      const int s = min(4 * (wave + W * k) + g, active - 1);
      tops[k] = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(memory, s * part_bytes + col * 4, 0, kAcrossDies));
      sums[k] = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(memory, s * part_bytes + (kHeads + col) * 4, 0, kAcrossDies));
    }
    // an output of four elements per thread; where there are fewer than threads, several share one
    const int outputs = heads_here * D / 4, sharers = max(1, kThreads / outputs);
    const int e0 = (int)threadIdx.x % (outputs * sharers) % outputs, sharer = (int)threadIdx.x / outputs;
    u32x4 next[kJoin];
    auto fetch = [&](int e, int first) {
#pragma unroll
      for (int k = 0; k < kJoin; ++k)
        next[k] = __builtin_amdgcn_raw_buffer_load_b128(memory, min(first + k * sharers, active - 1) * part_bytes + (2 * kHeads + e * 4) * 4, 0, kAcrossDies);
    };
    fetch(e0, sharer);
    float m = -INFINITY, l = 0.0f;
#pragma unroll
    for (int k = 0; k < kPer; ++k) m = fmaxf(m, tops[k]);
    m = across_groups_max(m);
    if (g == 0) joined_m[wave][col] = m;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < W; ++w) m = fmaxf(m, joined_m[w][col]);
    const float from = m > -INFINITY ? m : 0.0f;
#pragma unroll
    for (int k = 0; k < kPer; ++k) {
      tops[k] = 4 * (wave + W * k) + g < active ? __builtin_amdgcn_exp2f(tops[k] - from) : 0.0f;
      l += sums[k] * tops[k];
    }
    l = across_groups_sum(l);
    if (g == 0) joined_l[wave][col] = l;
    __syncthreads();
    l = 0.0f;
#pragma unroll
    for (int w = 0; w < W; ++w) l += joined_l[w][col];
    const float inverse = 1.0f / l;
    float* weights = joined_o;   // [kMostSplits][kHeads]
#pragma unroll
    for (int k = 0; k < kPer; ++k) weights[(4 * (wave + W * k) + g) * kHeads + col] = tops[k] * inverse;
    if (a.lse && wave == 0 && g == 0 && col < heads_here) a.lse[(int64_t)i * a.heads + head0 + col] = (m + __log2f(l)) * kLn2;
    __syncthreads();
    f32x4* shared_out = (f32x4*)(joined_o + kMostSplits * kHeads);   // [kThreads]
    if (sharers == 1 && sharer > 0) return;   // threads left over
    for (int e = e0; e < outputs; e += kThreads) {
      const int h = e * 4 / D;
      f32x4 x = {0, 0, 0, 0};
      if (sharer < sharers) {
        for (int s = sharer;;) {
#pragma unroll
          for (int k = 0; k < kJoin; ++k) {
            const int at = s + k * sharers;
            const float w = at < active ? weights[at * kHeads + h] : 0.0f;
            x += at < active ? __builtin_bit_cast(f32x4, next[k]) * w : f32x4{0, 0, 0, 0};
          }
          s += kJoin * sharers;
          if (s >= active) break;
          fetch(e, s);
        }
      }
      if (sharers > 1) {   // (then this loop has one turn)
        shared_out[threadIdx.x] = x;
        __syncthreads();
        if (sharer > 0) return;
        for (int k = 1; k < sharers; ++k) x += shared_out[threadIdx.x + k * outputs];
      } else if (e + kThreads < outputs) {
        fetch(e + kThreads, sharer);
      }
      typename T::elem* out = (typename T::elem*)(a.out + i * a.out_entry + (head0 + h) * a.out_head) + e * 4 % D;
      float y[4] = {x[0], x[1], x[2], x[3]};
      within_type<T, EIGHT>(y);
#pragma unroll
      for (int k = 0; k < 4; ++k) out[k] = (typename T::elem)y[k];
    }
  }
}

// ---- keys and values in 8 bits, and reading back (pgxcache8.hip) ---------------------------------------------------------------------------
int64_t write8_blocks(const Cache& c, int n, int tokens);
// last_only: the one token given is the slots' last, not the first of those that the last advance made room for
hipError_t write8(const Cache& c, bool f16, int layer, int n, const int32_t* slots, int tokens, int last_only, const Tokens& k, const Tokens& v, hipStream_t stream);
bool attend8_fits(const Cache& c, const AttendArgs& a);   // into a launch
hipError_t attend8(const Cache& c, bool f16, const AttendArgs& a, hipStream_t stream);
int64_t read_blocks(const Cache& c, int n, int tokens);
hipError_t read_back(const Cache& c, bool f16, int layer, int n, const int32_t* slots, const int32_t* firsts, int first, int tokens, const Tokens& k, const Tokens& v,
                     hipStream_t stream);

}  // namespace pgxcache_parts

#endif  // CACHE_COMMON_HPP_
