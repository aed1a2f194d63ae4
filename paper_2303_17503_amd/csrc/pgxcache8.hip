// pgxcache8.hip -- keys and values held in 8 bits (include/pgxcache.h): rounding them as they are written, attention over them, reading them back, gfx950.
//
// An element is an e4m3 number times the scale of its block: 16 tokens of a slot (beginning with a multiple of 16) in one layer and head, keys or
// values.  A head's block is one run of 16 head_dim bytes, half the rows of a matrix tile of attention, so that a wavefront knows its scale as one number.
//
// Bound by the bytes where there are many.  Measured, bfloat16, 2 heads of 64 unless said: attention of 4096 slots of 1 to 722 tokens 74 to 77 us, 5.2 TB/s in runs of 1 KB at random places (over 16 bits 134), of 3
// sequences of 110000, 8 heads of 128 in float16, 110 to 126 us, 5.4 to 6.2 TB/s; of one slot of 722 6.2 us, a chain of round trips.  Writing 256 prompts of 60 to 500 tokens 17 us, 3.3 TB/s (a chain of
// round trips for 2 KB, and wavefronts for the longest prompt's blocks, of which 44 % find no token); one
// token in each of 4096 slots 7.5 us (list, length, page, scale, block: a round trip each).  Reading 1024 slots of 1 to 722 tokens back 94 to 96 us, 5.0 TB/s.
#include "cache_common.hpp"

namespace pgxcache_parts {
namespace {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

constexpr int kBlock = 1 << kBlockShift;   // tokens of a block
int blocks_of(int tokens) { return (int)(((int64_t)tokens + kBlock - 2) / kBlock + 1); }   // that so many tokens can lie in
// Blocks that a wavefront of a write takes one after the other: all of an entry's where these are up to four and there are more than the machine's 8192 wavefronts hold at once, since
// most of them have no token (4096 entries of 8 to 16 tokens, 2 heads of 64: 11.9 us, by a wavefront for each block 19.5; 2048 of 20 to 40 14.8 / 20.8), otherwise one (256 of 60 to 500
// tokens 17.0 us, by runs of four blocks 20.7).
int blocks_per_run(const Cache& c, int n, int tokens) {
  const int64_t blocks = (int64_t)n * blocks_of(tokens) * 2 * c.kv_heads;
  return blocks >= 16384 && blocks_of(tokens) <= 4 ? blocks_of(tokens) : 1;
}
int runs_of(const Cache& c, int n, int tokens) { return (blocks_of(tokens) + blocks_per_run(c, n, tokens) - 1) / blocks_per_run(c, n, tokens); }

__device__ __forceinline__ int64_t scale_index(const Cache& c, int64_t page, int layer, int which) {   // which: keys of all heads, then values
  return page * c.page_scales() + ((int64_t)layer * 2 * c.kv_heads + which) * c.page_blocks();
}

// The scale for a largest magnitude m: the smallest power of two with m <= 448 of it (1.75 2^8), no smaller than 2^-100.
__device__ __forceinline__ float scale_for(float m) {
  const int e = (int)((__float_as_uint(m) + 0x1FFFFFu) >> 23) - 8;   // one up where the fraction is above 1.75
  return __uint_as_float((uint32_t)max(e, 27) << 23);
}
__device__ __forceinline__ bool finite(float x) { return fabsf(x) <= 0x1.fffffep127f; }

__device__ __forceinline__ float reciprocal(float scale) { return __builtin_amdgcn_rcpf(scale); }   // exact for powers of two

template <class T>
__device__ __forceinline__ void unpack(const u32x4& w, float* x) {
  const typename T::x8 h = __builtin_bit_cast(typename T::x8, w);
#pragma unroll
  for (int j = 0; j < 8; ++j) x[j] = (float)h[j];
}
// eight e4m3 codes, to nearest, ties to even; what is not finite becomes NaN
__device__ __forceinline__ u32x2 encode(const float* x, float inverse) {
  float y[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) y[j] = finite(x[j]) ? x[j] * inverse : __builtin_nanf("");
  u32x2 w;
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    int v = __builtin_amdgcn_cvt_pk_fp8_f32(y[4 * j], y[4 * j + 1], 0, false);
    w[j] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y[4 * j + 2], y[4 * j + 3], v, true);
  }
  return w;
}
__device__ __forceinline__ void decode(const u32x2& w, float* x) {
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[j], false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[j], true);
    x[4 * j] = a[0]; x[4 * j + 1] = a[1]; x[4 * j + 2] = b[0]; x[4 * j + 3] = b[1];
  }
}
__device__ __forceinline__ float largest(const float* x, float m) {
#pragma unroll
  for (int j = 0; j < 8; ++j) m = fmaxf(m, finite(x[j]) ? fabsf(x[j]) : 0.0f);
  return m;
}
template <int DPP>
__device__ __forceinline__ float moved(float x) {   // lanes exchanged within each 16
  return __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(x), DPP, 0xF, 0xF, false));
}
// over the 32 lanes of a half of the wavefront: rotations within 16, then the other 16
__device__ __forceinline__ float half_max(float x) {
  x = fmaxf(x, moved<0x128>(x));
  x = fmaxf(x, moved<0x124>(x));
  x = fmaxf(x, moved<0x122>(x));
  x = fmaxf(x, moved<0x121>(x));
  return fmaxf(x, __shfl_xor(x, 16));
}

// A block's earlier tokens are rounded once more for a larger scale: `units` runs of 8 elements, `lanes` lanes, N at most for each, eight under way together.
template <int N>
__device__ __forceinline__ void round_again(char* block, int units, int lane, int lanes, float ratio) {
  constexpr int kAhead = N < 8 ? N : 8;
  for (int u0 = lane; u0 < units; u0 += lanes * kAhead) {
    u32x2 w[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) w[k] = *(const u32x2*)(block + min(u0 + k * lanes, units - 1) * 8);
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      float x[8];
      decode(w[k], x);
      if (u0 + k * lanes < units) *(u32x2*)(block + (u0 + k * lanes) * 8) = encode(x, ratio);
    }
  }
}

// ---- writing -----------------------------------------------------------------------------------------------------------------------------
// Several tokens: a wavefront for each head, keys or values, and block of tokens, or with MANY for `per` blocks one after the other, the next one's elements and page on their way.
template <class T, int NT, bool MANY>
__global__ void __launch_bounds__(256) write8_kernel(Cache c, int layer, int n, const int32_t* slots, int tokens, int runs, int per, Tokens k, Tokens v) {
  constexpr int D = NT * 32, kUnits = D / 8;   // units of 8 elements of a token
  const int lane = (int)threadIdx.x & 63, heads = 2 * c.kv_heads;
  const int64_t piece = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
  const int64_t entry_run = piece / heads;
  const int which = (int)(piece - entry_run * heads), i = (int)(entry_run / runs), run = (int)(entry_run - (int64_t)i * runs);
  if (i >= n) return;
  const int slot = slots ? slots[i] : i;
  if ((uint32_t)slot >= (uint32_t)c.slots) return;
  const int grown = c.grown[slot], first = c.length(slot) - grown, end = first + min(grown, tokens);
  if (grown <= 0 || first < 0) return;
  const int block0 = (first >> kBlockShift) + run * per, block_end = min(block0 + per, (end + kBlock - 1) >> kBlockShift);
  if (block0 >= block_end) return;
  const bool value = which >= c.kv_heads;
  const Tokens& from = value ? v : k;
  const char* p = from.p + (int64_t)i * from.entry + (value ? which - c.kv_heads : which) * from.head;
  const int32_t* row = c.row(slot);
  auto load = [&](int block, u32x4 (&raw)[NT], int& page) {
#pragma unroll
    for (int r = 0; r < NT; ++r) {
      const int u = lane + 64 * r, t = (block << kBlockShift) + u / kUnits;
      raw[r] = u32x4{0, 0, 0, 0};
      if (t >= first && t < end) raw[r] = *(const u32x4_2*)(p + (int64_t)(t - first) * from.token + u % kUnits * 16);
    }
    page = row[block >> (c.page_shift - kBlockShift)];
  };
  auto write = [&](int block, const u32x4 (&raw)[NT], int page) {
    if (!c.is_page(page)) return;
    const int t0 = block << kBlockShift;
    char* to = c.kv + page * c.page_bytes(1) + ((int64_t)layer * 2 * c.kv_heads + which) * c.head_bytes(1) + (int64_t)(t0 & ((1 << c.page_shift) - 1)) * D;
    float* scale = c.scales + scale_index(c, page, layer, which) + (block & (c.page_blocks() - 1));
    const bool had = first > t0;
    const float was = had ? *scale : 0.0f;
    float x[NT][8], m = 0.0f;
#pragma unroll
    for (int r = 0; r < NT; ++r) {
      unpack<T>(raw[r], x[r]);
      m = largest(x[r], m);
    }
    m = half_max(m);
    m = fmaxf(m, __shfl_xor(m, 32));
    const float own = scale_for(m), now = had && was >= own ? was : own, inverse = reciprocal(now);
#pragma unroll
    for (int r = 0; r < NT; ++r) {
      const int u = lane + 64 * r, t = t0 + u / kUnits;
      if (t >= first && t < end) *(u32x2*)(to + u * 8) = encode(x[r], inverse);
    }
    if (had && now != was) round_again<NT>(to, (first - t0) * kUnits, lane, 64, was / now);
    if (lane == 0 && !(had && now == was)) *scale = now;
  };
  u32x4 raw[2][NT];
  int page[2];
  load(block0, raw[0], page[0]);
  if (!MANY) {
    write(block0, raw[0], page[0]);
    return;
  }
  for (int block = block0;; block += 2) {
    const bool second = block + 1 < block_end;
    if (second) load(block + 1, raw[1], page[1]);
    write(block, raw[0], page[0]);
    if (!second) break;
    const bool third = block + 2 < block_end;
    if (third) load(block + 2, raw[0], page[0]);
    write(block + 1, raw[1], page[1]);
    if (!third) break;
  }
}

// One token: as many lanes as it has runs of 8 elements, or the next power of two, for each entry, head and keys or values; its elements are on their way while its place is
// looked up.
template <class T, int NT>
__global__ void __launch_bounds__(256) write8_one_kernel(Cache c, int layer, int n, const int32_t* slots, int last, Tokens k, Tokens v) {
  constexpr int D = NT * 32, kUnits = D / 8, kGroup = kUnits <= 4 ? 4 : kUnits <= 8 ? 8 : kUnits <= 16 ? 16 : 32;
  const int u = (int)threadIdx.x % kGroup, heads = 2 * c.kv_heads;
  const int64_t piece = (int64_t)blockIdx.x * (256 / kGroup) + (int)threadIdx.x / kGroup;
  const int entry = (int)(piece / heads), which = (int)(piece - (int64_t)entry * heads), i = min(entry, n - 1);
  const bool value = which >= c.kv_heads;
  const Tokens& from = value ? v : k;
  u32x4 raw = {0, 0, 0, 0};
  if (u < kUnits) raw = *(const u32x4_2*)(from.p + (int64_t)i * from.entry + (value ? which - c.kv_heads : which) * from.head + u * 16);
  const int slot = slots ? slots[i] : i;
  const bool is_slot = entry < n && (uint32_t)slot < (uint32_t)c.slots;
  const int at_slot = is_slot ? slot : 0, length = c.length(at_slot), grown = c.grown[at_slot], t = length - (last ? 1 : grown);
  const bool there = is_slot && grown > 0 && t >= 0;
  const int page = c.row(at_slot)[there ? t >> c.page_shift : 0];
  const bool writes = there && c.is_page(page);
  float* scale = c.scales + scale_index(c, writes ? page : 0, layer, which) + (t >> kBlockShift & (c.page_blocks() - 1));
  const int before = t & (kBlock - 1);
  const float was = writes && before > 0 ? *scale : 0.0f;
  float x[8];
  unpack<T>(raw, x);
  float m = largest(x, 0.0f);   // (over the group: neighbours first, then mirrored, when halves are alike)
  m = fmaxf(m, moved<0xB1>(m));
  m = fmaxf(m, moved<0x4E>(m));
  if (kGroup >= 8) m = fmaxf(m, moved<0x141>(m));
  if (kGroup >= 16) m = fmaxf(m, moved<0x140>(m));
  if (kGroup >= 32) m = fmaxf(m, __shfl_xor(m, 16));
  if (!writes) return;
  const float own = scale_for(m), now = before > 0 && was >= own ? was : own;
  char* to = c.kv + page * c.page_bytes(1) + ((int64_t)layer * 2 * c.kv_heads + which) * c.head_bytes(1) + (int64_t)(t & ((1 << c.page_shift) - 1) & ~(kBlock - 1)) * D;
  if (u < kUnits) *(u32x2*)(to + before * D + u * 8) = encode(x, reciprocal(now));
  if (before == 0 || now != was) {
    if (before > 0) round_again<15>(to, before * kUnits, u, kGroup, was / now);
    if (u == 0) *scale = now;
  }
}

// ---- reading back: a thread per 8 elements of a head's key or value and four tokens; both ways of holding them ----------------------------
constexpr int kTokensPerThread = 4;
template <class T, bool EIGHT>
__global__ void __launch_bounds__(256) read_kernel(Cache c, int layer, int n, const int32_t* slots, const int32_t* firsts, int first_of_all, int tokens, Tokens k, Tokens v) {
  const uint32_t units = (uint32_t)c.head_dim / 8, per_entry = 2u * (uint32_t)c.kv_heads * units;
  const int64_t x = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const uint32_t runs = (uint32_t)(tokens + kTokensPerThread - 1) / kTokensPerThread;
  const int64_t token_run = x / per_entry;
  const uint32_t u = (uint32_t)(x - token_run * per_entry);
  if (token_run >= (int64_t)n * runs) return;
  const int i = (int)(token_run / runs), j0 = (int)(token_run - (int64_t)i * runs) * kTokensPerThread;
  const int slot = slots ? slots[i] : i;
  const bool is_slot = (uint32_t)slot < (uint32_t)c.slots;
  const int length = is_slot ? c.length(slot) : 0;
  const int64_t first = firsts ? firsts[i] : first_of_all;
  const uint32_t which = u / units, at = u % units * 8;   // which: keys of all heads, then values
  const bool value = which >= (uint32_t)c.kv_heads;
  const uint32_t head = value ? which - (uint32_t)c.kv_heads : which;
  const Tokens& to = value ? v : k;
  char* p = (char*)to.p + i * to.entry + head * to.head + at * 2;
  const int32_t* row = c.row(is_slot ? slot : 0);
  const char* from = c.kv + ((int64_t)layer * 2 * c.kv_heads + which) * c.head_bytes(EIGHT ? 1 : 2) + at * (EIGHT ? 1 : 2);
  int page[kTokensPerThread];
#pragma unroll
  for (int j = 0; j < kTokensPerThread; ++j) {
    const int64_t t = first + j0 + j;
    page[j] = t >= 0 && t < length ? row[t >> c.page_shift] : -1;
  }
  u32x4 data[kTokensPerThread];
  float scale[kTokensPerThread];
#pragma unroll
  for (int j = 0; j < kTokensPerThread; ++j) {
    const int t = (int)(first + j0 + j);
    scale[j] = 0.0f;
    if (EIGHT && c.is_page(page[j])) scale[j] = c.scales[scale_index(c, page[j], layer, (int)which) + (t >> kBlockShift & (c.page_blocks() - 1))];
  }
#pragma unroll
  for (int j = 0; j < kTokensPerThread; ++j) {
    const int t = (int)(first + j0 + j);
    data[j] = u32x4{0, 0, 0, 0};
    if (!c.is_page(page[j])) continue;
    const char* source = from + page[j] * c.page_bytes(EIGHT ? 1 : 2) + (int64_t)(t & ((1 << c.page_shift) - 1)) * c.head_dim * (EIGHT ? 1 : 2);
    if (EIGHT) {
      const u32x2 w = *(const u32x2*)source;
      data[j][0] = w[0];
      data[j][1] = w[1];
    } else {
      data[j] = *(const u32x4*)source;
    }
  }
  // A code times its scale may lie beyond the type's end where the value that it stands for did not: then it is the largest number.  Scales are asked for first, so that one look at
  // them chooses for the wavefront while the elements are on their way (1024 slots of 1 to 722 tokens 94.5 us; a look per token 98.5, comparing every element 102).
  auto store = [&](auto within) __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < kTokensPerThread; ++j) {
      if (j0 + j >= tokens) break;
      u32x4 x = data[j];
      if (EIGHT) {
        float y[8];
        decode(u32x2{data[j][0], data[j][1]}, y);
        typename T::x8 h;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          y[e] *= scale[j];
          if (within.value) y[e] = y[e] > T::kLargest ? T::kLargest : y[e] < -T::kLargest ? -T::kLargest : y[e];   // (NaN stays)
          h[e] = (typename T::elem)y[e];
        }
        x = __builtin_bit_cast(u32x4, h);
      }
      *(u32x4_2*)(p + (int64_t)(j0 + j) * to.token) = x;
    }
  };
  if (EIGHT && __any(fmaxf(fmaxf(scale[0], scale[1]), fmaxf(scale[2], scale[3])) > T::kLargest / 448.0f)) store(std::true_type{});
  else store(std::false_type{});
}

// ---- attention of one token per entry ----------------------------------------------------------------------------------------------------
// The products of attention over 16 bits (pgxcache.hip) on codes that are turned into 16-bit numbers, exactly, on their way into the matrix instructions:
// keys into the type of the queries, values into bfloat16, whose range holds probabilities times any scale.  Scores are multiplied by their block's scale,
// probabilities by that of the values.  A tile is 32 tokens, two blocks.  The contraction of the first product may run over the elements in any order that both
// operands share: a lane takes 16 neighbouring elements of its key at once, for two matrix instructions.
template <int NT>
struct Tile8 {
  uint32_t k[2][2 * NT], v[8][(NT + 1) / 2];
};
template <class T>
struct Decoded;
template <>
struct Decoded<BF16> {
  static __device__ __forceinline__ uint32_t low(uint32_t w) { return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, false)); }
  static __device__ __forceinline__ uint32_t high(uint32_t w) { return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, true)); }
};
template <>
struct Decoded<F16> {
  static __device__ __forceinline__ uint32_t low(uint32_t w) { return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.0f, false)); }
  static __device__ __forceinline__ uint32_t high(uint32_t w) { return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.0f, true)); }
};

// where the 8 elements begin that group g of the m-th instruction of the first product takes
template <int NT>
__device__ __forceinline__ constexpr int key_element(int m, int g) { return (NT & 1) && m == NT - 1 ? m * 32 + g * 8 : m / 2 * 64 + g * 16 + (m & 1) * 8; }

// W wavefronts share a row: an entry, a key head and a tile of 16 query heads.  SPLIT: a row may be split over blocks.  STREAM: keys and values are read with the hint
// that they are not read again soon.
template <class T, int NT, int W, int BUF, bool SPLIT, bool STREAM>
__global__ void __launch_bounds__(64 * W, BUF == 2 && NT == 8 ? 1 : 2) attend8_kernel(Cache c, AttendArgs a) {
  typedef typename T::x8 x8;
  typedef typename BF16::x8 v8;
  constexpr int D = NT * 32, kOut = 8 * NT;   // elements of the output per lane
  const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), lane = (int)threadIdx.x & 63, col = lane & 15, g = lane >> 4;
  // What runs together reads neighbouring memory: heads are next to each other in the launch, then the parts of a sequence.  Blocks go to the eight dies in turn, so with
  // by_die the heads of a part are eight blocks apart: the tiles of query heads of one key head find its keys and values in one die's L2 (201 slots of up to 4001 tokens, 20 heads of
  // 256 on one key head: 217 MB read from memory and not twice that), and the key heads the lines that hold their scales.
  const uint32_t per_part = (uint32_t)(c.kv_heads * a.head_tiles);
  uint32_t part, in_part;
  if (a.by_die) {
    const uint32_t eight = blockIdx.x / (8u * per_part), inside = blockIdx.x - eight * 8u * per_part;
    in_part = inside >> 3;
    part = eight * 8 + (inside & 7);
    if (part >= (uint32_t)(a.n * a.splits)) return;
  } else {
    part = blockIdx.x / per_part;
    in_part = blockIdx.x - part * per_part;
  }
  const int i = SPLIT ? (int)(part / (uint32_t)a.splits) : (int)part, split = SPLIT ? (int)(part - (uint32_t)i * (uint32_t)a.splits) : 0;
  const int kv_head = (int)(in_part / (uint32_t)a.head_tiles), head_tile = (int)(in_part - (uint32_t)(kv_head * a.head_tiles));
  const uint32_t unit = ((uint32_t)i * (uint32_t)c.kv_heads + (uint32_t)kv_head) * (uint32_t)a.head_tiles + (uint32_t)head_tile;
  const int slot = a.slots ? a.slots[i] : i;
  const bool is_slot = (uint32_t)slot < (uint32_t)c.slots;
  const int heads_here = min(kHeads, a.group - head_tile * kHeads), head0 = kv_head * a.group + head_tile * kHeads;

  // what depends on the entry only is asked for first, beside the slot's length
  u32x4 query[NT], fresh = {0, 0, 0, 0};
#pragma unroll
  for (int m = 0; m < NT; ++m) query[m] = *(const u32x4_2*)(a.q + i * a.q_entry + (head0 + min(col, heads_here - 1)) * a.q_head + key_element<NT>(m, g) * 2);
  const bool writes = (lane & 31) < D / 8;   // the new token: its key in the lower lanes, its value in the upper ones
  if (a.k && writes) fresh = *(const u32x4_2*)((lane < 32 ? a.k + i * a.k_entry + kv_head * a.k_head : a.v + i * a.v_entry + kv_head * a.v_head) + (lane & 31) * 16);
  const int32_t* row = c.row(is_slot ? slot : 0);
  // page of half-tile lane & 1 of the wavefront's tile number (a multiple of 32) + lane / 2; the first ones are asked for before the length is known
  int ids = 0;
  if (!SPLIT) ids = row[min((((wave + (lane >> 1) * W) * 2 + (lane & 1)) << 4) >> c.page_shift, c.width - 1)];
  const int length = is_slot ? c.length(slot) : 0, grown = a.k && is_slot ? c.grown[slot] : 0;

  if (length == 0) {   // nothing to attend to
    if (split == 0 && wave == 0 && col < heads_here) {
      char* out = a.out + i * a.out_entry + (head0 + col) * a.out_head + g * kOut * 2;
#pragma unroll
      for (int u = 0; u < NT; ++u) *(u32x4_2*)(out + u * 16) = u32x4{0, 0, 0, 0};
      if (a.lse && g == 0) a.lse[(int64_t)i * a.heads + head0 + col] = -INFINITY;
    }
    return;
  }
  const int tiles = (int)(((int64_t)length + 31) >> 5);
  const int chunk = SPLIT ? ((tiles + a.splits - 1) / a.splits + W - 1) / W * W : tiles, active = SPLIT ? (tiles + chunk - 1) / chunk : 1;
  if (SPLIT && split >= active) return;
  const int begin = split * chunk, end = min(tiles, begin + chunk);

  const int64_t page_bytes = c.page_bytes(1), head_bytes = c.head_bytes(1), page_scales = c.page_scales();
  const char* keys = c.kv + ((int64_t)a.layer * 2 * c.kv_heads + kv_head) * head_bytes;
  const char* values = keys + c.kv_heads * head_bytes;
  float* key_scales = c.scales + ((int64_t)a.layer * 2 * c.kv_heads + kv_head) * c.page_blocks();
  float* value_scales = key_scales + c.kv_heads * c.page_blocks();
  const int in_page = (1 << c.page_shift) - 1, in_blocks = c.page_blocks() - 1;

  const bool alone = W > 1 && tiles <= 1;   // nothing to share: the first wavefront goes on by itself
  if (alone && wave > 0) return;

  x8 q[NT];
#pragma unroll
  for (int m = 0; m < NT; ++m) q[m] = __builtin_bit_cast(x8, col < heads_here ? query[m] : u32x4{0, 0, 0, 0});

  float top = -INFINITY, sum = 0.0f;   // of the lane's head: the exponent that all four groups use, and this group's sum
  f32x4 acc[2 * NT];
#pragma unroll
  for (int m = 0; m < 2 * NT; ++m) acc[m] = f32x4{0, 0, 0, 0};

  const int mine = (end - begin - wave + W - 1) / W;   // this wavefront's tiles
  const int last_half = (length - 1) >> 4;
  uint64_t pages_there = 0;   // which of the pages in ids are pages (behind the sequence, and where the table is wrong: what is read there is page 0's and does not count)
  auto take_pages = [&](int p) {
    pages_there = __ballot(c.is_page(p));
    ids = c.is_page(p) ? p : 0;
  };
  take_pages(ids);
  // Scales of the half-tiles whose pages are in ids.  They are asked for ahead of the tile's keys and values and taken over behind them: a register that a load may
  // still be on its way to would have every tile wait for all loads.
  float asked_key_scale = 0.0f, asked_value_scale = 0.0f, key_scale = 0.0f, value_scale = 0.0f;
  auto lane_of = [](float x, int at) { return __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(x), at)); };
  auto look_up = [&](int number) {   // pages and scales of the wavefront's tiles number to number + 31
    const int half = (begin + wave + (number + (lane >> 1)) * W) * 2 + (lane & 1);
    if (SPLIT || number > 0) take_pages(row[(min(half, last_half) << 4) >> c.page_shift]);
    const int64_t at = ids * page_scales + (half & in_blocks);
    asked_key_scale = key_scales[at];
    asked_value_scale = value_scales[at];
  };
  auto take_over = [&](int number) {
    const int half = (begin + wave + (number + (lane >> 1)) * W) * 2 + (lane & 1);
    key_scale = asked_key_scale * a.scale;
    value_scale = half <= last_half ? asked_value_scale : 0.0f;   // (a block behind the last token may have any scale)
  };
  // The new token goes into the cache ahead of the loads of the last tile, by the wavefront that reads that (nobody else reads its block, and a
  // wavefront's own memory operations are in order), beside its first tile's on their way.
  const bool renews = grown > 0 && mine > 0 && end == tiles && wave == (tiles - 1 - begin) % W;
  auto renew = [&](const float* x, float own) {   // the elements, and the scale that they ask for
    const int at = length - 1, before = at & (kBlock - 1), half = (mine - 1) * 2 + (at >> kBlockShift & 1);   // (of the first 32 tiles: a lane's)
    const bool near = half < 64;
    const int page = near ? (pages_there >> half & 1 ? __builtin_amdgcn_readlane(ids, half) : -1) : row[at >> c.page_shift];
    if (!c.is_page(page)) return;
    const int64_t scale_at = page * page_scales + (at >> kBlockShift & in_blocks);
    char* block = (char*)(lane < 32 ? keys : values) + page * page_bytes + (int64_t)(at & in_page & ~(kBlock - 1)) * D;
    const float was = near ? (lane < 32 ? lane_of(asked_key_scale, half) : lane_of(asked_value_scale, half)) : (lane < 32 ? key_scales : value_scales)[scale_at];
    const float now = before > 0 && was >= own ? was : own;
    if (writes) *(u32x2*)(block + before * D + (lane & 31) * 8) = encode(x, reciprocal(now));
    if (before == 0 || now != was) {
      if (before > 0) round_again<2 * NT>(block, before * (D / 8), lane & 31, 32, was / now);
      if ((lane & 31) == 0) (lane < 32 ? key_scales : value_scales)[scale_at] = now;
    }
    const float key_now = lane_of(now, 0), value_now = lane_of(now, 32);
    key_scale = lane == half ? key_now * a.scale : key_scale;
    value_scale = lane == half ? value_now : value_scale;
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  };
  auto load_half = [&](int number, int h) { return (int64_t)__builtin_amdgcn_readlane(ids, (number & 31) * 2 + h) * page_bytes + (int64_t)(((begin + wave + number * W) * 32 + h * 16) & in_page) * D; };
  auto load_keys = [&](Tile8<NT>& t, int number) {   // of the wavefront's tile of that number
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const char* k = keys + load_half(number, h) + col * D;
#pragma unroll
      for (int m = 0; m < NT / 2; ++m) {
        const u32x4 w = read_once<STREAM>((const u32x4*)(k + m * 64 + g * 16));
#pragma unroll
        for (int e = 0; e < 4; ++e) t.k[h][m * 4 + e] = w[e];
      }
      if (NT & 1) {
        const u32x2 w = read_once<STREAM>((const u32x2*)(k + (NT - 1) * 32 + g * 8));
        t.k[h][2 * NT - 2] = w[0];
        t.k[h][2 * NT - 1] = w[1];
      }
    }
  };
  auto load_values = [&](Tile8<NT>& t, int number) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const char* v = values + load_half(number, h) + (g * 4 * D + col * NT * 2);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        uint32_t* to = t.v[h * 4 + j];
        if constexpr (NT == 8) {
          const u32x4 w = read_once<STREAM>((const u32x4*)(v + j * D));
          to[0] = w[0]; to[1] = w[1]; to[2] = w[2]; to[3] = w[3];
        } else if constexpr (NT == 4) {
          const u32x2 w = read_once<STREAM>((const u32x2*)(v + j * D));
          to[0] = w[0]; to[1] = w[1];
        } else if constexpr (NT == 3) {   // (6 bytes from an even address)
          const uint16_t* w = (const uint16_t*)(v + j * D);
          to[0] = read_once<STREAM>(w) | (uint32_t)read_once<STREAM>(w + 1) << 16;
          to[1] = read_once<STREAM>(w + 2);
        } else if constexpr (NT == 2) {
          to[0] = read_once<STREAM>((const uint32_t*)(v + j * D));
        } else {
          to[0] = read_once<STREAM>((const uint16_t*)(v + j * D));
        }
      }
    }
  };
  // BUF = 2: the next tile is under way while one is computed.  BUF = 1: its keys take the place of the present ones as soon as the scores are there, its values when
  // the present ones are added up.
  auto compute = [&](Tile8<NT>& t, Tile8<NT>& next, int number, auto last) {
    f32x4 s[2];
    float key_scales_here[2], value_scales_here[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      key_scales_here[h] = lane_of(key_scale, (number & 31) * 2 + h);
      value_scales_here[h] = lane_of(value_scale, (number & 31) * 2 + h);
    }
    auto turn = [&]() {
      if (((number + 1) & 31) == 0) {
        look_up(number + 1);
        take_over(number + 1);
      }
    };
    if (BUF == 2 && !last.value) {
      turn();
      load_keys(next, number + 1);
      load_values(next, number + 1);
    }
    s[0] = s[1] = f32x4{0, 0, 0, 0};
#pragma unroll
    for (int m = 0; m < NT; ++m)
#pragma unroll
      for (int h = 0; h < 2; ++h) {   // (two chains of products that do not wait for each other)
        const uint32_t w0 = t.k[h][2 * m], w1 = t.k[h][2 * m + 1];
        s[h] = T::mfma(__builtin_bit_cast(x8, u32x4{Decoded<T>::low(w0), Decoded<T>::high(w0), Decoded<T>::low(w1), Decoded<T>::high(w1)}), q[m], s[h]);
      }
#pragma unroll
    for (int h = 0; h < 2; ++h) s[h] *= key_scales_here[h];
    if (BUF == 1 && !last.value) {
      turn();
      load_keys(t, number + 1);
    }
    if (last.value) {   // tokens behind the sequence's last: no score, and their values may hold anything
      const int first = (begin + wave + number * W) * 32 + g * 4;
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const bool there = first + h * 16 + r < length;
          s[h][r] = there ? s[h][r] : -INFINITY;
#pragma unroll
          for (int w = 0; w < (NT + 1) / 2; ++w) t.v[h * 4 + r][w] = there ? t.v[h * 4 + r][w] : 0;
        }
    }
    const float most = fmaxf(fmaxf(fmaxf(s[0][0], s[0][1]), fmaxf(s[0][2], s[0][3])), fmaxf(fmaxf(s[1][0], s[1][1]), fmaxf(s[1][2], s[1][3])));
    if (__any(most > top + BF16::kMost)) {
      const float now = across_groups_max(fmaxf(most, top));
      const float factor = now > -INFINITY ? __builtin_amdgcn_exp2f(top - now) : 1.0f;
      top = now;
      sum *= factor;
#pragma unroll
      for (int m = 0; m < 2 * NT; ++m) acc[m] *= factor;
    }
    const float from = top > -INFINITY ? top : 0.0f;
    v8 high, low;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      float p = __builtin_amdgcn_exp2f(s[j >> 2][j & 3] - from);
      sum += p;
      p *= value_scales_here[j >> 2];
      high[j] = (__bf16)p;
      low[j] = (__bf16)(p - (float)high[j]);
    }
#pragma unroll
    for (int m = 0; m < NT; ++m) {   // elements 2 m and 2 m + 1 of the lane's 2 NT
      u32x4 x, y;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const uint32_t w = __builtin_amdgcn_perm(t.v[2 * j + 1][m / 2], t.v[2 * j][m / 2], m & 1 ? 0x07030602u : 0x05010400u);
        x[j] = Decoded<BF16>::low(w);
        y[j] = Decoded<BF16>::high(w);
      }
      acc[2 * m] = BF16::mfma(__builtin_bit_cast(v8, x), high, acc[2 * m]);
      acc[2 * m + 1] = BF16::mfma(__builtin_bit_cast(v8, y), high, acc[2 * m + 1]);
      acc[2 * m] = BF16::mfma(__builtin_bit_cast(v8, x), low, acc[2 * m]);
      acc[2 * m + 1] = BF16::mfma(__builtin_bit_cast(v8, y), low, acc[2 * m + 1]);
      if (NT == 8 && m % 2 == 1) __builtin_amdgcn_sched_barrier(0);   // (decoding far ahead of the products takes registers that are not there)
    }
    if (BUF == 1 && !last.value) load_values(t, number + 1);
  };
  if (mine > 0) {
    constexpr std::false_type inner{};
    constexpr std::true_type outer{};
    Tile8<NT> t0, t1;
    look_up(0);
    if (!renews || mine > 1) {
      load_keys(t0, 0);
      load_values(t0, 0);
    }
    float x[8], own = 0.0f;
    if (renews) {
      unpack<T>(fresh, x);
      own = scale_for(half_max(largest(x, 0.0f)));
    }
    take_over(0);
    if (renews) {
      renew(x, own);
      if (mine == 1) {
        load_keys(t0, 0);
        load_values(t0, 0);
      }
    }
    int number = 0;
    if constexpr (BUF == 1) {
      for (; number + 1 < mine; ++number) compute(t0, t0, number, inner);
      compute(t0, t0, number, outer);
    } else {
      for (; number + 2 < mine; number += 2) {
        compute(t0, t1, number, inner);
        compute(t1, t0, number + 1, inner);
      }
      if (number + 1 < mine) {
        compute(t0, t1, number, inner);
        compute(t1, t0, number + 1, outer);
      } else {
        compute(t0, t1, number, outer);
      }
    }
  }
  finish_row<T, NT, W, SPLIT, true>(a, Spot{wave, lane, col, g, i, head0, heads_here, split, active, unit, alone}, top, sum, acc);
}

// How an attend call is spread.
struct Spread {
  int waves, splits;   // wavefronts to a block, blocks to a row
  bool by_die;
  int64_t blocks;      // of the launch
};
Spread spread_of(const Cache& c, const AttendArgs& a) {
  // The lengths are known on the device only, so the choice goes by how long a slot can be and by the rows (2 key heads here, lengths from 1 up, us).
  //  * Up to 10 tiles of 32 tokens and from 1024 rows on a wavefront each (with 1, 2, 4 wavefronts: 1024 slots of up to 160 tokens, heads of 32 6.9 7.3 8.7, 64 7.4 8.1 10.2, 128 12.6 14.6
  //    22.1, 256 22 34 59; of up to 320, 64 11.8 12.5 13.4; 4096 of up to 320, 64 33.9 31.4 38.6, 128 75 77 100).
  //  * Up to 32 tiles and from 4096 rows on two (heads of 32, 64, 96, 128: 2048 slots of up to 400 17.7 22.9 31.3 38.2, with four 19.2 23.8 34.9 48.7, one 18.3 25.9 33.4 40.6; 4096 of up to 722 41.3
  //    84.2 156.6 160.7, with four 44.3 84.0 159.9 175.9, one 44.2 86.6 160.6 160.8; 1024 of up to 722 16.9 22.9 31.0 36.5, with four 16.6 20.2 29.5 36.6), but for heads of 32 and 64 below 6144 rows
  //    up to 16 tiles (2048 of up to 520 20.8 27.9 38.6 63.3, with four 22.2 27.4 40.5 71.1; of up to 722 25.7 38.1 76.7 81.9, with four 25.6 33.6 76.6 88.7; 3072 of up to 722 35.0 57.6 108.1 120.5, with
  //    four 37.6 58.7 109.5 132.2).  Heads of 256, whose four have a compute unit to
  //    themselves: from 256 rows on (200 of up to 722 27.9 20.7 24.7, 1024 81 82 105), and from 1024 on however long (1024 of up to 1500 157 149 167).
  //  * Otherwise four (200 slots of up to 722, 64 13.7 11.4 8.2; 64, 128 16.4 10.9 8.4; 1024 of up to 1500, 64 41.9 41.1 36.0, of 4000 126 122 102); eight take as long with few rows and
  //    longer with many (one of 722 6.8 / 6.9, 256 9.3 / 8.3, 1024 26 / 21).
  //  * Few rows that can be longer than 32 tiles are split over blocks, two for each compute unit at most (16 slots of 20000 tokens 20.8, with twice the blocks 27; 512
  //    slots of 2000 tokens in two blocks each 30.6, in one 23).
  const int64_t rows = (int64_t)a.n * c.kv_heads * a.head_tiles, most_tiles = (((int64_t)c.width << c.page_shift) + 31) / 32;
  Spread s{4, 1, false, 0};
  if (most_tiles > 32) {
    const int64_t spread = kSplitBlocks / rows, useful = (most_tiles + 7) / 8;
    const int64_t splits = spread < useful ? spread : useful;
    s.splits = (int)(splits < 1 ? 1 : splits > kMostSplits ? kMostSplits : splits);
  }
  if (s.splits == 1) {
    if (rows >= 1024 && most_tiles <= 10) s.waves = 1;
    else if (c.head_dim == 256 ? rows >= 1024 || (rows >= 256 && most_tiles <= 32) : rows >= 4096 && most_tiles <= (c.head_dim <= 64 && rows < 6144 ? 16 : 32)) s.waves = 2;
  }
  const int64_t parts = (int64_t)a.n * s.splits, heads = (int64_t)c.kv_heads * a.head_tiles;
  s.by_die = a.head_tiles > 1 || parts >= 64;
  s.blocks = s.by_die ? (parts + 7) / 8 * 8 * heads : parts * heads;
  return s;
}

template <class T, int NT, int W, int BUF, bool SPLIT>
hipError_t launch_attend_by(const Cache& c, const AttendArgs& a, int64_t blocks, hipStream_t stream) {
  const bool streamed = (int64_t)c.pages * c.page_bytes(1) > (int64_t)256 << 20;   // (as over 16 bits)
  const size_t join = (size_t)(W - 1) * kHeads * NT * 32 * 4, weights = SPLIT ? (size_t)kMostSplits * kHeads * 4 + 64 * W * 16 : 0;
  const dim3 grid((unsigned)blocks), block(64 * W);
  if (streamed) hipLaunchKernelGGL((attend8_kernel<T, NT, W, BUF, SPLIT, true>), grid, block, join > weights ? join : weights, stream, c, a);
  else hipLaunchKernelGGL((attend8_kernel<T, NT, W, BUF, SPLIT, false>), grid, block, join > weights ? join : weights, stream, c, a);
  return hipGetLastError();
}
template <class T, int NT>
hipError_t launch_attend(const Cache& c, AttendArgs a, hipStream_t stream) {
  const Spread s = spread_of(c, a);
  a.splits = s.splits;
  a.by_die = s.by_die;
  if (s.splits > 1) return launch_attend_by<T, NT, 4, NT < 8 ? 2 : 1, true>(c, a, s.blocks, stream);   // (heads of 256: 201 slots of 2000 tokens 45.5 us, with the next tile beside the present 54)
  if (s.waves == 1) return launch_attend_by<T, NT, 1, 2, false>(c, a, s.blocks, stream);
  if (s.waves == 2) return launch_attend_by<T, NT, 2, 2, false>(c, a, s.blocks, stream);
  return launch_attend_by<T, NT, 4, 2, false>(c, a, s.blocks, stream);
}

template <class T>
hipError_t attend8_for(const Cache& c, const AttendArgs& a, hipStream_t stream) {
  switch (c.head_dim) {
    case 32: return launch_attend<T, 1>(c, a, stream);
    case 64: return launch_attend<T, 2>(c, a, stream);
    case 96: return launch_attend<T, 3>(c, a, stream);
    case 128: return launch_attend<T, 4>(c, a, stream);
    default: return launch_attend<T, 8>(c, a, stream);
  }
}
template <class T, int NT>
hipError_t launch_write(const Cache& c, int layer, int n, const int32_t* slots, int tokens, int last_only, const Tokens& k, const Tokens& v, hipStream_t stream) {
  const dim3 grid((unsigned)write8_blocks(c, n, tokens)), block(256);
  if (tokens == 1) hipLaunchKernelGGL((write8_one_kernel<T, NT>), grid, block, 0, stream, c, layer, n, slots, last_only, k, v);
  else if (blocks_per_run(c, n, tokens) > 1) hipLaunchKernelGGL((write8_kernel<T, NT, true>), grid, block, 0, stream, c, layer, n, slots, tokens, 1, blocks_of(tokens), k, v);
  else hipLaunchKernelGGL((write8_kernel<T, NT, false>), grid, block, 0, stream, c, layer, n, slots, tokens, blocks_of(tokens), 1, k, v);
  return hipGetLastError();
}
template <class T>
hipError_t write8_for(const Cache& c, int layer, int n, const int32_t* slots, int tokens, int last_only, const Tokens& k, const Tokens& v, hipStream_t stream) {
  switch (c.head_dim) {
    case 32: return launch_write<T, 1>(c, layer, n, slots, tokens, last_only, k, v, stream);
    case 64: return launch_write<T, 2>(c, layer, n, slots, tokens, last_only, k, v, stream);
    case 96: return launch_write<T, 3>(c, layer, n, slots, tokens, last_only, k, v, stream);
    case 128: return launch_write<T, 4>(c, layer, n, slots, tokens, last_only, k, v, stream);
    default: return launch_write<T, 8>(c, layer, n, slots, tokens, last_only, k, v, stream);
  }
}

}  // namespace

int64_t write8_blocks(const Cache& c, int n, int tokens) {   // of the launch
  if (tokens > 1) return ((int64_t)n * runs_of(c, n, tokens) * 2 * c.kv_heads + 3) / 4;
  const int group = c.head_dim <= 32 ? 4 : c.head_dim <= 64 ? 8 : c.head_dim <= 128 ? 16 : 32;
  return ((int64_t)n * 2 * c.kv_heads * group + 255) / 256;
}
hipError_t write8(const Cache& c, bool f16, int layer, int n, const int32_t* slots, int tokens, int last_only, const Tokens& k, const Tokens& v, hipStream_t stream) {
  return f16 ? write8_for<F16>(c, layer, n, slots, tokens, last_only, k, v, stream) : write8_for<BF16>(c, layer, n, slots, tokens, last_only, k, v, stream);
}

bool attend8_fits(const Cache& c, const AttendArgs& a) {
  const Spread s = spread_of(c, a);
  return launchable(s.blocks, 64 * s.waves);
}
hipError_t attend8(const Cache& c, bool f16, const AttendArgs& a, hipStream_t stream) { return f16 ? attend8_for<F16>(c, a, stream) : attend8_for<BF16>(c, a, stream); }

int64_t read_blocks(const Cache& c, int n, int tokens) {
  const int64_t runs = ((int64_t)tokens + kTokensPerThread - 1) / kTokensPerThread;
  return ((int64_t)n * runs * 2 * c.kv_heads * (c.head_dim / 8) + 255) / 256;
}
hipError_t read_back(const Cache& c, bool f16, int layer, int n, const int32_t* slots, const int32_t* firsts, int first, int tokens, const Tokens& k, const Tokens& v, hipStream_t stream) {
  const dim3 grid((unsigned)read_blocks(c, n, tokens)), block(256);
  if (!c.scales) hipLaunchKernelGGL((read_kernel<BF16, false>), grid, block, 0, stream, c, layer, n, slots, firsts, first, tokens, k, v);   // (copies either type)
  else if (f16) hipLaunchKernelGGL((read_kernel<F16, true>), grid, block, 0, stream, c, layer, n, slots, firsts, first, tokens, k, v);
  else hipLaunchKernelGGL((read_kernel<BF16, true>), grid, block, 0, stream, c, layer, n, slots, firsts, first, tokens, k, v);
  return hipGetLastError();
}

}  // namespace pgxcache_parts
