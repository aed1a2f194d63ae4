// pgxcache.hip -- a paged cache of keys and values whose slots follow the environments' (include/pgxcache.h), gfx950.
//
// A page holds its tokens for all layers and heads, [layers][2][kv_heads][page_size][head_dim], so that a copied or moved page is one
// run of memory, and a head's tokens in a page are one run for attention.  Which pages are free is kept twice: as counters
// of the table entries that name a page (the caller's), and as a bit per page (work memory), which calls that give out pages look through.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>
#include <stdlib.h>

#include <new>
#include <type_traits>

#include "cache_common.hpp"
#include "rows_apart.hpp"

namespace {

using namespace pgxcache_parts;

thread_local int g_last_hip = 0;

#define HIPCHK(expr)                                   \
  do {                                                 \
    hipError_t e_ = (expr);                            \
    if (e_ != hipSuccess) {                            \
      g_last_hip = (int)e_;                            \
      return PGXCACHE_EHIP;                            \
    }                                                  \
  } while (0)

constexpr int kOneBlock = 1024;      // threads of the kernels that give out pages

// Pages that come free in a block.  Those of one word of the bits are gathered in LDS, so that a word is written once: pages given out together
// often come free together, and 64 blocks that each add one to the same word take 4 us.
struct Freed {
  static constexpr int kWords = 64;
  int key[kWords];
  unsigned long long mask[kWords];
  __device__ __forceinline__ void begin() {
    if (threadIdx.x < kWords) {
      key[threadIdx.x] = -1;
      mask[threadIdx.x] = 0;
    }
    __syncthreads();
  }
  __device__ __forceinline__ void release(const Cache& c, int p) {   // one table entry less names the page
    if (!c.is_page(p) || atomicSub(&c.refs[p], 1) != 1) return;
    const int w = p >> 6, k = w % kWords;
    const int was = atomicCAS(&key[k], -1, w);
    if (was == -1 || was == w) atomicOr(&mask[k], 1ull << (p & 63));
    else atomicOr((unsigned long long*)&c.free_bits[w], 1ull << (p & 63));
  }
  __device__ __forceinline__ void end(const Cache& c) {
    __syncthreads();
    if (threadIdx.x < kWords && mask[threadIdx.x]) atomicOr((unsigned long long*)&c.free_bits[key[threadIdx.x]], mask[threadIdx.x]);
  }
};

__global__ void __launch_bounds__(256) scan_refs_kernel(Cache c, uint32_t* arrived, int first) {   // first: the work memory holds nothing yet
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const uint64_t free = __ballot(i < c.pages && c.refs[min(i, (int64_t)c.pages - 1)] == 0);
  if ((threadIdx.x & 63) == 0 && i < ((int64_t)c.pages + 63) / 64 * 64) {
    c.free_bits[i >> 6] = free;
    c.taken[i >> 6] = 0;
  }
  if (first && i < c.slots) c.grown[i] = 0;
  if (first && i < kSplitBlocks) arrived[i] = 0;
}

// ---- giving out pages ----------------------------------------------------------------------------------------------------------------
// A call takes the lowest free pages, its entries in their order.  Which entry gets which follows from the free pages' bits and the
// needs of the entries before it, and every block of a planning kernel works both out for itself from memory that no one writes
// meanwhile (so a plan of n entries reads n^2 / 2048 of them: 65536 take 78 us); a second kernel then takes the pages out of the bits.  Bound by the round trips to memory that depend on each other (the list, the
// lengths it names; the bits beside them), so the bits are kept in LDS.  4096 entries of a pool of 143000 pages: one block that took the
// entries 1024 at a time and looked the bits up in memory took 40 us for a fork's plan; blocks of 1024 entries side by side take 8 to 10.
constexpr int kBitsInLds = 4096;   // words: pools of up to 262144 pages; beyond, the bits are looked up in memory

// sum over the threads before this one; *total: over all
template <class U>
__device__ __forceinline__ U exclusive_sum(U x, U* shared /* kOneBlock / 64 numbers */, U* total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  U s = x;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const U up = __shfl_up(s, d);
    if (lane >= d) s += up;
  }
  __syncthreads();
  if (lane == 63) shared[wave] = s;
  __syncthreads();
  U before = 0, all = 0;
#pragma unroll
  for (int w = 0; w < kOneBlock / 64; ++w) {
    const U v = shared[w];
    before += w < wave ? v : 0;
    all += v;
  }
  *total = all;
  return before + s - x;
}

// The free pages in ascending order.  Thread t has counted those in its stretch of the bits; at[t]: how many lie before it.
struct FreePages {
  const uint64_t* bits;
  uint64_t own[kBitsInLds / kOneBlock];   // this thread's words, while they are on their way to LDS
  int words, stretch;
  uint32_t* at;          // LDS, kOneBlock
  uint32_t count;

  // load() begins, ready() ends: what is done between the two waits for memory at the same time
  __device__ __forceinline__ void load(const Cache& c) {
    bits = c.free_bits;
    words = (c.pages + 63) / 64;
    stretch = (words + kOneBlock - 1) / kOneBlock;
    if (words <= kBitsInLds) {
#pragma unroll
      for (int k = 0; k < kBitsInLds / kOneBlock; ++k) {
        const int w = (int)threadIdx.x * stretch + k;
        own[k] = k < stretch && w < words ? bits[w] : 0;
      }
    }
  }
  __device__ __forceinline__ void ready(uint64_t* lds /* kBitsInLds */, uint32_t* at_, uint32_t* shared) {
    at = at_;
    uint32_t n = 0;
    if (words <= kBitsInLds) {
#pragma unroll
      for (int k = 0; k < kBitsInLds / kOneBlock; ++k) {
        if (k < stretch) lds[(int)threadIdx.x * stretch + k] = own[k];
        n += (uint32_t)__popcll(own[k]);
      }
      bits = lds;
    } else {
      for (int w = (int)threadIdx.x * stretch; w < min(words, ((int)threadIdx.x + 1) * stretch); ++w) n += (uint32_t)__popcll(bits[w]);
    }
    at[threadIdx.x] = exclusive_sum(n, shared, &count);
    __syncthreads();
  }
  // the place in `b` of its set bit with `left` set ones below it
  static __device__ __forceinline__ int place(uint64_t b, uint32_t left) {
    int bit = 0;
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) {
      const uint32_t low = (uint32_t)__popcll(b >> bit & ((1ull << d) - 1));
      if (left >= low) { left -= low; bit += d; }
    }
    return bit;
  }
  // the free page with `rank` free ones below it (rank < count)
  __device__ __forceinline__ int select(uint32_t rank) const {
    int t = 0;
#pragma unroll
    for (int d = kOneBlock / 2; d > 0; d >>= 1)
      if (at[t + d] <= rank) t += d;
    uint32_t left = rank - at[t];
    int w = t * stretch;
    uint64_t b = bits[w];
    while (left >= (uint32_t)__popcll(b)) {
      left -= (uint32_t)__popcll(b);
      b = bits[++w];
    }
    return w * 64 + place(b, left);
  }
  // the next free page above p (there has to be one)
  __device__ __forceinline__ int next(int p) const {
    int w = p >> 6;
    uint64_t b = (p & 63) == 63 ? 0 : bits[w] & ~0ull << ((p & 63) + 1);
    while (b == 0) b = bits[++w];
    return w * 64 + (int)__builtin_ctzll(b);
  }
  // the page in use with `rank` ones in use below it (there has to be one)
  __device__ __forceinline__ int select_used(uint32_t rank) const {
    int t = 0;
#pragma unroll
    for (int d = kOneBlock / 2; d > 0; d >>= 1)
      if ((t + d) * stretch < words && (uint32_t)((t + d) * stretch * 64) - at[t + d] <= rank) t += d;
    int w = t * stretch;
    uint32_t left = rank - ((uint32_t)(w * 64) - at[t]);
    uint64_t b = ~bits[w];
    while (left >= (uint32_t)__popcll(b)) {
      left -= (uint32_t)__popcll(b);
      b = ~bits[++w];
    }
    return w * 64 + place(b, left);
  }
  // f(word, its bits, those of them with ranks from lo to hi - 1) for the words of this thread's stretch that have such
  template <class F>
  __device__ __forceinline__ void ranks(uint32_t lo, uint32_t hi, F&& f) const {
    uint32_t before = at[threadIdx.x];
    for (int w = (int)threadIdx.x * stretch; w < min(words, ((int)threadIdx.x + 1) * stretch) && before < hi; ++w) {
      const uint64_t b = bits[w];
      const uint32_t n = (uint32_t)__popcll(b);
      if (before + n > lo) {
        uint64_t mask = b;
        if (before < lo) mask &= ~0ull << place(b, lo - before);
        if (before + n > hi) mask &= (1ull << place(b, hi - before)) - 1;
        if (mask) f(w, b, mask);
      }
      before += n;
    }
  }
  // free pages below page p
  __device__ __forceinline__ uint32_t below(int p) const {
    const int t = (p >> 6) / stretch;
    if (p >> 6 >= words) return count;
    uint32_t n = at[t];
    for (int w = t * stretch; w < p >> 6; ++w) n += (uint32_t)__popcll(bits[w]);
    return n + (uint32_t)__popcll(bits[p >> 6] & ((1ull << (p & 63)) - 1));
  }
};

struct Advance {   // what an entry of an advance call asks for
  int slot, more, length;
  uint32_t need;
  uint8_t said;
  bool is_slot;
};
__device__ __forceinline__ Advance asked(const Cache& c, int n, const int32_t* slots, const int32_t* counts, int count, int i) {
  Advance e;
  const bool entry = i < n;   // (loads without a condition: those of several entries are then under way together)
  const int at = min(i, n - 1);
  e.slot = slots ? slots[at] : at;
  e.more = counts ? counts[at] : count;
  e.is_slot = entry && (uint32_t)e.slot < (uint32_t)c.slots;
  e.length = c.length(e.is_slot ? e.slot : 0);
  if (!entry) e.slot = -1;
  e.need = 0;
  e.said = e.slot == -1 || (e.is_slot && e.more >= 0) ? 0 : PGXCACHE_BAD_ENTRY;
  if (e.is_slot && e.said == 0) {
    if ((int64_t)e.length + e.more > c.capacity()) e.said = PGXCACHE_FULL;
    else e.need = (uint32_t)(c.pages_of(e.length + e.more) - c.pages_of(e.length));
  }
  return e;
}
__device__ __forceinline__ void finish(const Cache& c, const Advance& e, bool done) {
  if (e.is_slot) c.grown[e.slot] = done ? e.more : 0;
  if (done && e.more > 0) c.lengths[e.slot] = e.length + e.more;
}
// PER = 1: a block per kOneBlock entries; one block ends the call itself, more are followed by advance_apply_kernel.  PER > 1: one block, PER
// neighbouring entries per thread, all their loads under way together, for up to 4096 entries that get one page each at most (a call of 4096 with
// one token more each: 10.4 us, by the two kernels 12.3, of 2048 8.8 / 11.1; with 0 to 39 tokens more: 32.3 by one block, 16.5 by the two kernels, of
// 2048 23.0 / 14.4).
// The pages that the entries get are the free ones of consecutive ranks (an entry that cannot have its pages is followed by others that cannot),
// so they leave the bits a word at a time (4600 pages, taken out one by one: 52 us, now 12).
constexpr uint32_t kWanted = 1536;
template <int PER, bool ALONE>
__global__ void __launch_bounds__(kOneBlock) advance_kernel(Cache c, int n, const int32_t* slots, const int32_t* counts, int count, int32_t* plan, uint8_t* status) {
  __shared__ uint64_t lds_bits[kBitsInLds];
  __shared__ uint32_t at[kOneBlock], shared[kOneBlock / 64], ends[kOneBlock], taken_end;
  __shared__ int32_t row_of[kOneBlock], have_of[kOneBlock];
  __shared__ int2 wanted[PER > 1 ? kWanted : 1];   // (slot, place in its row) of each page
  const int tid = (int)threadIdx.x, first = ALONE ? 0 : (int)blockIdx.x * kOneBlock;
  if (tid == 0) taken_end = 0;
  FreePages free;
  free.load(c);
  Advance e[PER];
#pragma unroll
  for (int k = 0; k < PER; ++k) e[k] = asked(c, n, slots, counts, count, first + tid * PER + k);
  // Needs of the entries before.  An entry needs 2^20 pages at most (the widest row), so a block's needs fit 32 bits; those of all earlier
  // blocks are added in 64 and cut off at 2^31, which no pool's pages reach.
  uint32_t before = 0, all, mine = 0;
  if constexpr (!ALONE) {
    __shared__ uint64_t shared_sums[kOneBlock / 64];
    uint64_t sum = 0, total;
    for (int k = 0; k < (int)blockIdx.x; ++k) sum += asked(c, n, slots, counts, count, k * kOneBlock + tid).need;
    exclusive_sum(sum, shared_sums, &total);
    before = (uint32_t)min(total, (uint64_t)1 << 31);
  }
#pragma unroll
  for (int k = 0; k < PER; ++k) mine += e[k].need;
  const uint32_t inside = exclusive_sum(mine, shared, &all);
  free.ready(lds_bits, at, shared);
  uint32_t rank = before + inside;
#pragma unroll
  for (int k = 0; k < PER; ++k) {
    const int i = first + tid * PER + k;
    const uint8_t said = e[k].need > 0 && (rank > free.count || e[k].need > free.count - rank) ? PGXCACHE_NO_PAGES : e[k].said;
    const bool done = e[k].is_slot && said == 0;
    if (status && i < n) status[i] = said;
    if (done && e[k].need > 0) {
      atomicMax(&taken_end, rank + e[k].need);
      if (PER > 1) {
        for (uint32_t j = 0; j < e[k].need; ++j) {
          const int place = c.pages_of(e[k].length) + (int)j;
          if (all <= kWanted) {
            wanted[rank - before + j] = make_int2(e[k].slot, place);
          } else {
            const int p = free.select(rank + j);
            c.row(e[k].slot)[place] = p;
            c.refs[p] = 1;
          }
        }
      }
    }
    if (PER == 1) {
      ends[tid] = inside + e[k].need;
      row_of[tid] = e[k].slot;
      have_of[tid] = c.pages_of(e[k].length);
    }
    if (ALONE) finish(c, e[k], done);
    else if (i < n) plan[i] = done ? 1 : 0;
    rank = min(rank + e[k].need, 0x7FFFFFFFu);
  }
  __syncthreads();
  const uint32_t there = taken_end > before ? taken_end - before : 0;
  if (PER > 1) {
    if (all <= kWanted) {
      for (uint32_t r = (uint32_t)tid; r < there; r += kOneBlock) {
        const int p = free.select(before + r);
        c.row(wanted[r].x)[wanted[r].y] = p;
        c.refs[p] = 1;
      }
    }
  } else {   // an equal share of the pages for each thread, whichever entries they are for
    const uint32_t share = (there + kOneBlock - 1) / kOneBlock, begin = (uint32_t)tid * share, end = min(begin + share, there);
    if (begin < end) {
      int t = 0;   // the entry of the first: the one whose pages end above it
#pragma unroll
      for (int d = kOneBlock / 2; d > 0; d >>= 1)
        if (ends[t + d - 1] <= begin) t += d;
      int p = free.select(before + begin);
      for (uint32_t r = begin;;) {
        c.row(row_of[t])[have_of[t] + (int)(r - (t > 0 ? ends[t - 1] : 0))] = p;
        c.refs[p] = 1;
        if (++r == end) break;
        while (ends[t] <= r) ++t;
        p = free.next(p);
      }
    }
  }
  __syncthreads();
  // nobody looks at the bits any more
  free.ranks(before, taken_end, [&](int w, uint64_t b, uint64_t mask) {
    if (ALONE) c.free_bits[w] = b & ~mask;
    else atomicOr((unsigned long long*)&c.taken[w], mask);
  });
}
__global__ void __launch_bounds__(256) advance_apply_kernel(Cache c, int n, const int32_t* slots, const int32_t* counts, int count, const int32_t* plan) {
  const int i = (int)blockIdx.x * 256 + (int)threadIdx.x;
  if (i < (c.pages + 63) / 64) {
    const uint64_t taken = c.taken[i];
    if (taken) {
      c.free_bits[i] &= ~taken;
      c.taken[i] = 0;
    }
  }
  if (i < n) finish(c, asked(c, n, slots, counts, count, i), plan[i] != 0);
}

__global__ void __launch_bounds__(kOneBlock) fork_plan_kernel(Cache c, int n, const int32_t* src, const int32_t* dst, ForkEntry* plan, uint8_t* status) {
  __shared__ uint64_t lds_bits[kBitsInLds];
  __shared__ uint32_t at[kOneBlock], shared[kOneBlock / 64];
  FreePages free;
  free.load(c);
  struct Look {
    int s, d, length;
    bool slots, nothing, need;
  };
  auto look = [&](int i) {   // (loads without a condition, as above)
    Look e;
    const int at = min(i, n - 1), s = src[at], d = dst[at];
    e.s = i < n ? s : -1;
    e.d = i < n ? d : -1;
    e.slots = (uint32_t)e.s < (uint32_t)c.slots && (uint32_t)e.d < (uint32_t)c.slots;
    e.nothing = e.s == e.d || e.s == -1 || e.d == -1;
    const int length = c.length(e.slots ? e.s : 0);
    e.length = e.slots ? length : 0;
    e.need = e.slots && !e.nothing && (e.length & ((1 << c.page_shift) - 1)) != 0;
    return e;
  };
  const int i = (int)blockIdx.x * kOneBlock + (int)threadIdx.x;
  const Look e = look(i);
  const int page = c.row(e.need ? e.s : 0)[e.need ? e.length >> c.page_shift : 0], had = c.pages_of(c.length(e.slots ? e.d : 0));
  const int last = e.need ? page : -1, old = e.slots ? had : 0;
  uint32_t before = 0, all;
  if (blockIdx.x > 0) {
    uint32_t sum = 0;
    for (int k0 = 0; k0 < (int)blockIdx.x; k0 += 4)   // four blocks' entries under way together (65536 entries: 78 us, one block at a time 85)
#pragma unroll
      for (int k = k0; k < k0 + 4; ++k) {
        const bool need = look(min(k, (int)blockIdx.x - 1) * kOneBlock + (int)threadIdx.x).need;
        sum += need && k < (int)blockIdx.x;
      }
    exclusive_sum(sum, shared, &before);
  }
  const uint32_t rank = before + exclusive_sum((uint32_t)e.need, shared, &all);
  free.ready(lds_bits, at, shared);
  uint8_t said = e.slots || e.nothing ? 0 : PGXCACHE_BAD_ENTRY;
  int tail = !e.slots || e.nothing ? kSkip : kNoTail;
  if (e.need) {
    if (rank < free.count) tail = free.select(rank);
    else { tail = kSkip; said = PGXCACHE_NO_PAGES; }
  }
  if (i < n) {
    plan[i] = ForkEntry{tail, e.s, e.d, e.length, last, old, {0, 0}};
    if (status) status[i] = said;
  }
  free.ranks(before, min(before + all, free.count), [&](int w, uint64_t, uint64_t mask) { atomicOr((unsigned long long*)&c.taken[w], mask); });
}

// `per` threads for each entry: a wavefront where pages have up to 16 KB, two up to 32 KB, four above.  A call of 4096 entries, by one, two and four wavefronts
// each: pages of 8 KB 15.9, 18.4 and 23.3 us, 16 KB 21.2, 21.6 and 24.4, 32 KB 31.7, 30.8 and 30.8, 64 KB 53.7, 52.5 and 50.0; of 256 entries, 32 KB
// 11.0, 9.7 and 9.8, 64 KB 14.0, 11.4 and 10.4.  A page that both slots name keeps
// the source's reference throughout, so none comes free in between.
__global__ void __launch_bounds__(256) fork_kernel(Cache c, int n, const ForkEntry* plan, int per) {
  __shared__ Freed freed;
  const int entries = 256 / per, blocks = (n + entries - 1) / entries;
  if ((int)blockIdx.x >= blocks) {   // the blocks behind the entries' take the plan's pages out of the bits
    const int w = ((int)blockIdx.x - blocks) * 256 + (int)threadIdx.x;
    if (w >= (c.pages + 63) / 64) return;
    const uint64_t taken = c.taken[w];
    if (taken) {
      atomicAnd((unsigned long long*)&c.free_bits[w], ~taken);
      c.taken[w] = 0;
    }
    return;
  }
  const int tid = (int)threadIdx.x & (per - 1), i = (int)blockIdx.x * entries + (int)threadIdx.x / per;
  ForkEntry e = plan[min(i, n - 1)];
  if (i >= n) e.tail = kSkip;
  freed.begin();
  const int tail = e.tail, length = e.length, old = e.old, last = tail >= 0 ? e.last : -1;
  const int full = length >> c.page_shift, filled = length & ((1 << c.page_shift) - 1), most = tail == kSkip ? 0 : max(old, full + (tail >= 0));
  if (tail != kSkip) {
    const int32_t* from = c.row(e.src);
    int32_t* to = c.row(e.dst);
    // the rows' entries and the page that is copied are asked for together
    auto entry = [&](int k, int* now, int* before) {
      *now = k < full ? from[k] : k == full ? tail : -1;
      *before = k < old ? to[k] : -1;
    };
    auto exchange = [&](int k, int now, int before) {
      if (now == before) return;   // a page that both had, as the nodes of one search tree have their root's
      if (k < full && c.is_page(now)) atomicAdd(&c.refs[now], 1);
      freed.release(c, before);
      to[k] = now;
    };
    int now0 = -1, before0 = -1;
    if (tid < most) entry(tid, &now0, &before0);
    constexpr int kAhead = 8;
    const uint32_t heads = (uint32_t)(c.layers * 2 * c.kv_heads), units = (uint32_t)(filled * c.head_dim * c.element_bytes() / 16), all = c.is_page(last) ? heads * units : 0;
    const uint32_t head = (uint32_t)(c.head_bytes() / 16);
    // the filled blocks' scales of every head
    const uint32_t blocks = (uint32_t)(filled + (1 << kBlockShift) - 1) >> kBlockShift, all_scales = c.scales && c.is_page(last) ? heads * blocks : 0;
    auto scale_at = [&](uint32_t u) { return u / blocks * (uint32_t)c.page_blocks() + u % blocks; };
    float scale0 = 0.0f;
    if ((uint32_t)tid < all_scales) scale0 = c.scales[last * c.page_scales() + scale_at((uint32_t)tid)];
    const u32x4* a = (const u32x4*)(c.kv + last * c.page_bytes());
    u32x4* b = (u32x4*)(c.kv + tail * c.page_bytes());
    for (uint32_t u = (uint32_t)tid; u < all; u += (uint32_t)per * kAhead) {   // the filled beginning of every head's keys and values
      u32x4 x[kAhead];
      uint32_t at[kAhead];
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {
        const uint32_t v = min(u + (uint32_t)(k * per), all - 1), h = v / units;
        at[k] = h * head + (v - h * units);
        x[k] = a[at[k]];
      }
#pragma unroll
      for (int k = 0; k < kAhead; ++k)
        if (u + (uint32_t)(k * per) < all) b[at[k]] = x[k];
    }
    for (uint32_t u = (uint32_t)tid; u < all_scales; u += (uint32_t)per)
      c.scales[tail * c.page_scales() + scale_at(u)] = u == (uint32_t)tid ? scale0 : c.scales[last * c.page_scales() + scale_at(u)];
    if (tid < most) exchange(tid, now0, before0);
    for (int k = tid + per; k < most; k += per) {
      int now, before;
      entry(k, &now, &before);
      exchange(k, now, before);
    }
    if (tid == 0) {
      c.lengths[e.dst] = length;
      c.grown[e.dst] = 0;
      if (tail >= 0) c.refs[tail] = 1;
    }
  }
  freed.end(c);
}

__global__ void __launch_bounds__(256) free_kernel(Cache c, int n, const int32_t* slots) {
  __shared__ Freed freed;
  const int i = (int)blockIdx.x * 4 + (int)(threadIdx.x >> 6), lane = (int)threadIdx.x & 63;
  const int slot = i >= n ? -1 : slots ? slots[i] : i;
  freed.begin();
  if ((uint32_t)slot < (uint32_t)c.slots) {
    int32_t* row = c.row(slot);
    for (int k = lane, old = c.pages_of(c.length(slot)); k < old; k += 64) freed.release(c, atomicExch(&row[k], -1));
    if (lane == 0) {
      c.lengths[slot] = 0;
      c.grown[slot] = 0;
    }
  }
  freed.end(c);
}

// a thread per page that moves: the r-th of those in use at and above `used` goes to the r-th free one
__global__ void __launch_bounds__(kOneBlock) compact_plan_kernel(Cache c, int2* moves, int32_t* moved_to, int32_t* counts, int32_t* used_out) {
  __shared__ uint64_t lds_bits[kBitsInLds];
  __shared__ uint32_t at[kOneBlock], shared[kOneBlock / 64];
  FreePages free;
  free.load(c);
  free.ready(lds_bits, at, shared);
  const int used = c.pages - (int)free.count, n = (int)free.below(used);   // as many free pages lie below `used` as pages in use above
  const int i = (int)blockIdx.x * kOneBlock + (int)threadIdx.x;
  if (i == 0) {
    counts[0] = used;
    counts[1] = n;
    if (used_out) *used_out = used;
  }
  for (int r = i; r < n; r += (int)gridDim.x * kOneBlock) {
    const int from = free.select_used((uint32_t)(used - n + r)), to = free.select((uint32_t)r);
    moves[r] = make_int2(from, to);
    moved_to[from] = to;
  }
}

__global__ void __launch_bounds__(256) compact_move_kernel(Cache c, const int2* moves, const int32_t* moved_to, const int32_t* counts) {
  const int used = counts[0], n = counts[1], lane = (int)threadIdx.x & 63;
  if (n == 0) return;
  for (int64_t w = (int64_t)blockIdx.x * 256 + threadIdx.x; w < (c.pages + 63) / 64; w += (int64_t)gridDim.x * 256) {
    const int64_t page = w * 64, inside = min((int64_t)64, c.pages - page);
    const uint64_t there = inside == 64 ? ~0ull : (1ull << inside) - 1;
    c.free_bits[w] = page + 64 <= used ? 0ull : page >= used ? there : there & ~0ull << (used - page);
  }
  for (int64_t slot = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); slot < c.slots; slot += (int64_t)gridDim.x * 4) {
    int32_t* row = c.row((int)slot);
    for (int k = lane, have = c.pages_of(c.length((int)slot)); k < have; k += 64) {
      const int p = row[k];
      if (p >= used && p < c.pages) row[k] = moved_to[p];
    }
  }
  const int64_t units = c.page_bytes() / 16;
  for (int m = (int)blockIdx.x; m < n; m += (int)gridDim.x) {
    const int2 move = moves[m];
    if (threadIdx.x == 0) {
      c.refs[move.y] = c.refs[move.x];
      c.refs[move.x] = 0;
    }
    const u32x4* a = (const u32x4*)(c.kv + move.x * c.page_bytes());
    u32x4* b = (u32x4*)(c.kv + move.y * c.page_bytes());
    for (int64_t u = threadIdx.x; u < units; u += 256) b[u] = a[u];
    if (c.scales)
      for (int64_t u = threadIdx.x; u < c.page_scales(); u += 256) c.scales[move.y * c.page_scales() + u] = c.scales[move.x * c.page_scales() + u];
  }
}


// A thread per 16 bytes of a head's key or value and four tokens.
constexpr int kTokensPerThread = 4;
__global__ void __launch_bounds__(256) write_kernel(Cache c, int layer, int n, const int32_t* slots, int tokens, Tokens k, Tokens v) {
  const uint32_t units = (uint32_t)c.head_dim / 8, per_entry = 2u * (uint32_t)c.kv_heads * units;
  const int64_t x = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const uint32_t runs = (uint32_t)(tokens + kTokensPerThread - 1) / kTokensPerThread;
  const int64_t token_run = x / per_entry;
  const uint32_t u = (uint32_t)(x - token_run * per_entry);
  if (token_run >= (int64_t)n * runs) return;
  const int i = (int)(token_run / runs), t0 = (int)(token_run - (int64_t)i * runs) * kTokensPerThread;
  const int slot = slots ? slots[i] : i;
  if ((uint32_t)slot >= (uint32_t)c.slots) return;
  const int grown = min(c.grown[slot], tokens), first = c.length(slot) - c.grown[slot];
  if (t0 >= grown || first < 0) return;
  const uint32_t which = u / units, at = u % units * 16;   // which: keys of all heads, then values
  const bool value = which >= (uint32_t)c.kv_heads;
  const uint32_t head = value ? which - (uint32_t)c.kv_heads : which;
  const Tokens& from = value ? v : k;
  const char* p = from.p + i * from.entry + head * from.head + at;
  char* to = c.kv + ((int64_t)layer * 2 * c.kv_heads + which) * c.head_bytes(2) + at;
  const int32_t* row = c.row(slot);
  u32x4 data[kTokensPerThread];
  int page[kTokensPerThread];
#pragma unroll
  for (int j = 0; j < kTokensPerThread; ++j) {
    const int t = min(t0 + j, grown - 1);
    data[j] = *(const u32x4_2*)(p + t * from.token);
    page[j] = row[(first + t) >> c.page_shift];
  }
#pragma unroll
  for (int j = 0; j < kTokensPerThread; ++j)
    if (t0 + j < grown && c.is_page(page[j]))
      *(u32x4*)(to + page[j] * c.page_bytes(2) + (int64_t)((first + t0 + j) & ((1 << c.page_shift) - 1)) * c.head_dim * 2) = data[j];
}

// ---- attention of one token per entry ------------------------------------------------------------------------------------------------
// Bound by the keys and values, which are read once: 2 head_dim elements per token and key head against 4 head_dim multiplications
// per query head.  The 16 columns of a matrix tile are the query heads that share a key head (those beyond the group are zero), its
// rows are tokens, 32 at a time:
//     S^T [32 tokens][16 heads] = K [32][D] * Q^T [D][16],    O^T [D][16] += V^T [D][32] * P^T [32][16]
// A wavefront keeps everything in registers.  Lane 16 g + c of v_mfma_f32_16x16x32 has row (column) c of its left (right) operand
// for the 8 contraction indices of group g, and column c, rows 4 g + r of the result.  So a lane that has scored tokens 4 g + r
// (and 16 + 4 g + r from the second half) holds its probabilities just where the second product wants them, if contraction
// index 8 g + j there means token 4 g + j for j < 4 and 16 + 4 g + j - 4 above.  V is read along its rows, the lane taking elements
// c D/16 ... of its 8 tokens; a byte permutation per two values turns them into left operands, the m-th of which has row c stand for
// element c D/16 + m.  The result then has elements (4 g + r) D/16 + m in the lane: D/4 neighbouring ones per lane.
template <int NT>
struct Tile {   // 32 tokens: keys [half][32-element part], values [token][dword]
  u32x4 k[2][NT];
  uint32_t v[8][NT];
};

// W wavefronts share a row (an entry and a key head); with four a row may also be split over blocks.  STREAM: keys and values are read with
// the hint that they are not read again soon.
template <class T, int NT, int W, bool STREAM>
__global__ void __launch_bounds__(64 * W, NT < 8 ? 2 : 1) attend_kernel(Cache c, AttendArgs a) {
  typedef typename T::x8 x8;
  constexpr int D = NT * 32, kOut = 8 * NT;   // elements of the output per lane
  const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), lane = (int)threadIdx.x & 63, col = lane & 15, g = lane >> 4;
  // head tiles and key heads are next to each other in the launch, then the parts of a sequence: what runs together reads neighbouring memory
  const uint32_t place = blockIdx.x, per_part = (uint32_t)(c.kv_heads * a.head_tiles);
  const uint32_t part = place / per_part, in_part = place - part * per_part;
  const int i = (int)(part / (uint32_t)a.splits), split = (int)(part - (uint32_t)i * (uint32_t)a.splits);
  const int kv_head = (int)(in_part / (uint32_t)a.head_tiles), head_tile = (int)(in_part - (uint32_t)(kv_head * a.head_tiles));
  const uint32_t unit = (uint32_t)i * per_part + in_part;
  const int slot = a.slots ? a.slots[i] : i;
  const bool is_slot = (uint32_t)slot < (uint32_t)c.slots;
  const int first_head = head_tile * kHeads, heads_here = min(kHeads, a.group - first_head), head0 = kv_head * a.group + first_head;

  // what depends on the entry only is asked for first, beside the slot's length
  u32x4 query[NT], fresh = {0, 0, 0, 0};
#pragma unroll
  for (int m = 0; m < NT; ++m) query[m] = *(const u32x4_2*)(a.q + i * a.q_entry + (head0 + min(col, heads_here - 1)) * a.q_head + g * 16 + m * 64);
  const bool writes = lane < 2 * D / 8;
  const int fresh_at = lane % (D / 8) * 16;
  if (a.k && wave == 0 && writes)
    fresh = *(const u32x4_2*)((lane < D / 8 ? a.k + i * a.k_entry + kv_head * a.k_head : a.v + i * a.v_entry + kv_head * a.v_head) + fresh_at);
  const int32_t* row = c.row(is_slot ? slot : 0);
  // page of half-tile lane & 1 of the wavefront's tile number (a multiple of 32) + lane / 2; the first ones are asked for before the length is known
  int ids = 0;
  if (a.splits == 1) ids = row[min((((wave + (lane >> 1) * W) * 2 + (lane & 1)) << 4) >> c.page_shift, c.width - 1)];
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
  const int chunk = ((tiles + a.splits - 1) / a.splits + W - 1) / W * W, active = (tiles + chunk - 1) / chunk;
  if (split >= active) return;
  const int begin = split * chunk, end = min(tiles, begin + chunk);

  const int64_t page_bytes = c.page_bytes(2), head_bytes = c.head_bytes(2);
  const char* keys = c.kv + ((int64_t)a.layer * 2 * c.kv_heads + kv_head) * head_bytes;
  const char* values = keys + c.kv_heads * head_bytes;
  const int in_page = (1 << c.page_shift) - 1;

  const bool alone = W > 1 && tiles <= 1;   // nothing to share: the first wavefront goes on by itself
  if (alone && wave > 0) return;

  // the new token's key and value go into the cache first, by the block that reads the last tile
  if (grown > 0 && end == tiles) {
    const int at = length - 1, page = row[at >> c.page_shift];
    if (wave == 0 && c.is_page(page) && writes)
      *(u32x4*)((char*)(lane < D / 8 ? keys : values) + page * page_bytes + (int64_t)(at & in_page) * D * 2 + fresh_at) = fresh;
    // (a wavefront's own memory operations are in order; other wavefronts wait)
    if (W > 1 && !alone) __syncthreads();
    else __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  }

  x8 q[NT];
#pragma unroll
  for (int m = 0; m < NT; ++m) q[m] = __builtin_bit_cast(x8, col < heads_here ? query[m] : u32x4{0, 0, 0, 0});

  float top = -INFINITY, sum = 0.0f;   // of the lane's head: the exponent that all four groups use, and this group's sum
  float peak = -INFINITY;              // kNarrow: the largest score when the exponent was last moved
  f32x4 acc[2 * NT];
#pragma unroll
  for (int m = 0; m < 2 * NT; ++m) acc[m] = f32x4{0, 0, 0, 0};

  if (!c.is_page(ids)) ids = 0;   // (behind the sequence: what is read there does not count)
  const int last_half = (length - 1) >> 4;
  auto load = [&](Tile<NT>& t, int number) {   // the wavefront's tile of that number
    const int tile = begin + wave + number * W;
    if ((number & 31) == 0 && (number > 0 || a.splits > 1)) {
      const int half = min((tile + (lane >> 1) * W) * 2 + (lane & 1), last_half);
      const int p = row[(half << 4) >> c.page_shift];
      ids = c.is_page(p) ? p : 0;
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int64_t page = (int64_t)__builtin_amdgcn_readlane(ids, (number & 31) * 2 + h) * page_bytes + (int64_t)((tile * 32 + h * 16) & in_page) * (D * 2);
      const char* k = keys + page + (col * D * 2 + g * 16);
#pragma unroll
      for (int m = 0; m < NT; ++m) t.k[h][m] = read_once<STREAM>((const u32x4*)(k + m * 64));
      const char* v = values + page + (g * 4 * D * 2 + col * NT * 4);
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int w = 0; w < NT; ++w) t.v[h * 4 + j][w] = read_once<STREAM>((const uint32_t*)(v + j * D * 2) + w);
    }
  };
  auto compute = [&](Tile<NT>& t, int number, auto last) {
    f32x4 s[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      s[h] = f32x4{0, 0, 0, 0};
#pragma unroll
      for (int m = 0; m < NT; ++m) s[h] = T::mfma(__builtin_bit_cast(x8, t.k[h][m]), q[m], s[h]);
      s[h] *= a.scale;
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
          for (int w = 0; w < NT; ++w) t.v[h * 4 + r][w] = there ? t.v[h * 4 + r][w] : 0;
        }
    }
    float most = fmaxf(fmaxf(fmaxf(s[0][0], s[0][1]), fmaxf(s[0][2], s[0][3])), fmaxf(fmaxf(s[1][0], s[1][1]), fmaxf(s[1][2], s[1][3])));
    const bool below = T::kNarrow && most < top + T::kLeast && most > -INFINITY && top > peak - (T::kDepth + T::kRoom);
    if (__any(most > top + T::kMost || below)) {
      float now;
      if (T::kNarrow) {
        const float here = across_groups_max(most);   // the tile's largest score
        peak = fmaxf(peak, here);
        const bool move = here > top + T::kMost || (here < top + T::kLeast && here > -INFINITY);
        now = move ? fmaxf(here, peak - T::kDepth) - T::kRoom : top;
      } else {
        now = across_groups_max(fmaxf(most, top));
      }
      const float factor = now > -INFINITY ? __builtin_amdgcn_exp2f(top - now) : 1.0f;
      top = now;
      sum *= factor;
#pragma unroll
      for (int m = 0; m < 2 * NT; ++m) acc[m] *= factor;
    }
    const float from = top > -INFINITY ? top : 0.0f;
    // with one number for p the output's error against 64 bits is 1.24 to 1.38 times that of its own rounding, and the time the same (4096 slots of 1 to 722 tokens 133.7 against 133.6 us, 1024 of 1 to 160 0.1 us less per layer)
    x8 high, low;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float p = __builtin_amdgcn_exp2f(s[j >> 2][j & 3] - from);
      sum += p;
      high[j] = (typename T::elem)p;
      low[j] = (typename T::elem)(p - (float)high[j]);
    }
#pragma unroll
    for (int m = 0; m < 2 * NT; ++m) {
      u32x4 x;
#pragma unroll
      for (int j = 0; j < 4; ++j) x[j] = __builtin_amdgcn_perm(t.v[2 * j + 1][m / 2], t.v[2 * j][m / 2], m & 1 ? 0x07060302u : 0x05040100u);
      acc[m] = T::mfma(__builtin_bit_cast(x8, x), high, acc[m]);
      acc[m] = T::mfma(__builtin_bit_cast(x8, x), low, acc[m]);
    }
  };
  const int mine = (end - begin - wave + W - 1) / W;   // this wavefront's tiles
  if (mine > 0) {   // the next tile is under way while one is computed (without a condition: the waits for memory are counted, not complete)
    constexpr std::false_type inner{};
    constexpr std::true_type outer{};
    Tile<NT> t0, t1;
    load(t0, 0);
    int number = 0;
    for (; number + 2 < mine; number += 2) {
      load(t1, number + 1);
      compute(t0, number, inner);
      load(t0, number + 2);
      compute(t1, number + 1, inner);
    }
    if (number + 1 < mine) {
      load(t1, number + 1);
      compute(t0, number, inner);
      compute(t1, number + 1, outer);
    } else {
      compute(t0, number, outer);
    }
  }
  finish_row<T, NT, W, (W >= 4), false>(a, Spot{wave, lane, col, g, i, head0, heads_here, split, active, unit, alone}, top, sum, acc);
}

template <class T, int NT, int W>
hipError_t launch_attend_by(const Cache& c, const AttendArgs& a, int64_t rows, hipStream_t stream) {
  // A pool beyond the 256 MB memory-side cache is streamed (4096 slots of 1 to 722 tokens, 757 MB: 132 us, without the hint 139; all of 722: 241 / 263; 3
  // sequences of 110000, 1.35 GB: 220 / 243), a smaller one stays in that cache from step to step (1024 slots of 1 to 722, 189 MB: 33 us, with the hint 39;
  // of 1 to 160 10.3 / 11.8).  The host knows the pool's size and not how much of it slots hold: the same 189 MB in a pool of 1 GB are
  // streamed, and take 42 us instead of 34.
  const bool streamed = (int64_t)c.pages * c.page_bytes() > (int64_t)256 << 20;
  const size_t join = (size_t)(W - 1) * kHeads * NT * 32 * 4, weights = a.splits > 1 ? (size_t)kMostSplits * kHeads * 4 + 64 * W * 16 : 0;
  if (!launchable(rows * a.splits, 64 * W)) return hipErrorInvalidConfiguration;
  const dim3 grid((unsigned)(rows * a.splits)), block(64 * W);
  if (streamed) hipLaunchKernelGGL((attend_kernel<T, NT, W, true>), grid, block, join > weights ? join : weights, stream, c, a);
  else hipLaunchKernelGGL((attend_kernel<T, NT, W, false>), grid, block, join > weights ? join : weights, stream, c, a);
  return hipGetLastError();
}
template <class T, int NT>
hipError_t launch_attend(const Cache& c, AttendArgs a, hipStream_t stream) {
  // The lengths are known on the device only, so the choice goes by how long a slot can be.
  //  * Short ones and many rows: a wavefront each (1 to 160 tokens, 2 key heads; with four in parentheses: 1024 slots, heads of 32 5.7 us (10.1), 64 10.3 (12.1), 128
  //    17.5 (22.8), 256 31.9 (59.5); 4096 slots, 64 30.8 (34.8), 128 73 (96), 256 170 (280)).  Longer ones: four (heads of 64; with one in parentheses: 1024
  //    of 1 to 722 tokens 33 us (36), 4096 132 (137), one of 722 7.0 (10.9)).
  //  * Few rows that can be longer than 32 tiles are split over blocks, 8 tiles to each if all tiles are there (one sequence, 2 key heads of 64, in one block in
  //    parentheses: 2048 tokens 8.5 us (13.7), 8192 9.0 (44.8)), as long as the machine's 256 compute units have two blocks each at most (3 x 8 rows of
  //    110000 tokens of 128 elements: 220 us with 504 blocks, 231 with 1008, 234 with 2016). Beyond 128 parts the joining costs more than the
  //    reading (one of 131072 tokens: 19.8 us in 128 parts, 25.0 in 256; 19.3 in 64).
  const int64_t rows = (int64_t)a.n * c.kv_heads * a.head_tiles, most_tiles = (((int64_t)c.width << c.page_shift) + 31) / 32;
  a.splits = 1;
  if (most_tiles <= 8 && rows >= 1024) return launch_attend_by<T, NT, 1>(c, a, rows, stream);
  if (most_tiles > 32) {
    const int64_t spread = kSplitBlocks / rows, useful = (most_tiles + 7) / 8;
    const int64_t splits = spread < useful ? spread : useful;
    a.splits = (int32_t)(splits < 1 ? 1 : splits > kMostSplits ? kMostSplits : splits);
  }
  return launch_attend_by<T, NT, 4>(c, a, rows, stream);
}
template <class T>
hipError_t launch_attend_for(const Cache& c, const AttendArgs& a, hipStream_t stream) {
  switch (c.head_dim) {
    case 32: return launch_attend<T, 1>(c, a, stream);
    case 64: return launch_attend<T, 2>(c, a, stream);
    case 96: return launch_attend<T, 3>(c, a, stream);
    case 128: return launch_attend<T, 4>(c, a, stream);
    default: return launch_attend<T, 8>(c, a, stream);
  }
}

// ---- host side -------------------------------------------------------------------------------------------------------------------------
bool opts_ok(const pgxcache_opts* o) {
  if (!o || o->slots < 1 || o->pages < 1 || o->width < 1 || o->layers < 1 || o->kv_heads < 1) return false;
  if (o->width > (1 << 20) || o->layers > 4096 || o->kv_heads > 4096 || o->pages > 0x7FFFFFC0) return false;
  if (o->page_size < 16 || o->page_size > 1024 || (o->page_size & (o->page_size - 1)) != 0) return false;
  if (o->head_dim != 32 && o->head_dim != 64 && o->head_dim != 96 && o->head_dim != 128 && o->head_dim != 256) return false;
  // tokens of a slot and bytes of a page are counted in 32 bits
  if ((int64_t)o->width * o->page_size > PGXCACHE_MAX_LENGTH || (int64_t)o->layers * o->kv_heads * o->page_size * o->head_dim * 4 > PGXCACHE_MAX_PAGE_BYTES) return false;
  return o->type == PGXCACHE_F16 || o->type == PGXCACHE_BF16;
}

struct Layout {
  size_t free_bits, taken, grown, plan, forks, moved_to, moves, counts, arrived, partial, total;
};
Layout layout(const pgxcache_opts& o) {
  Layout l;
  size_t at = 0;
  auto take = [&](size_t bytes) { const size_t here = at; at += (bytes + 255) / 256 * 256; return here; };
  l.free_bits = take(((size_t)o.pages + 63) / 64 * 8);
  l.taken = take(((size_t)o.pages + 63) / 64 * 8);
  l.grown = take((size_t)o.slots * 4);
  l.plan = take((size_t)o.slots * 4);
  l.forks = take((size_t)o.slots * sizeof(ForkEntry));
  l.moved_to = take((size_t)o.pages * 4);
  l.moves = take((size_t)o.pages * 8);
  l.counts = take(8);
  l.arrived = take(kSplitBlocks * 4);
  l.partial = take((size_t)kSplitBlocks * kHeads * ((size_t)o.head_dim + 2) * 4);
  l.total = at;
  return l;
}

Cache cache_of(pgxcache_t h) {
  Cache c;
  c.kv = (char*)h->kv; c.scales = h->scales; c.table = h->table; c.lengths = h->lengths; c.refs = h->refs; c.free_bits = h->free_bits; c.taken = h->taken; c.grown = h->grown;
  c.slots = h->o.slots; c.pages = h->o.pages; c.width = h->o.width; c.page_shift = __builtin_ctz((unsigned)h->o.page_size);
  c.layers = h->o.layers; c.kv_heads = h->o.kv_heads; c.head_dim = h->o.head_dim;
  return c;
}
bool list_ok(pgxcache_t h, int32_t n) { return h && n >= 0 && n <= h->o.slots; }
int scan(pgxcache_t h, int first) {
  const int64_t most = h->o.pages > h->o.slots ? h->o.pages : h->o.slots, threads = most > kSplitBlocks ? most : kSplitBlocks;
  hipLaunchKernelGGL(scan_refs_kernel, dim3((unsigned)((threads + 255) / 256)), dim3(256), 0, (hipStream_t)h->o.stream, cache_of(h), h->arrived, first);
  HIPCHK(hipGetLastError());
  return PGXCACHE_OK;
}

}  // namespace

extern "C" {

size_t pgxcache_work_bytes(const pgxcache_opts* opts) { return opts_ok(opts) ? layout(*opts).total : 0; }

int pgxcache_rescan(pgxcache_t h) { return h ? scan(h, 0) : PGXCACHE_EINVAL; }

static int init(pgxcache_t* out, const pgxcache_opts* opts, void* kv_dev, float* scales_dev, int32_t* table_dev, int32_t* lengths_dev, int32_t* refs_dev,
                void* work_dev, size_t work_bytes) {
  if (!out || !opts_ok(opts) || !kv_dev || !table_dev || !lengths_dev || !refs_dev || !work_dev) return PGXCACHE_EINVAL;
  if (((uintptr_t)kv_dev & 15u) != 0 || ((uintptr_t)work_dev & 255u) != 0) return PGXCACHE_EINVAL;
  if ((((uintptr_t)table_dev | (uintptr_t)lengths_dev | (uintptr_t)refs_dev) & 3u) != 0) return PGXCACHE_EINVAL;
  const Layout l = layout(*opts);
  if (work_bytes < l.total) return PGXCACHE_EINVAL;
  pgxcache_t h = new (std::nothrow) pgxcache_ctx;
  if (!h) return PGXCACHE_ENOMEM;
  char* w = (char*)work_dev;
  h->o = *opts;
  h->kv = kv_dev; h->scales = scales_dev; h->table = table_dev; h->lengths = lengths_dev; h->refs = refs_dev;
  h->free_bits = (uint64_t*)(w + l.free_bits); h->taken = (uint64_t*)(w + l.taken); h->grown = (int32_t*)(w + l.grown); h->plan = (int32_t*)(w + l.plan); h->forks = (ForkEntry*)(w + l.forks);
  h->moved_to = (int32_t*)(w + l.moved_to); h->moves = (int2*)(w + l.moves); h->counts = (int32_t*)(w + l.counts);
  h->arrived = (uint32_t*)(w + l.arrived); h->partial = (float*)(w + l.partial);
  const int rc = scan(h, 1);
  if (rc != PGXCACHE_OK) { delete h; return rc; }
  *out = h;
  return PGXCACHE_OK;
}

int pgxcache_init(pgxcache_t* out, const pgxcache_opts* opts, void* kv_dev, int32_t* table_dev, int32_t* lengths_dev, int32_t* refs_dev,
                  void* work_dev, size_t work_bytes) {
  return init(out, opts, kv_dev, nullptr, table_dev, lengths_dev, refs_dev, work_dev, work_bytes);
}
int pgxcache_init_e4m3(pgxcache_t* out, const pgxcache_opts* opts, void* kv_dev, float* scales_dev, int32_t* table_dev, int32_t* lengths_dev, int32_t* refs_dev,
                       void* work_dev, size_t work_bytes) {
  if (!scales_dev || ((uintptr_t)scales_dev & 3u) != 0) return PGXCACHE_EINVAL;
  return init(out, opts, kv_dev, scales_dev, table_dev, lengths_dev, refs_dev, work_dev, work_bytes);
}

int pgxcache_destroy(pgxcache_t h) {
  if (!h) return PGXCACHE_EINVAL;
  delete h;
  return PGXCACHE_OK;
}

int pgxcache_advance(pgxcache_t h, int32_t n, const int32_t* slots_dev, const int32_t* counts_dev, int32_t count, uint8_t* status_dev) {
  if (!list_ok(h, n) || (!counts_dev && count < 0)) return PGXCACHE_EINVAL;
  if (n == 0) return PGXCACHE_OK;
  const hipStream_t stream = (hipStream_t)h->o.stream;
  const Cache c = cache_of(h);
  if (n <= kOneBlock || (n <= 4 * kOneBlock && !counts_dev && count <= h->o.page_size)) {   // one launch (counts: prompts, of any number of pages)
    if (n <= kOneBlock) hipLaunchKernelGGL((advance_kernel<1, true>), dim3(1), dim3(kOneBlock), 0, stream, c, n, slots_dev, counts_dev, count, h->plan, status_dev);
    else hipLaunchKernelGGL((advance_kernel<4, true>), dim3(1), dim3(kOneBlock), 0, stream, c, n, slots_dev, counts_dev, count, h->plan, status_dev);
    HIPCHK(hipGetLastError());
    return PGXCACHE_OK;
  }
  hipLaunchKernelGGL((advance_kernel<1, false>), dim3(((unsigned)n + kOneBlock - 1) / kOneBlock), dim3(kOneBlock), 0, stream, c, n, slots_dev, counts_dev, count, h->plan, status_dev);
  HIPCHK(hipGetLastError());
  const int words = (c.pages + 63) / 64, threads = n > words ? n : words;
  hipLaunchKernelGGL(advance_apply_kernel, dim3(((unsigned)threads + 255) / 256), dim3(256), 0, stream, c, n, slots_dev, counts_dev, count, h->plan);
  HIPCHK(hipGetLastError());
  return PGXCACHE_OK;
}

int pgxcache_write(pgxcache_t h, int32_t layer, int32_t n, const int32_t* slots_dev, int32_t tokens, const void* k_dev, int64_t k_entry_stride,
                   int64_t k_token_stride, int64_t k_head_stride, const void* v_dev, int64_t v_entry_stride, int64_t v_token_stride, int64_t v_head_stride) {
  if (!list_ok(h, n) || layer < 0 || layer >= h->o.layers || tokens < 0) return PGXCACHE_EINVAL;
  if (n == 0 || tokens == 0) return PGXCACHE_OK;
  if (!k_dev || !v_dev || (((uintptr_t)k_dev | (uintptr_t)v_dev) & 1u) != 0) return PGXCACHE_EINVAL;
  const int64_t runs = ((int64_t)tokens + kTokensPerThread - 1) / kTokensPerThread;
  const Cache c = cache_of(h);
  const int64_t blocks = c.scales ? write8_blocks(c, n, tokens) : ((int64_t)n * runs * 2 * h->o.kv_heads * (h->o.head_dim / 8) + 255) / 256;
  if (!launchable(blocks, 256)) return PGXCACHE_EINVAL;
  const Tokens k = {(const char*)k_dev, k_entry_stride * 2, k_token_stride * 2, k_head_stride * 2}, v = {(const char*)v_dev, v_entry_stride * 2, v_token_stride * 2, v_head_stride * 2};
  if (c.scales) {
    HIPCHK(write8(c, h->o.type == PGXCACHE_F16, layer, n, slots_dev, tokens, 0, k, v, (hipStream_t)h->o.stream));
    return PGXCACHE_OK;
  }
  hipLaunchKernelGGL(write_kernel, dim3((unsigned)blocks), dim3(256), 0, (hipStream_t)h->o.stream, c, layer, n, slots_dev, tokens, k, v);
  HIPCHK(hipGetLastError());
  return PGXCACHE_OK;
}

int pgxcache_attend(pgxcache_t h, int32_t layer, int32_t n, const int32_t* slots_dev, int32_t heads, const void* q_dev, int64_t q_entry_stride,
                    int64_t q_head_stride, const void* k_dev, int64_t k_entry_stride, int64_t k_head_stride, const void* v_dev, int64_t v_entry_stride,
                    int64_t v_head_stride, float scale, void* out_dev, int64_t out_entry_stride, int64_t out_head_stride, float* lse_dev) {
  if (!list_ok(h, n) || layer < 0 || layer >= h->o.layers || heads < 1 || heads > 65536 || heads % h->o.kv_heads != 0) return PGXCACHE_EINVAL;
  if ((n > 1 && llabs(out_entry_stride) < h->o.head_dim) || (heads > 1 && llabs(out_head_stride) < h->o.head_dim)) return PGXCACHE_EINVAL;   // rows written twice
  if (!(scale - scale == 0.0f) || (k_dev != nullptr) != (v_dev != nullptr)) return PGXCACHE_EINVAL;
  if (n == 0) return PGXCACHE_OK;
  if (!q_dev || !out_dev || (((uintptr_t)q_dev | (uintptr_t)k_dev | (uintptr_t)v_dev | (uintptr_t)out_dev) & 1u) != 0) return PGXCACHE_EINVAL;
  AttendArgs a;
  a.q = (const char*)q_dev; a.k = (const char*)k_dev; a.v = (const char*)v_dev; a.out = (char*)out_dev; a.lse = lse_dev;
  a.q_entry = q_entry_stride * 2; a.q_head = q_head_stride * 2; a.k_entry = k_entry_stride * 2; a.k_head = k_head_stride * 2;
  a.v_entry = v_entry_stride * 2; a.v_head = v_head_stride * 2; a.out_entry = out_entry_stride * 2; a.out_head = out_head_stride * 2;
  a.slots = slots_dev; a.partial = h->partial; a.arrived = h->arrived;
  a.n = n; a.layer = layer; a.heads = heads; a.group = heads / h->o.kv_heads; a.head_tiles = (a.group + kHeads - 1) / kHeads;
  a.scale = scale * 1.44269504088896340736f;
  if ((int64_t)n * h->o.kv_heads * a.head_tiles > 0x7FFFFFFF) return PGXCACHE_EINVAL;
  const Cache c = cache_of(h);
  if (c.scales) {
    if (!attend8_fits(c, a)) return PGXCACHE_EINVAL;
    if (a.k && a.head_tiles > 1) {   // several blocks read the new token's block: it is written before, since rounding a block again is not the same twice
      const Tokens k = {a.k, a.k_entry, 0, a.k_head}, v = {a.v, a.v_entry, 0, a.v_head};
      HIPCHK(write8(c, h->o.type == PGXCACHE_F16, layer, n, slots_dev, 1, 1, k, v, (hipStream_t)h->o.stream));
      a.k = a.v = nullptr;
    }
    HIPCHK(attend8(c, h->o.type == PGXCACHE_F16, a, (hipStream_t)h->o.stream));
    return PGXCACHE_OK;
  }
  const hipError_t e = h->o.type == PGXCACHE_F16 ? launch_attend_for<F16>(c, a, (hipStream_t)h->o.stream) : launch_attend_for<BF16>(c, a, (hipStream_t)h->o.stream);
  if (e == hipErrorInvalidConfiguration) return PGXCACHE_EINVAL;
  HIPCHK(e);
  return PGXCACHE_OK;
}

int pgxcache_read(pgxcache_t h, int32_t layer, int32_t n, const int32_t* slots_dev, const int32_t* first_dev, int32_t first, int32_t tokens, void* k_dev,
                  int64_t k_entry_stride, int64_t k_token_stride, int64_t k_head_stride, void* v_dev, int64_t v_entry_stride, int64_t v_token_stride, int64_t v_head_stride) {
  if (!list_ok(h, n) || layer < 0 || layer >= h->o.layers || tokens < 0 || (!first_dev && first < 0)) return PGXCACHE_EINVAL;
  if (n == 0 || tokens == 0) return PGXCACHE_OK;
  if (!k_dev || !v_dev || (((uintptr_t)k_dev | (uintptr_t)v_dev) & 1u) != 0) return PGXCACHE_EINVAL;
  const int64_t sizes[3] = {n, tokens, h->o.kv_heads}, ks[3] = {k_entry_stride, k_token_stride, k_head_stride}, vs[3] = {v_entry_stride, v_token_stride, v_head_stride};
  if (!rows_apart(sizes, ks, h->o.head_dim) || !rows_apart(sizes, vs, h->o.head_dim)) return PGXCACHE_EINVAL;
  if (rows_meet(Rows{k_dev, {sizes[0], sizes[1], sizes[2]}, {ks[0], ks[1], ks[2]}}, Rows{v_dev, {sizes[0], sizes[1], sizes[2]}, {vs[0], vs[1], vs[2]}}, h->o.head_dim, 2)) return PGXCACHE_EINVAL;
  const Cache c = cache_of(h);
  if (!launchable(read_blocks(c, n, tokens), 256)) return PGXCACHE_EINVAL;
  const Tokens k = {(const char*)k_dev, k_entry_stride * 2, k_token_stride * 2, k_head_stride * 2}, v = {(const char*)v_dev, v_entry_stride * 2, v_token_stride * 2, v_head_stride * 2};
  HIPCHK(read_back(c, h->o.type == PGXCACHE_F16, layer, n, slots_dev, first_dev, first, tokens, k, v, (hipStream_t)h->o.stream));
  return PGXCACHE_OK;
}

int pgxcache_fork(pgxcache_t h, int32_t n, const int32_t* src_slots_dev, const int32_t* dst_slots_dev, uint8_t* status_dev) {
  if (!list_ok(h, n)) return PGXCACHE_EINVAL;
  if (n == 0) return PGXCACHE_OK;
  if (!src_slots_dev || !dst_slots_dev) return PGXCACHE_EINVAL;
  const size_t page = (size_t)cache_of(h).page_bytes();
  const int per = page <= 16384 ? 64 : page <= 32768 ? 128 : 256, entries = 256 / per, words = (h->o.pages + 63) / 64;
  const int64_t blocks = ((int64_t)n + entries - 1) / entries + (words + 255) / 256;
  if (!launchable(blocks, 256)) return PGXCACHE_EINVAL;
  hipLaunchKernelGGL(fork_plan_kernel, dim3(((unsigned)n + kOneBlock - 1) / kOneBlock), dim3(kOneBlock), 0, (hipStream_t)h->o.stream, cache_of(h), n, src_slots_dev, dst_slots_dev, h->forks, status_dev);
  HIPCHK(hipGetLastError());
  hipLaunchKernelGGL(fork_kernel, dim3((unsigned)blocks), dim3(256), 0, (hipStream_t)h->o.stream, cache_of(h), n, h->forks, per);
  HIPCHK(hipGetLastError());
  return PGXCACHE_OK;
}

int pgxcache_free(pgxcache_t h, int32_t n, const int32_t* slots_dev) {
  if (!list_ok(h, n)) return PGXCACHE_EINVAL;
  if (n == 0) return PGXCACHE_OK;
  const int64_t blocks = ((int64_t)n + 3) / 4;
  if (!launchable(blocks, 256)) return PGXCACHE_EINVAL;
  hipLaunchKernelGGL(free_kernel, dim3((unsigned)blocks), dim3(256), 0, (hipStream_t)h->o.stream, cache_of(h), n, slots_dev);
  HIPCHK(hipGetLastError());
  return PGXCACHE_OK;
}

int pgxcache_compact(pgxcache_t h, int32_t* used_dev) {
  if (!h) return PGXCACHE_EINVAL;
  hipLaunchKernelGGL(compact_plan_kernel, dim3(16), dim3(kOneBlock), 0, (hipStream_t)h->o.stream, cache_of(h), h->moves, h->moved_to, h->counts, used_dev);
  HIPCHK(hipGetLastError());
  hipLaunchKernelGGL(compact_move_kernel, dim3(2048), dim3(256), 0, (hipStream_t)h->o.stream, cache_of(h), h->moves, h->moved_to, h->counts);
  HIPCHK(hipGetLastError());
  return PGXCACHE_OK;
}

const char* pgxcache_strerror(int code) {
  switch (code) {
    case PGXCACHE_OK: return "ok";
    case PGXCACHE_EINVAL: return "invalid argument";
    case PGXCACHE_EHIP: return "HIP runtime error";
    case PGXCACHE_ENOMEM: return "out of host memory";
    default: return "unknown error";
  }
}

int pgxcache_last_hip_error(void) { return g_last_hip; }

}  // extern "C"
