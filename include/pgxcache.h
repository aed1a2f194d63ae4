/*
 * pgxcache.h -- C ABI of a paged cache of keys and values for policies that read a game as its sequence of moves (gfx950).
 *
 * A tree search keeps a pool of game states and steps from copies of them (pgxgo_step_slots / pgxgo_copy_slots in pgxgo.h).
 * A policy whose input is the sequence of moves has, for each such state, the keys and values of the moves so far.  This
 * cache holds them for a pool of slots that follow the states: a slot's tokens lie in pages, slots that share a beginning
 * share its full pages, so that copying a state copies one page at most.
 *
 * Memory (all device memory, the caller's; the cache can be looked at, saved and filled through it):
 *   kv_dev      [pages][layers][2][kv_heads][page_size][head_dim] of `type`; index 0 of the third dimension: keys, 1: values
 *   table_dev   [slots][width] int32: the slot's pages in the order of its tokens, -1 behind them
 *   lengths_dev [slots] int32: tokens of the slot
 *   refs_dev    [pages] int32: how many table entries name the page; 0: free
 *   work_dev    pgxcache_work_bytes(): what the calls need between themselves; nothing of it has to be saved
 *   scales_dev  8 bits only: [pages][layers][2][kv_heads][page_size / 16] float32
 * Only full pages are shared: a partly filled last page belongs to one slot.
 * The calls read table, lengths and refs as they find them; a page number outside the pool is never followed.
 *
 * Conventions are those of pgxgo.h: asynchronous on the stream given at the beginning, no allocation, no synchronisation,
 * negative codes, nothing throws or aborts.  One handle's calls share work_dev and belong on one stream.  A call that would need 2^32 threads (attend: 2^24 entries times key
 * heads where slots can be long, read and write: a thread for 8 elements of 4 tokens or fewer, fork: 2^24 entries, free: 2^26) is refused and does nothing: it can be made in parts.
 *
 * Held in 8 bits (pgxcache_init_e4m3): kv_dev has elements of 8 bits in the same order, e4m3 codes (4 bits of exponent, 3 of fraction, up to
 * 448, no infinities).  An element is its code times the scale of its block: 16 tokens of a slot, from a multiple of 16 on, in one layer and head, keys or values.
 * `type` is that of the queries, keys, values and outputs of the calls.  Writing tokens into a block:
 *     m = the largest finite magnitude among the block's elements that the call writes
 *     s = the smallest power of two with m <= 448 s, at least 2^-100
 *     if tokens of the block were there before those that the call writes:  s = max(s, the block's scale), and where that makes the scale larger,
 *         their codes become  to nearest, ties to even (code * old scale / s)
 *     code = to nearest, ties to even (x / s);  NaN where x is not finite
 * so a value is held to 2^-4 of itself, or where it is smaller than 2^-6 s to 2^-10 s, 2^-9 s if later tokens have raised the scale (each time it is rounded to half a step of the
 * new scale, 2^-10 of that, and the scales before it add up to less than the last).  A slot's tokens are written in their order: what a block holds behind the
 * tokens that a call writes is given up.  Scales in memory that the caller fills are finite, above 0 and at most 2^126; if one is no power of two, it is x times a reciprocal, off by 2^-22 of
 * itself, that is rounded, and earlier codes times a quotient in 32 bits.
 * A finite value near the type's end (float16: above 63488, bfloat16: above 2^127.95) may be held as a number beyond it; it is read back as the type's largest number.
 *
 * Lists of slots: slots_dev[n] int32, n <= slots, pairwise distinct; NULL: slots 0 .. n-1.  An entry of -1 is left out (as action
 * -1 in the environments), an entry outside [-1, slots) touches nothing.  status_dev (nullable, uint8 [n]): 0 done (or left out),
 * PGXCACHE_NO_PAGES, PGXCACHE_FULL, PGXCACHE_BAD_ENTRY: nothing was done for the entry.
 */
#ifndef PGXCACHE_H_
#define PGXCACHE_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define PGXCACHE_OK 0
#define PGXCACHE_EINVAL (-1) /* null pointer, size out of range, misaligned or too small buffer, unsupported type or head size */
#define PGXCACHE_EHIP (-2)   /* a HIP runtime call failed; see pgxcache_last_hip_error() */
#define PGXCACHE_ENOMEM (-3) /* host allocation of the handle failed */

#define PGXCACHE_F16 1
#define PGXCACHE_BF16 2

#define PGXCACHE_MAX_LENGTH (1 << 30)     /* tokens that a slot's pages can hold */
#define PGXCACHE_MAX_PAGE_BYTES (1 << 30)

#define PGXCACHE_NO_PAGES 1    /* status: too few free pages */
#define PGXCACHE_FULL 2        /* status: more tokens than width pages hold */
#define PGXCACHE_BAD_ENTRY 255 /* status: no such slot, or a negative number of tokens */

typedef struct pgxcache_ctx* pgxcache_t;

typedef struct {
  int32_t slots, pages;
  int32_t width;     /* pages a slot can have */
  int32_t page_size; /* tokens of a page: a power of two from 16 to 1024 */
  int32_t layers, kv_heads;
  int32_t head_dim;  /* 32, 64, 96, 128 or 256 */
  int32_t type;      /* PGXCACHE_F16 or PGXCACHE_BF16 */
  void* stream;      /* hipStream_t of the caller; NULL = default stream */
} pgxcache_opts;

/* Bytes of work memory for these sizes (256-byte aligned); 0 if they are out of range. */
size_t pgxcache_work_bytes(const pgxcache_opts* opts);

/* Takes the memory as it is: an empty cache has table -1, lengths 0 and refs 0; a saved one goes on where it was (save it when the tokens
 * that there is room for have been written: what an advance before the call made room for is not remembered).  kv_dev 16-byte
 * aligned.  Enqueues one kernel that looks through refs_dev; to be called again (pgxcache_rescan) after the caller has written to
 * refs_dev, which leaves all else as it is. */
int pgxcache_init(pgxcache_t* out, const pgxcache_opts* opts, void* kv_dev, int32_t* table_dev, int32_t* lengths_dev, int32_t* refs_dev,
                  void* work_dev, size_t work_bytes);
/* The same for keys and values held in 8 bits; scales_dev 4-byte aligned. */
int pgxcache_init_e4m3(pgxcache_t* out, const pgxcache_opts* opts, void* kv_dev, float* scales_dev, int32_t* table_dev, int32_t* lengths_dev, int32_t* refs_dev,
                       void* work_dev, size_t work_bytes);
int pgxcache_destroy(pgxcache_t h); /* frees the host handle only */
int pgxcache_rescan(pgxcache_t h);

/* Room for counts_dev[i] more tokens (NULL: `count` for every entry) at the end of each slot.  Pages are given out in ascending
 * order, the lowest free ones first, to the entries in their order; an entry gets all it needs or nothing, and what it needs
 * counts before later entries either way.  The new tokens are there for pgxcache_write / pgxcache_attend, which take them
 * to be the last ones of the slot, until the slot's next pgxcache_advance, pgxcache_fork (as destination) or pgxcache_free. */
int pgxcache_advance(pgxcache_t h, int32_t n, const int32_t* slots_dev, const int32_t* counts_dev, int32_t count, uint8_t* status_dev);

/* Keys and values of the tokens that the last pgxcache_advance of each slot made room for (the first `tokens` of them), in one layer:
 * element [i][t][head][.] at i * entry_stride + t * token_stride + head * head_stride, elements of the cache's type. */
int pgxcache_write(pgxcache_t h, int32_t layer, int32_t n, const int32_t* slots_dev, int32_t tokens, const void* k_dev, int64_t k_entry_stride,
                   int64_t k_token_stride, int64_t k_head_stride, const void* v_dev, int64_t v_entry_stride, int64_t v_token_stride, int64_t v_head_stride);

/* Keys and values as they are held (a copy, or code * scale rounded to `type`, and no further than its largest number): the tokens first_dev[i] (NULL: `first`), ... + tokens - 1 of each slot, in one layer, to
 * element [i][t][head][.] at i * entry_stride + t * token_stride + head * head_stride; neither rows nor the two outputs may overlap (rows of the one between those of the other are apart): such calls are refused.  Zeros where a slot has no such token, and
 * for an entry that is no slot.  Entries may repeat. */
int pgxcache_read(pgxcache_t h, int32_t layer, int32_t n, const int32_t* slots_dev, const int32_t* first_dev, int32_t first, int32_t tokens, void* k_dev,
                  int64_t k_entry_stride, int64_t k_token_stride, int64_t k_head_stride, void* v_dev, int64_t v_entry_stride, int64_t v_token_stride, int64_t v_head_stride);

/* Attention of one token per entry over all tokens of its slot, in one layer:
 *     out[i][h] = sum_t softmax_t(scale * q[i][h] . K[t][h / group]) V[t][h / group],     group = heads / kv_heads
 * q_dev, out_dev: elements of the cache's type, [i][h][.] at i * entry_stride + h * head_stride (those of the output may not
 * overlap: strides below head_dim are refused); heads a multiple of kv_heads.  lse_dev
 * (nullable): float32 [n][heads], log sum_t exp(scale * q . K[t]).  k_dev and v_dev (both or neither): the key and value of each slot's
 * last token, [i][head][.], written to the cache by this call where the slot's last pgxcache_advance made room for it (and otherwise
 * ignored), so that a step takes one launch per layer (in 8 bits with more than 16 heads to a key head two); without them entries may repeat.  A slot without tokens, and an entry that is no slot, gives zeros and -infinity.
 * Scores, sums and the output before its rounding are held in 32 bits; probabilities are multiplied as two numbers of the
 * cache's type that add up to them within 2^-17 (float16: of the sum of 32 tokens' probabilities), however small they are.
 * With elements of 8 bits the probabilities, times the values' scales, are two bfloat16 numbers whatever `type` is, and a float16 output between its largest number and
 * 2^16 (1 + 2^-10) is that number: averages of held values may lie there.  Other outputs beyond the type's end are infinite.  Either way of holding sums up to 2^8 times a value for
 * each token, in 32 bits: where bfloat16 values reach 2^119 over the number of tokens, the output may be infinite.
 * A key or value that is infinite or NaN makes what it counts for NaN; places behind a slot's last token may hold anything. */
int pgxcache_attend(pgxcache_t h, int32_t layer, int32_t n, const int32_t* slots_dev, int32_t heads, const void* q_dev, int64_t q_entry_stride,
                    int64_t q_head_stride, const void* k_dev, int64_t k_entry_stride, int64_t k_head_stride, const void* v_dev, int64_t v_entry_stride,
                    int64_t v_head_stride, float scale, void* out_dev, int64_t out_entry_stride, int64_t out_head_stride, float* lse_dev);

/* slot[dst_slots_dev[i]] = slot[src_slots_dev[i]], as pgxgo_copy_slots does for states and with its constraints: destinations are pairwise
 * distinct and none is the source of another entry.  Full pages are shared, a partly filled last one is copied to the lowest
 * free page.  What the destination held is given up; pages that come free by it can be taken by later calls, not by this one.  Tokens of
 * the source that have not been written yet are to be written before it is forked.  An entry with src == dst does nothing.  On PGXCACHE_NO_PAGES the destination keeps what it had. */
int pgxcache_fork(pgxcache_t h, int32_t n, const int32_t* src_slots_dev, const int32_t* dst_slots_dev, uint8_t* status_dev);

/* The slots' tokens are given up; pages that no other slot shares come free. */
int pgxcache_free(pgxcache_t h, int32_t n, const int32_t* slots_dev);

/* Moves pages so that those in use are 0 .. used-1: the ones at and above `used` go, in ascending order, to the free ones below it.
 * used_dev (nullable): int32, the number of pages in use.  Slots keep their contents. */
int pgxcache_compact(pgxcache_t h, int32_t* used_dev);

const char* pgxcache_strerror(int code);
int pgxcache_last_hip_error(void); /* hipError_t of the most recent PGXCACHE_EHIP on this thread, else 0 */

#ifdef __cplusplus
}
#endif
#endif /* PGXCACHE_H_ */
