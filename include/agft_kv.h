/*
 * agft_kv.h -- C ABI of a serving node's paged key/value cache on AMD Instinct
 * MI355X (gfx950): block tables and slot maps, a cache held in 8 bits, and the
 * attention that reads it.
 *
 * The tuner of agft.h chooses the clock of a node that serves requests from
 * such a cache; the environment of agft_sim.h describes that node's window in
 * closed form.  The calls here are the window's own work, so that a study can
 * run and measure it.
 *
 * A window goes
 *
 *   agft_kv_plan     the requests' new tokens get pages and slots
 *   per layer:
 *   agft_kv_append   the layer's new keys and values go to their slots
 *   agft_kv_attend   the new tokens attend to everything their requests hold
 *   agft_kv_commit   the plan's lengths become the tables' lengths
 *
 * and agft_kv_export reads slots back as dense tensors.  One set of tables
 * serves every layer; each layer has a cache of its own.
 *
 * Lengths.  Request i holds L_i tokens (0 at the start).  A window asks for
 * add_i more: > 0 new tokens, 0 none, < 0 the request ends.  With
 * pages(n) = ceil(n / page), a_i = add_i where 0 < add_i and L_i + add_i <=
 * row_pages * page and else 0, need_i = pages(L_i + a_i) - pages(L_i):
 *
 *   granted_i = a_i  if (need_i = 0 or sum_{j<=i} need_j <= free pages)
 *                    and sum_{j<=i} a_j <= max_tokens,  else 0.
 *
 * Tokens keep their place whether granted or not: request i's rows of the
 * window's tensors start at starts_i = min(max_tokens, sum_{j<i} a_j).  A token
 * that is not granted has slot -1; it is not stored and its attention is 0.
 * Pages come from the head of a ring of free pages and go back to its tail, in
 * the requests' order, so equal histories give equal tables.  Pages of a
 * request that ends are free from the next window on.
 *
 * Codes.  A page holds, per head and side (keys, values), page x dim codes of 8
 * bits and one exponent e: a code c stands for value(c) * 2^e, value(c) being
 * the e4m3 number (range +-448, no infinity) or the integer in -127..127.  The
 * first write to a page (the one that starts at its first token) takes the
 * smallest e >= -64 whose range holds its numbers; later writes raise it where
 * they need more and re-round the older codes, to nearest even each time.
 * Exponents are whole so that this costs e4m3 codes nothing (bar what falls
 * below its smallest numbers) and keeps integer codes within one step of the
 * number stored.  Infinities are held as the range's end, NaN as 0.
 *
 * Layout, by blocks of 16 tokens and 64 numbers, as the matrix instructions
 * take them: codes [pages][heads][2][page/16][dim/64][64][16] bytes.  In a
 * block, byte b of entry 16 g + m is, of the keys, token m's number 16 g + b;
 * of the values, token 4 g + b % 4's number 16 (b / 4) + m.  Exponents: int32
 * [pages][heads][2].
 *
 * Memory, streams and errors follow agft.h: caller-owned device buffers,
 * 256-byte aligned, no allocation, work only enqueued on the given stream,
 * negative status codes (the AGFT_E_* values) on invalid arguments, before
 * anything is enqueued.  No call keeps state on the host, so any of them can be
 * recorded into a graph.  Buffers of one call must not overlap.  What a call
 * cannot check on the host is its caller's: block tables, lengths and rings as
 * agft_kv_plan and agft_kv_commit leave them (a page that no pool has is read as
 * the pool's last), steps that agft_kv_plan has written, and steps and tables
 * under the configuration that they were written with (layers may differ in dim and form; with other requests, row_pages,
 * pages, page, heads or group their parts are looked for in the wrong places, out
 * of the buffers too), and work within 2^31 units (64 tokens of a request, for each
 * head and 16 rows of queries; 288 GB of cache make 2^26 of single tokens).
 */
#ifndef AGFT_KV_H
#define AGFT_KV_H

#include <stddef.h>
#include <stdint.h>

#include "agft.h"

#ifdef __cplusplus
extern "C" {
#endif

/* agft_kv_config.form: how the cache holds numbers */
#define AGFT_KV_E4M3 0
#define AGFT_KV_INT8 1

/* types of dense tensors */
#define AGFT_KV_BF16 0
#define AGFT_KV_FP16 1
#define AGFT_KV_FP32 2 /* new keys and values, exports; not queries */

typedef struct agft_kv_config {
    int32_t requests;  /* rows of the block table, 1..65536 */
    int32_t row_pages; /* pages a request can hold, >= 1; row_pages * page < 2^30 */
    int32_t pages;     /* pages of the pool, 1..2^28 */
    int32_t page;      /* tokens of a page: 16, 32, 64 or 128 */
    int32_t heads;     /* key/value heads, 1..256 */
    int32_t group;     /* query heads per key/value head, 1..128 */
    int32_t dim;       /* numbers of a head: 64, 128 or 256 (others AGFT_E_UNSUPPORTED) */
    int32_t form;      /* AGFT_KV_E4M3 or AGFT_KV_INT8 */
} agft_kv_config;

/* Where the tables' and a step's parts lie in their buffers. */
typedef struct agft_kv_tables_view {
    int32_t *counters; /* [8]: ring's head, free pages, and zeros */
    int32_t *lengths;  /* [requests] */
    int32_t *table;    /* [requests][row_pages] pages of a request's tokens, in order */
    int32_t *ring;     /* [pages] free pages from the ring's head on */
} agft_kv_tables_view;

typedef struct agft_kv_step_view {
    int32_t *counters; /* [8] after the window: ring's head, free pages; the window's tokens,
                          requests refused, pages taken, pages given back; zeros */
    int32_t *lengths;  /* [requests] after the window */
    int32_t *granted;  /* [requests] new tokens that got slots */
    int32_t *starts;   /* [requests + 1] first row of each request */
    int64_t *slots;    /* [max_tokens] page * page_size + token of the page, or -1 */
} agft_kv_step_view;

/* Bytes of the device buffers; 0 if cfg (or max_tokens, 1..2^30) is invalid. */
size_t agft_kv_tables_bytes(const agft_kv_config *cfg);
size_t agft_kv_step_bytes(const agft_kv_config *cfg, int32_t max_tokens);
size_t agft_kv_cache_bytes(const agft_kv_config *cfg);
/* workspace of agft_kv_attend, whatever it holds */
size_t agft_kv_attend_bytes(const agft_kv_config *cfg, int32_t max_tokens);

int agft_kv_tables_at(const agft_kv_config *cfg, void *d_tables, size_t nbytes, agft_kv_tables_view *out);
int agft_kv_step_at(const agft_kv_config *cfg, int32_t max_tokens, void *d_step, size_t nbytes,
                    agft_kv_step_view *out);

/* Empty tables: no request holds a token, every page is free. */
int agft_kv_reset(const agft_kv_config *cfg, void *d_tables, size_t tables_bytes, void *stream);

/*
 * Plan a window: writes the step's parts, the new entries of the block table
 * and, behind the ring's tail, the pages that come free.  The tables' lengths
 * and counters stay until agft_kv_commit, so a plan can be made again.
 * d_add  int32 [requests], device.
 */
int agft_kv_plan(const agft_kv_config *cfg, void *d_tables, size_t tables_bytes, const int32_t *d_add,
                 void *d_step, size_t step_bytes, int32_t max_tokens, void *stream);

/* The planned window's lengths and counters become the tables'. */
int agft_kv_commit(const agft_kv_config *cfg, void *d_tables, size_t tables_bytes, const void *d_step,
                   size_t step_bytes, int32_t max_tokens, void *stream);

/*
 * A dense tensor [tokens][heads][dim] of a window: numbers of a head are
 * contiguous, strides count numbers.  Base and strides: multiples of 16 bytes;
 * strides of an output are not 0 (of an input they may be).
 */
typedef struct agft_kv_dense {
    void *data;
    int64_t token_stride, head_stride;
    int32_t type; /* AGFT_KV_BF16, AGFT_KV_FP16 or AGFT_KV_FP32 */
} agft_kv_dense;

/* Store the window's new keys and values [tokens][heads][dim], rows as in the
   step; tensors cover the step's tokens.  Equal types. */
int agft_kv_append(const agft_kv_config *cfg, void *d_cache, size_t cache_bytes, const void *d_step,
                   size_t step_bytes, int32_t max_tokens, const agft_kv_dense *k, const agft_kv_dense *v,
                   void *stream);

/*
 * out = softmax(scale q K^T) V for every token of the window over the tokens
 * of its request up to itself.  q and out: [tokens][heads * group][dim], bf16
 * or fp16, equal types; query heads group*h .. group*h + group-1 share
 * key/value head h.  d_lse: fp32 [max_tokens][heads * group], the natural logarithm
 * of the sums, or NULL.  Tokens that were not granted: out 0, log sum
 * -infinity.  Rows past the window's tokens are left alone.
 * max_new: no request has more new tokens than this (1..max_tokens); short
 * bounds save launches.  Where a request has more, the rows that only a saved
 * launch would have made are NaN, in out and d_lse.
 * Products and sums are kept in fp32, the sum of the probabilities too;
 * probabilities meet the values in fp16: with 2^ev_j the scale of token j's
 * values, p_j 2^ev_j keeps eleven bits (within 2^-11 of itself) down to 2^-21 of
 * the row's largest, fewer below, and is lost 2^-32 below it.  Where the exponents
 * of a request's pages lie more than 100 apart (values of 1e20 beside zeros), the
 * smaller ones' share of the sum can be lost.
 * Calls that share a step or a workspace run one after another: partial sums
 * meet there.  The step's other parts stay as they are.
 */
int agft_kv_attend(const agft_kv_config *cfg, const void *d_cache, size_t cache_bytes, const void *d_tables,
                   size_t tables_bytes, void *d_step, size_t step_bytes, int32_t max_tokens,
                   int32_t max_new, const agft_kv_dense *q, const agft_kv_dense *out, float *d_lse, float scale,
                   void *d_work, size_t work_bytes, void *stream);

/* Slots back as dense tensors [n][heads][dim]; d_slots int64 [n], -1 gives zeros.
   Equal types; the tensors' strides as in agft_kv_dense. */
int agft_kv_export(const agft_kv_config *cfg, const void *d_cache, size_t cache_bytes, const int64_t *d_slots,
                   int64_t n, const agft_kv_dense *k, const agft_kv_dense *v, void *stream);

#ifdef __cplusplus
}
#endif

#endif /* AGFT_KV_H */
