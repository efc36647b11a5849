/*
 * agft_pages.h -- C ABI of which requests of a serving node hold which pages of
 * its cache (agft_kv.h), on AMD Instinct MI355X (gfx950): requests that continue
 * others' tokens, tokens taken back, and held pages moved together.
 *
 * A change of the tables is an edit.  Like a window, it is planned, then made in
 * every layer's cache, then committed:
 *
 *   agft_pages_fork, agft_pages_trim or agft_pages_compact
 *   per layer:
 *   agft_pages_copy    the edit's pages are copied (a trim has none)
 *   agft_pages_commit  the edit's lengths, pages and counters become the tables'
 *
 * A plan can be made again; until the commit the tables' lengths, counters and
 * owners and the pages that requests hold stay as they are.  Plans of windows and
 * of edits count on the tables as they find them: commit one before the next is
 * planned, and commit an edit once.
 *
 * Owners.  A page may be held by several requests: owners counts those beyond the
 * first, and the tables' counters[2] is the sum over all pages (less than 2^31).
 * Only pages whose tokens are all there are shared, so no write meets a shared
 * page (whoever fills the tables otherwise sees to that).  While counters[2] is not 0, requests end by agft_pages_trim: agft_kv_plan
 * refuses an end (add < 0) then, leaves the request as it is and counts it among
 * the refused ones.  Whoever fills the tables with pages in common and does not count
 * their owners sets counters[3] to 1: trims refuse every request then as well, since no
 * page could be told to be free.
 *
 * Fork.  For j = 0 .. n - 1 request dst_j gets the first t_j = min(tokens_j,
 * L(src_j)) tokens of request src_j.  It is asked for if src_j and dst_j are
 * requests, differ, dst_j holds nothing and is named once in dst, and t_j > 0; it
 * needs a page if page does not divide t_j:
 *
 *   granted_j = t_j  if asked for and (need_j = 0 or sum_{i<=j} need_i <= free),  else 0.
 *
 * The floor(t_j / page) whole pages are shared.  A page that t_j fills in part is
 * copied into a fresh one from the ring's head: moves_j = (old, fresh), else (-1,
 * -1).  Lengths are those before the call, so a request that another fork of the
 * call fills has none to give.
 *
 * Trim.  Request i keeps keep_i tokens, if 0 <= keep_i < L_i (else all of them; 0
 * ends it).  One that would end inside a page with further owners is refused: its
 * next tokens would be written there (fork what it is to keep, and end it); all are while
 * owners are not counted.  Pages
 * go back behind the ring's tail when their last owner lets them go, in the order
 * of the requests and of their pages, a page that several let go in the place of
 * the last.
 *
 * Compact.  With n pages not free, the ones from n on move to the free ones below
 * n, both in ascending order: moves_k = (k-th held page >= n, k-th free one < n),
 * (-1, -1) from the last move on.  The ring becomes 0, 1, .. pages - 1 and its
 * head n: pages n .. pages - 1 are free, in ascending order.
 *
 * Memory, streams and errors are those of agft_kv.h.  Every page number that a
 * kernel takes from memory is held to the pool, and every request's to the table.
 */
#ifndef AGFT_PAGES_H
#define AGFT_PAGES_H

#include "agft_kv.h"

#ifdef __cplusplus
extern "C" {
#endif

/* agft_pages_view.counters[7]: what the edit is */
#define AGFT_PAGES_FORK 1
#define AGFT_PAGES_TRIM 2
#define AGFT_PAGES_COMPACT 3

/* Where an edit's parts lie in its buffer. */
typedef struct agft_pages_view {
    int32_t *counters; /* [8] after the edit: ring's head, free pages, owners beyond the first of all pages;
                          requests refused, pages taken, pages given back, entries of moves, kind */
    int32_t *lengths;  /* [requests] after the edit */
    int32_t *granted;  /* [max_moves] of a fork: tokens that dst_j got */
    int32_t *moves;    /* [max_moves][2] pages to copy: from, to; -1 where there is none */
} agft_pages_view;

/* Bytes of an edit's buffer; 0 if cfg (or max_moves, 1..2^27) is invalid. */
size_t agft_pages_edit_bytes(const agft_kv_config *cfg, int32_t max_moves);
int agft_pages_edit_at(const agft_kv_config *cfg, int32_t max_moves, void *d_edit, size_t nbytes, agft_pages_view *out);

/* Owners beyond the first, int32 [pages], in the tables' buffer (agft_kv_reset sets them to 0; whoever fills the tables
   otherwise fills these and counters[2], or sets counters[3], too). */
int agft_pages_owners_at(const agft_kv_config *cfg, void *d_tables, size_t nbytes, int32_t **out);

/*
 * Plans.  d_src, d_dst, d_tokens  int32 [n], device, 1 <= n <= min(65536, max_moves); d_tokens NULL: all tokens.
 * d_keep  int32 [requests], device.  A compaction's max_moves is at least pages / 2.
 */
int agft_pages_fork(const agft_kv_config *cfg, void *d_tables, size_t tables_bytes, const int32_t *d_src,
                    const int32_t *d_dst, const int32_t *d_tokens, int32_t n, void *d_edit, size_t edit_bytes,
                    int32_t max_moves, void *stream);
int agft_pages_trim(const agft_kv_config *cfg, void *d_tables, size_t tables_bytes, const int32_t *d_keep, void *d_edit,
                    size_t edit_bytes, int32_t max_moves, void *stream);
int agft_pages_compact(const agft_kv_config *cfg, void *d_tables, size_t tables_bytes, void *d_edit, size_t edit_bytes,
                       int32_t max_moves, void *stream);

/* Copy the planned edit's pages, codes and exponents, in one layer's cache (layers may differ in dim and form). */
int agft_pages_copy(const agft_kv_config *cfg, void *d_cache, size_t cache_bytes, const void *d_edit, size_t edit_bytes,
                    int32_t max_moves, void *stream);

/* The planned edit becomes the tables'. */
int agft_pages_commit(const agft_kv_config *cfg, void *d_tables, size_t tables_bytes, const void *d_edit,
                      size_t edit_bytes, int32_t max_moves, void *stream);

#ifdef __cplusplus
}
#endif

#endif /* AGFT_PAGES_H */
