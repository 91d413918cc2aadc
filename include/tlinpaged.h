/*
 * libtlinattn - a paged key/value cache and the attention that reads it.
 *
 * tlinattn.h takes the history of a window as one dense tensor.  A program that serves many sequences
 * keeps their rows in pages instead: a cache is a pool of num_pages pages of page_rows rows, and a table
 * names, for every sequence, the pages that hold its rows in order.  These calls work on such a cache:
 *
 *   tlin_rope            rotary positions, and their gradient
 *   tlin_paged_append    new rows of every sequence: queries and keys rotated, keys and values put into pages
 *   tlin_paged_attn      attention of every sequence's new rows over its rows in the cache
 *   tlin_pages_reserve / _fork / _free / _compact / _copy      the pages themselves
 *
 * Conventions are those of tlinattn.h: device pointers owned by the caller, element strides with D
 * contiguous, rows in 16-byte pieces (all strides multiples of 16 bytes, a row owns D elements rounded up to
 * whole pieces), launches on `stream` without synchronising, nothing allocated, errors by return code, checks
 * on the host before any HIP call, capture into a HIP graph once a call of the same shape has run outside one.
 * What differs:
 *   - Strides are below 2^47 bytes (refused).
 *   - New rows are ragged: those of sequence s are rows starts[s] .. starts[s+1]-1 of tensors
 *     [heads, T, D], and they are the LAST rows of the sequence, which has lens[s] rows with them: row
 *     starts[s] + i is at position lens[s] - (starts[s+1] - starts[s]) + i.
 *   - A stride of 0 repeats what is read; a tensor that is written has none on an axis longer than one (refused).
 *   - A workspace belongs to a call from its first launch to the end of its last.  Calls that share one follow each other
 *     on one stream, all launches of one before the first of the next: two host threads that call at once have two.
 *   - Key heads may be shared: query head h reads key head h / (H / HK); HK divides H.
 *   - What the device arrays hold cannot be refused by the host, so the kernels check it: lengths are cut to
 *     what the table can name (table_width * page_rows) and starts to [0, T]; a page id outside
 *     [0, num_pages) names no page: its keys are not there (weight 0), rows appended to it are dropped.
 *     starts has to rise (a sequence whose starts fall has no new rows); sequences must not share new rows.
 */
#ifndef TLINPAGED_H
#define TLINPAGED_H

#include "tlinattn.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct {
    int32_t B, H, rows;  /* x is [B, H, rows, D], each >= 1 */
    int32_t D;           /* head dimension: a multiple of 4 in [8, 128] */
    int32_t rot;         /* rotated columns: even, in [2, D]; the rest stay as they are */
    int32_t interleaved; /* pair i is columns 2i, 2i+1; 0: columns i, i + rot/2 */
    int32_t transpose;   /* the transposed rotation (angles negated): the gradient of x from that of y */
    int32_t dtype;       /* tlin_dtype of x and y */
    float amplitude;     /* factor of the rotated columns, finite; 1 where positions are not scaled */
    int32_t pos_stride;  /* positions of batch b start at pos + b * pos_stride; 0: the same for all */
    int64_t x_stride[3], y_stride[3];   /* {batch, head, row}; all 0 = dense */
} tlin_rope_params;

/* y = x with pair i of a row at position p turned by the angle p * freqs[i] and multiplied by amplitude:
 *   y1 = a (x1 cos - x2 sin),  y2 = a (x1 sin + x2 cos).
 * pos: int32 [rows] or [B, rows].  freqs: double [rot/2], on the device; angles are reduced in 64 bits, so that
 * positions may be any int32.  y may be x (the same strides), and must not overlap it otherwise.  More rows than a
 * launch has workgroups for (2^24, of 1 to 16 rows with all heads) are TLIN_ERR_UNSUPPORTED. */
tlin_status tlin_rope(const tlin_rope_params *p, const void *x, void *y, const int32_t *pos, const double *freqs, void *stream);

/* Frequencies for tlin_rope, host arithmetic only: freqs[i] = base^(-2i/rot), i < rot/2, for
 *   TLIN_ROPE_PLAIN    as they are
 *   TLIN_ROPE_LINEAR   divided by factor (positions interpolated)
 *   TLIN_ROPE_BASE     base raised to base * factor^(rot/(rot-2)): the slowest pair is interpolated by factor, the
 *                      fastest not at all (rot > 2)
 *   TLIN_ROPE_PARTS    pairs that turn more than `fast` times in `trained` positions stay, those that turn less
 *                      than `slow` times are interpolated, linearly in the turns between; *amplitude is
 *                      0.1 ln(factor) + 1 (1 for the others).
 * amplitude may be NULL. */
typedef enum { TLIN_ROPE_PLAIN = 0, TLIN_ROPE_LINEAR = 1, TLIN_ROPE_BASE = 2, TLIN_ROPE_PARTS = 3 } tlin_rope_scaling;
tlin_status tlin_rope_frequencies(int32_t rot, double base, int32_t scaling, double factor, double trained, double slow,
                                  double fast, double *freqs, double *amplitude);

typedef struct {
    int32_t S, T;         /* sequences (at most 65536), new rows of all of them together (at most 2^30); each >= 1 */
    int32_t H, HK;        /* query heads, key heads; HK divides H, at most 64 query heads to a key head */
    int32_t D;            /* head dimension: a multiple of 4 in [8, 128] */
    int32_t page_rows;    /* rows of a page: a power of two in [16, 65536] */
    int32_t table_width;  /* pages that a row of the table can name */
    int32_t num_pages;    /* pages of the cache; table_width * page_rows at most 2^30 */
    int32_t max_rows;     /* most new rows of one sequence as far as the caller knows, in [1, T]: picks the kernel's
                             shape; results do not depend on it, times do: T for a step of single rows fills
                             workgroups of up to 256 rows with a few */
    int32_t dtype;        /* tlin_dtype of queries, cache and new rows */
    int32_t out_dtype;    /* tlin_dtype of O (tlin_paged_attn) */
    int32_t causal;       /* new row i of a sequence sees the rows up to its own position; 0: all lens[s] rows */
    float scale;          /* logit multiplier, > 0, its product with log2(e) finite (as logits have to be in fp32) */
    int32_t table_stride; /* elements from one sequence's table row to the next; 0 = table_width */
    /* {head, row} of [heads, T, D] tensors, {page, head, row} of the caches [num_pages, HK, page_rows, D]; all 0 =
     * dense.  Row strides below 32 MiB; a cache's page stride, and page_rows row strides, below 4 GiB. */
    int64_t q_stride[2], o_stride[2], k_stride[2], v_stride[2], kp_stride[3], vp_stride[3];
} tlin_paged_params;

/* Puts the new rows k, v [HK, T, D] into the pages at their positions.  With r (rot, interleaved, amplitude of it
 * are used) and freqs, keys are rotated on the way, and so are the queries q [H, T, D] into q_out [H, T, D] (both
 * NULL: no queries; q_out may be q).  r NULL: nothing is rotated, q is not taken.  Strides: q_stride, o_stride
 * (q_out), k_stride, v_stride.  Reserve the pages first; a page must belong to one sequence alone.  More rows than a
 * launch has workgroups for are TLIN_ERR_UNSUPPORTED, as in tlin_rope. */
tlin_status tlin_paged_append(const tlin_paged_params *p, const tlin_rope_params *r, const void *q, void *q_out,
                              const void *k, const void *v, void *k_pages, void *v_pages, const int32_t *table,
                              const int32_t *lens, const int32_t *starts, const double *freqs, void *stream);

/* O[h, t] = sum_j softmax_j(scale <Q[h, t], K_j>) V_j over the rows j of t's sequence that it sees, for every new row.
 *   q [H, T, D]; O [H, T, D] in out_dtype; lse: nullable, dense fp32 [H, T], log(sum_j exp(scale <q, k_j>)).
 * A row that sees nothing gets zeros and -infinity.  Rows of O that belong to no sequence are left as they were.
 * ws: tlin_paged_workspace_bytes(p) bytes, 256-byte aligned.  The work is cut into equal shares of rows seen, whatever
 * the lengths are, on the device; results do not depend on the order in which shares run.
 * bf16: logits, weights and their sums are fp32, the weights rounded to bf16 for the value product, whatever out_dtype is.
 * Values of rows that a new row does not see, but another row of the call does, must be finite. */
size_t tlin_paged_workspace_bytes(const tlin_paged_params *p);
tlin_status tlin_paged_attn(const tlin_paged_params *p, const void *q, const void *k_pages, const void *v_pages,
                            const int32_t *table, const int32_t *lens, const int32_t *starts, void *O, float *lse, void *ws,
                            size_t ws_bytes, void *stream);

/* ---- pages.  A cache's book is on the device: table int32 [S, table_width] (row stride table_stride), lens int32
 * [S], refs int32 [num_pages], the number of table entries that name a page; 0: it is free.  Sequence s holds the
 * first ceil(lens[s] / page_rows) entries of its row, the others are -1. */
typedef struct {
    int32_t S, table_width, num_pages, page_rows; /* as in tlin_paged_params */
    int32_t table_stride;                         /* 0 = table_width */
} tlin_book_params;

/* Every listed sequence gives up its pages: refs of each one less, its table row -1, its length 0.  seqs int32 [n], n
 * at most 65536.  A sequence listed twice is freed once; ids outside [0, S) are passed over. */
tlin_status tlin_pages_free(const tlin_book_params *p, int32_t *table, int32_t *lens, int32_t *refs, const int32_t *seqs,
                            int32_t n, void *stream);

/* Sequence children[i] becomes a copy of sequence parents[i]: it names the same pages (refs of each one more) and has
 * the same length.  n at most 65536.  status int32 [n]: 0, or 1 where the pair was passed over: an id outside [0, S), a child that holds
 * rows, that an earlier pair names as a child, or that any pair names as a parent. */
tlin_status tlin_pages_fork(const tlin_book_params *p, int32_t *table, int32_t *lens, int32_t *refs,
                            const int32_t *parents, const int32_t *children, int32_t n, int32_t *status, void *stream);

/* Room for want[s] more rows of every sequence: pages are added from the free ones, lowest ids first, in the order of
 * sequences, and lens[s] grows by want[s].  Where the last page of a sequence that grows is not full and has
 * refs > 1 when the call begins, the sequence gets a page of its own in its place; the pairs (old, new) are listed in
 * moves int32 [S, 2], in the order of sequences, count[0] of them, the other entries are -1, for
 * tlin_pages_copy.  status int32 [S]: 0, or 1 where the row of the table or the free pages do not suffice (or want < 0):
 * that sequence is left as it was (pages are handed out in order of sequences: once the free ones do not suffice for
 * one, later ones that need any get none either).  ws: tlin_pages_workspace_bytes(p) bytes, 256-byte aligned. */
size_t tlin_pages_workspace_bytes(const tlin_book_params *p);
tlin_status tlin_pages_reserve(const tlin_book_params *p, int32_t *table, int32_t *lens, int32_t *refs, const int32_t *want,
                               int32_t *moves, int32_t *count, int32_t *status, void *ws, size_t ws_bytes, void *stream);

/* Brings the L pages that are in use to ids below L: the i-th free id below L, from the lowest up, takes the i-th page in
 * use from the highest down.  Writes the pairs (old, new) to moves int32 [num_pages / 2, 2], count[0] of them, the other
 * entries are -1, and the book after it to table_out (strides as table) and refs_out, which may be table and refs.
 * The pages' contents are moved by tlin_pages_copy. */
tlin_status tlin_pages_compact(const tlin_book_params *p, const int32_t *table, const int32_t *refs, int32_t *table_out,
                               int32_t *refs_out, int32_t *moves, int32_t *count, void *ws, size_t ws_bytes, void *stream);

/* Copies pages inside caches: for each of the first min(count[0], max_moves) pairs (from, to) of moves int32 [max_moves,
 * 2] the rows of page `from` to page `to`, in the caches a and b (b may be NULL) and in each of `layers` layers of
 * them.  No page may be both written and read, or written twice, in one call.  Pairs with an id outside [0, num_pages)
 * are passed over.  count NULL: all max_moves pairs.  Rows are copied in whole 16-byte pieces. */
typedef struct {
    int32_t layers, num_pages, HK, page_rows, D;
    int32_t dtype;
    int64_t layer_stride[2];        /* elements from a layer to the next, of a and of b; 0 = num_pages pages */
    int64_t a_stride[3], b_stride[3];   /* {page, head, row}; all 0 = dense */
} tlin_cache_params;
tlin_status tlin_pages_copy(const tlin_cache_params *p, void *a, void *b, const int32_t *moves, const int32_t *count,
                            int32_t max_moves, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* TLINPAGED_H */
