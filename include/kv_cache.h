/*
 * kv_cache.h -- C ABI of the gfx950 (MI355X) operators around a paged cache of keys and values: rotary positions, writing new
 * tokens to the cache, attention of new tokens over it, and the upkeep of its pages.
 *
 * The attention is the operation of attn_fwd.h for a serving program: the keys and values of a sequence lie in pages of a common
 * pool instead of one array, a call takes a packed batch of sequences of any lengths with one or more new tokens each, and several
 * query heads may share a key head.
 *
 * Conventions of every entry point.  All data pointers (arrays inside the structs too) are DEVICE pointers; the structs
 * themselves are read on the host during the call.  The caller owns every buffer; the library allocates nothing, retains nothing
 * and never synchronises: a call validates its arguments on the host, enqueues its kernels on `stream` (a hipStream_t passed as
 * void*, NULL = the default stream) on the current device and returns.  Calls are thread safe, and may be captured into a graph:
 * everything that a replay reads afresh (lengths, tables, positions, tokens) is read on the device.  Calls that may run at the same time must
 * not share a workspace.  Validation happens before any HIP call; nothing is enqueued when an error is returned.
 *
 * What only the device knows is not trusted: lengths and starts outside their bounds are brought into them, a page number outside
 * 0 ... pages - 1 is no page (nothing is read from it or written to it), whatever the arrays hold.
 */
#ifndef KV_CACHE_H
#define KV_CACHE_H

#ifdef __cplusplus
extern "C" {
#endif

enum {
    KV_OK = 0,
    KV_ERR_NULL = -1,       /* a pointer argument is NULL */
    KV_ERR_SHAPE = -2,      /* a size, a type code or a combination of them that is not supported */
    KV_ERR_SCALE = -3,      /* scale is NaN, infinite, zero or negative, or amplitude is NaN or infinite */
    KV_ERR_ALIGN = -4,      /* a pointer or a stride is not aligned */
    KV_ERR_OVERFLOW = -5,   /* too large for the kernels' index arithmetic or for a grid */
    KV_ERR_LAUNCH = -6,     /* the HIP runtime refused a launch */
    KV_ERR_ALIAS = -7,      /* an output (a workspace, a book that is changed) overlaps an input (arrays of a batch, lists, scales too) or another output */
    KV_ERR_STRIDE = -8,     /* a stride is smaller than a row, so rows would overlap */
    KV_ERR_WORKSPACE = -9   /* the workspace is smaller than the call needs */
};

/* Element types: 16-bit ones for tokens, all three for caches (E4M3: 1 sign, 4 exponent bits with bias 7, 3 fraction bits, no infinities). */
enum { KV_FP16 = 0, KV_BF16 = 1, KV_E4M3 = 2 };

/* Which elements of a head make a pair: i and i + rot/2, or 2i and 2i + 1. */
enum { KV_HALF = 0, KV_INTERLEAVED = 1 };

/*
 * A cache.  Element e of token t of page p, head h, layer l stands at
 *     l * layer_stride + p * page_stride + h * head_stride + t * token_stride + e        (in elements, for k and for v alike)
 * from k or v, so any order of the dimensions is a matter of the strides.  Rows (d elements) must not overlap; every stride of a
 * dimension larger than one is >= d, k and v are 16-byte aligned and strides are multiples of 16 bytes.  Where the cache is written, rows of k and of v must not
 * meet either; they may lie between each other where every stride steps over all that lies inside it.
 *   k_scale, v_scale   float32 [heads], both or neither; only with KV_E4M3, where a stored value x stands for x * scale (NULL: scales
 *                      of 1).  Finite and > 0.
 *   page_size          tokens per page: a power of two, 16 ... 4096.    d: 64 or 128.
 */
typedef struct kv_pages {
    void *k, *v;
    const float *k_scale, *v_scale;
    long long layer_stride, page_stride, head_stride, token_stride;
    int layers, pages, heads, page_size, d, dtype;
} kv_pages;

/*
 * A packed batch.  The new tokens of sequence s are the rows q_start[s] ... q_start[s + 1] - 1 of the token arrays, and are the LAST
 * of the kv_len[s] tokens that it has: token i of its n new ones has position kv_len[s] - n + i.  Rows from q_start[sequences] on
 * belong to nobody and are left as they are in every output.
 *   q_start      int32 [sequences + 1], not falling, 0 ... tokens.       kv_len   int32 [sequences].
 *   table        int32 [sequences][table_width], rows table_stride entries apart: page of the tokens j * page_size ... of a sequence.
 *   max_q        no sequence has more new tokens than this; max_kv: none is longer.  max_kv <= table_width * page_size.
 * Both bounds choose the launch (a tight one is faster).  Of a sequence beyond them, the first max_q new tokens and those at positions below max_kv are worked on, at the
 * positions that they have; the rest counts neither as tokens nor as keys, and its rows are left as they are in every output.
 */
typedef struct kv_batch {
    const int *q_start, *kv_len, *table;
    int sequences, tokens, table_width, table_stride, max_q, max_kv;
} kv_batch;

/* Heads of tokens: element e of head h of token t at t * token_stride + h * head_stride + e from p (in elements). */
typedef struct kv_rows {
    void *p;
    long long token_stride, head_stride;
} kv_rows;

/*
 * Attention of the new tokens over the cache.  For query head h (key head h / (heads / cache->heads)) of token i of a sequence with n new
 * ones:
 *     s_j = scale * <q, k_j>,  j < kv_len, causal: j <= kv_len - n + i;    O = sum_j softmax_j(s) v_j,    LSE = ln sum_j exp(s_j)
 * Keys in no page (see above) weigh nothing.  A row that sees no key has O = 0 and LSE = -infinity.
 *   q      tokens x heads rows of `dtype` (KV_FP16 / KV_BF16); heads a multiple of cache->heads.  A 16-bit cache has the same type.
 *   o      the same shape and type, written; rows must not overlap each other or any input.
 *   lse    float32 [tokens][heads], written; NULL: not wanted.
 * Layer 0 of the cache is read (a caller with several points k and v at the one it means).
 * Keys and values that a row does not see have no influence on it, NaN and infinities among them; a NaN in a key or value that it sees
 * makes the row NaN (in the value: the features that have one) and an infinity in a value makes the feature NaN or infinite, whatever the key's weight.
 * Scores, maxima and sums are float32; the weights are rounded to `dtype` for the product with V (values up to 2^8 relative to a
 * reference inside the row) and O is divided by the sum of the rounded ones, so it is a mean of the values; the LSE is that of the weights before rounding.  An E4M3
 * cache is widened to `dtype` without rounding.
 *   workspace   attn_paged_workspace bytes, 16-byte aligned (NULL if that is 0); need not be initialised.
 */
int attn_paged(const kv_pages *cache, const kv_batch *batch, const kv_rows *q, const kv_rows *o, float *lse, int heads, float scale, int causal,
               int dtype, void *workspace, long long workspace_bytes, void *stream);

/* Host-only argument check: what attn_paged would return before launching. */
int attn_paged_check_args(const kv_pages *cache, const kv_batch *batch, const kv_rows *q, const kv_rows *o, const float *lse, int heads, float scale,
                          int dtype, const void *workspace, long long workspace_bytes);

/* Bytes of workspace for a call with these sizes (of the batch: sequences, tokens, max_q, max_kv); -1 for sizes that no call accepts. */
long long attn_paged_workspace(const kv_pages *cache, const kv_batch *batch, int heads);

/*
 * Rotary positions.  Of every head the first `rot` elements are turned, pair m by the angle position * freq[m] (in radians), and multiplied by
 * `amplitude`; the others are copied:
 *     y_a = amplitude (x_a cos - x_b sin),  y_b = amplitude (x_b cos + x_a sin)
 * with (a, b) = (m, m + rot/2) or (2m, 2m + 1) by `layout`.  `inverse` turns back (the sign of the angle): that is the gradient with respect to
 * x for a gradient with respect to y, amplitude included.  The angle is computed in 64 bits and reduced there, its sine and cosine
 * and the products in 32, the result is rounded once.  rope_frequencies gives the usual frequencies.
 *   x, y     element e of head h of token n of batch b at b * batch_stride + h * head_stride + n * token_stride + e; d elements.  y == x with
 *            equal strides turns in place; otherwise they must not overlap.
 *   pos      int32, position of token n of batch b at b * pos_stride + n (pos_stride 0: the same for every batch); NULL: position n.
 *   freq     float64 [rot / 2] on the device.
 *   d        a multiple of 16, 16 ... 1024; rot a multiple of 16, 16 ... d.  Pointers and strides are multiples of 16 bytes (x, y), 8 bytes (freq), 4 (pos).
 */
typedef struct rope_tensor {
    void *p;
    long long batch_stride, head_stride, token_stride;
} rope_tensor;

int rope(const rope_tensor *x, const rope_tensor *y, int batches, int heads, int tokens, int d, const int *pos, long long pos_stride,
         const double *freq, int rot, int layout, float amplitude, int inverse, int dtype, void *stream);

/* Host-only argument check: what rope would return before launching. */
int rope_check_args(const rope_tensor *x, const rope_tensor *y, int batches, int heads, int tokens, int d, const int *pos, long long pos_stride,
                    const double *freq, int rot, int layout, float amplitude, int dtype);

/*
 * Frequencies in HOST memory, freq[m] = base^(-2m/rot) for m < rot/2, for a context `factor` times the trained one:
 *   ROPE_PLAIN     as they are (factor is ignored).
 *   ROPE_LINEAR    positions squeezed: freq / factor.
 *   ROPE_BASE      the base raised to base * factor^(rot / (rot - 2)): the slowest pair is stretched by factor, the fastest stays.  rot > 2.
 *   ROPE_PARTS     pair by pair, by the turns that it makes in `trained` positions, trained * freq / (2 pi): from `high` turns on it stays, up to
 *                  `low` turns it is freq / factor, in between both are mixed in proportion.
 * rot even, 2 ... 1024; base > 1, factor >= 1, trained > 0, 0 <= low < high, all finite (trained, low, high with ROPE_PARTS only): else KV_ERR_SHAPE.
 */
enum { ROPE_PLAIN = 0, ROPE_LINEAR = 1, ROPE_BASE = 2, ROPE_PARTS = 3 };
int rope_frequencies(double *freq, int rot, double base, int scaling, double factor, double trained, double low, double high);

/*
 * New tokens into the cache, in one launch: K is turned by its position (if freq is given) and stored, V is stored, Q is turned into q_out.
 *   k, v     tokens x cache->heads rows of `dtype`.       q, q_out   tokens x heads rows; both with p NULL (or the pointers NULL): no Q.
 *   freq, rot, layout, amplitude   as for rope; freq NULL: nothing is turned (then q must not be given), rot 0.
 * A 16-bit cache has the type of the tokens.  With KV_E4M3 a value is divided by its head's scale and rounded to nearest even, beyond +-448 to
 * +-448, NaN stays NaN.  A token at a negative position (kv_len smaller than the new tokens) or in no page is not stored; its Q is turned all the same.
 * Two new tokens must not share a place (a page that two sequences share is copied before either writes to it: see kv_fork).
 * Layer 0 of the cache is written.  No output may overlap an input or another output, but q_out may be q (same pointer and strides); rows that lie in
 * each other's gaps (heads of one array of tokens, as a projection of Q, K and V together leaves them) do not overlap.
 */
int kv_append(const kv_pages *cache, const kv_batch *batch, const kv_rows *k, const kv_rows *v, const kv_rows *q, const kv_rows *q_out, int heads,
              const double *freq, int rot, int layout, float amplitude, int dtype, void *stream);

/* Host-only argument check: what kv_append would return before launching. */
int kv_append_check_args(const kv_pages *cache, const kv_batch *batch, const kv_rows *k, const kv_rows *v, const kv_rows *q, const kv_rows *q_out,
                         int heads, const double *freq, int rot, int layout, float amplitude, int dtype);

/*
 * The upkeep of pages, on the device so that a captured step can do it.  The book of a cache:
 *   ref       int32 [pages], how many table entries hold the page; 0: free.
 *   table     int32 [rows][table_width], rows table_stride apart; kv_len int32 [rows]: row r holds the first ceil(kv_len[r] / page_size) entries of its row.
 * Pages are given out lowest number first.  Lists of rows and pages are int32 arrays on the device; entries outside their range are passed over.
 * All results are whole numbers and the same from run to run.
 */
typedef struct kv_book {
    int *ref, *table, *kv_len;
    int pages, rows, table_width, table_stride, page_size;
} kv_book;

/* Most rows in one list (of kv_reserve also: rows x table_width below 2^31, so that the pages wanted can be counted). */
enum { KV_MAX_LIST = 8192 };

/*
 * Room for growth: row list[i] gets pages for new_len[i] tokens in all (entries behind those it holds, in the order of the list and then of the
 * tokens) and kv_len = new_len[i]; a row that is as long already stays as it is.  What is longer than the table is cut to its width.
 * *missing is the number of pages that were not there: their entries are -1.  No row twice in a list.
 * kv_len counts the tokens of missing pages all the same (kv_append passes over them, attention sees nothing there), and an entry that was missing stays so: later calls
 * begin behind what kv_len counts, for a page given out there would show what its last owner left in it.  Such a row is given back and begun anew, or, before it
 * grows again and before anything is appended to it, its kv_len is set to page_size x the entries that it has (the missing ones are its last) and the call made again.
 */
int kv_reserve(const kv_book *book, const int *list, const int *new_len, int n, int *missing, void *stream);

/* The rows' pages are given back (a page is free when its last holder has gone), their entries become -1 and kv_len 0.  A row twice counts once. */
int kv_free(const kv_book *book, const int *list, int n, void *stream);

/*
 * Row dst[i] becomes a continuation of row src[i], i = 0 ... n - 1: full pages are shared, a last page that is not full is copied to a new one (all
 * layers, keys and values).  What a dst row held before is overwritten, not given back (kv_free does that).  *missing as above: such
 * a row has -1 for its last page.  A page that src does not have (its entry is none, see kv_reserve) dst does not have either: a last one has
 * -1 there, takes no page and is not counted in *missing.  No row twice in dst, no dst in src.
 */
int kv_fork(const kv_pages *cache, const kv_book *book, const int *src, const int *dst, int n, int *missing, void *stream);

/*
 * Pages in use move together: with u of them in use, the i-th (by number) of those numbered u or more moves to the i-th free one below u, contents, ref and table
 * entries.  Afterwards the pages 0 ... u - 1 are in use.  workspace: kv_compact_workspace(pages) bytes, 16-byte aligned.
 */
int kv_compact(const kv_pages *cache, const kv_book *book, void *workspace, long long workspace_bytes, void *stream);
long long kv_compact_workspace(int pages);

/* Page src[i] is copied to page dst[i], all layers, keys and values.  No page twice in dst, no dst in src. */
int kv_copy_pages(const kv_pages *cache, const int *src, const int *dst, int n, void *stream);

/* Static, NUL-terminated description of a return code.  Never NULL. */
const char *kv_strerror(int code);

#ifdef __cplusplus
}
#endif

#endif /* KV_CACHE_H */
