/*
 * attn_cache.h -- C ABI of libmi355attn.so: a paged cache of keys and values, and attention over it, for
 * MI355X (gfx950).
 *
 * The cache is a pool of n_pages pages.  A page holds page_size consecutive positions of one sequence,
 * for every key head:  k_pages[page][h][place][D], h < H_kv, place < page_size, and v_pages alike.
 *
 *     kind ATTN_CACHE_16BIT   elements of the type of the rows (bf16, or fp16 in the _f16 entry points)
 *     kind ATTN_CACHE_E4M3    e4m3 elements (OCP FP8, largest 448); every position and head of K and of V has a
 *                             power of two of its own, stored as its exponent + 127 in one byte of
 *                             k_scale / v_scale [page][h][place]: an element stands for e4m3 * 2^(scale - 127).
 *                             (attn_cache_write leaves 1 .. 247; a pool filled otherwise keeps to 1 .. 254)
 *
 * The calls take a batch of B sequences.  Three arrays say which rows and positions belong to whom:
 *
 *     page_table [B][table_width]   the pages of sequence b, in the order of its positions
 *     start [B+1]                   the rows start[b] .. start[b+1]-1 of a call are sequence b's, n_b in number;
 *                                   not decreasing, start[B] <= T
 *     kv_len [B]                    positions of sequence b in the cache, these rows included
 *
 * Row start[b] + i of a call is position kv_len[b] - n_b + i of sequence b, in page
 * page_table[b][position / page_size] at place position % page_size.  So a decoding step has n_b = 1, a
 * chunk of a prompt its size, a sequence that rests n_b = 0.  Rows before start[0] and from start[B] on
 * belong to nobody: they are neither read nor written.
 *
 * The arrays are device memory: their values may change between the replays of a captured graph.  The host
 * does not see them, so the kernels keep every access in bounds themselves: start is taken
 * as if clamped to [0, T], kv_len to [0, table_width * page_size]; a page number outside [0, n_pages) is no page.
 * A position without a page, or below 0, is not written, reads as zeros, and is not seen by any query.
 */
#ifndef MI355_ATTN_CACHE_H
#define MI355_ATTN_CACHE_H

#ifdef __cplusplus
extern "C" {
#endif

enum { ATTN_CACHE_16BIT = 0, ATTN_CACHE_E4M3 = 1 };

/*
 * attn_cache_write -- enqueue the copy of new rows of K and V into their pages and return (asynchronous).
 *
 *   k, v       device pointers, bf16, row t and head h of D contiguous elements at t * strides[0] + h * strides[1]
 *              (k), t * strides[2] + h * strides[3] (v): slices of a projection's rows are fine     (read only)
 *   strides    host array of 4, in elements, multiples of 8, not negative
 *   k_pages, v_pages, k_scale, v_scale   the cache; both scales are ignored (may be NULL) for ATTN_CACHE_16BIT
 *   page_table, start, kv_len            device pointers, int32                                     (read only)
 *   kind       ATTN_CACHE_16BIT or ATTN_CACHE_E4M3
 *   T, B, H_kv, n_pages, table_width     >= 1;  D 64, 128 or 256;  page_size a power of two, 16 .. 256;
 *              B and table_width * page_size at most 2^30
 *
 * ATTN_CACHE_E4M3: a row of amplitude a is stored in multiples of 2^e, the smallest e in [-126, 120] with
 * a <= 448 * 2^e, each element rounded to nearest even: a power of two keeps the division exact, so that the
 * only error is that rounding (2^-4 of the element at most, 2^-10 of 2^e for elements below 2^(e-6)).
 * Elements that would read back beyond the type's range are stored as its largest e4m3 multiple (2^-4 below
 * or less).  NaN and infinities are not checked: such a row's elements are unspecified.
 * Two rows of a call must not have the same place (pages that sequences share are written by none of them).
 *
 * Ownership, streams and errors are those of attn_fwd (attn_fwd.h); ATTN_ERR_SHAPE stands for sizes and strides, and
 * for a call that would take 2^32 threads (one head of 2^29 rows at D = 64),
 * ATTN_ERR_UNSUPPORTED for kind and page_size, ATTN_ERR_ALIGN for k, v, pages that are not 16-byte aligned, int32
 * arrays that are not 4-byte aligned and scales that are not 16-byte aligned.
 */
int attn_cache_write(const void *k, const void *v, const long long *strides,
                     void *k_pages, void *v_pages, unsigned char *k_scale, unsigned char *v_scale,
                     const int *page_table, const int *start, const int *kv_len, int kind,
                     int T, int B, int H_kv, int D, int n_pages, int page_size, int table_width, void *stream);
int attn_cache_write_f16(const void *k, const void *v, const long long *strides,
                         void *k_pages, void *v_pages, unsigned char *k_scale, unsigned char *v_scale,
                         const int *page_table, const int *start, const int *kv_len, int kind,
                         int T, int B, int H_kv, int D, int n_pages, int page_size, int table_width, void *stream);

/*
 * attn_cache_read -- enqueue the copy of the rows' positions out of the cache and return (asynchronous): the inverse of
 * attn_cache_write.  n_b = kv_len[b] reads the whole sequence.  Arguments as there, with k and v written and the cache
 * read only.  e4m3 elements are returned as the values they stand for, rounded to the row type (exact within its
 * normal range; what lies beyond the type, of a pool that rows of the other type have filled, is unspecified).  No two rows of k or of v may overlap.
 */
int attn_cache_read(void *k, void *v, const long long *strides,
                    const void *k_pages, const void *v_pages, const unsigned char *k_scale, const unsigned char *v_scale,
                    const int *page_table, const int *start, const int *kv_len, int kind,
                    int T, int B, int H_kv, int D, int n_pages, int page_size, int table_width, void *stream);
int attn_cache_read_f16(void *k, void *v, const long long *strides,
                        const void *k_pages, const void *v_pages, const unsigned char *k_scale, const unsigned char *v_scale,
                        const int *page_table, const int *start, const int *kv_len, int kind,
                        int T, int B, int H_kv, int D, int n_pages, int page_size, int table_width, void *stream);

/*
 * attn_paged_fwd -- enqueue the attention of new tokens over the cache and return (asynchronous).
 * H_q query heads share H_kv key heads: query head h reads key head h / (H_q / H_kv).  For row t = start[b] + i
 * at position p = kv_len[b] - n_b + i:
 *
 *     J       = { j : 0 <= j < kv_len[b], j has a page }                   causal == 0
 *             = { j : 0 <= j <= p, j has a page }                          causal != 0 (aligned to the last key)
 *     s_j     = scale * sum_d q[t,h,d] * k[j,h',d]
 *     lse[t,h] = ln sum_{j in J} exp(s_j),   o[t,h,:] = sum_{j in J} exp(s_j - lse) * v[j,h',:]
 *
 * An empty J gives o = 0 and lse = -inf.  (attn_fwd's causal mask is aligned to the first key; the two agree
 * where n_b = kv_len[b].)  The rows' own keys have to be in the cache: attn_cache_write comes first.
 * Products run on bf16 (fp16) MFMA with fp32 accumulation, e4m3 elements enter them as the values they stand for
 * (exact within the row type's normal range); as in attn_fwd, P is rounded to bf16 (fp16) before the second product and the
 * row sum is taken over the unrounded fp32 P.  Against 64 bits o is then off by 0.0021 to 0.0024 of its norm (bf16; 0.00028
 * fp16), of which rounding o alone makes 0.0017 (0.00021).
 *
 *   q          device pointer, bf16, row t and head h of D contiguous elements at t * strides[0] + h * strides[1]
 *   strides    host array of 2, in elements, multiples of 8, not negative
 *   o          device pointer, bf16, contiguous [T][H_q][D];  lse fp32, contiguous [T][H_q]
 *   k_pages .. kv_len, kind   as above (the cache read only)
 *   workspace  device pointer, 16-byte aligned, owned by the caller, overwritten; workspace_bytes at least
 *              attn_paged_fwd_workspace_bytes(T, B, H_q, H_kv, D), else ATTN_ERR_WORKSPACE.  It holds nothing
 *              between calls; calls that overlap in time need one each, layers that follow each other share one.
 *              It takes what the chip's workgroups leave at once, by rows (T * H_q / H_kv): at D = 128 9 MB up to 16 of
 *              them, 18 up to 32, 36 up to 128, 180 beyond; half of that at D = 64; at D = 256 18 up to 16, 36 up to 64,
 *              179 beyond; and 16 bytes for every token
 *   max_q      the largest n_b, or an upper bound (T if nothing better is known): it chooses the kernels.  A wrong
 *              value costs speed, not correctness
 *   H_q        a multiple of H_kv;  scale finite and > 0;  T * H_q and H_kv * page_size * D below 2^30
 *
 * Rows of o and lse that belong to nobody are left as they were.  NaN and infinities in q, K and V are not checked (what
 * the rows and sequences that hold them give is unspecified, causally earlier tokens of such a sequence's chunk
 * included), except that places behind a sequence's last position may hold anything.  Bitwise reproducible
 * for the same sizes, lengths and max_q (long sequences are cut into ranges whose partial results a second kernel merges;
 * the cut depends on the lengths of the whole batch).
 *
 * The host chooses the kernels by sizes alone, so a table that could hold long sequences gets the launches that those
 * need: one token over 1000 positions (16 heads, D = 64) takes 9.4 us with a table of 1000 positions and 10.6 with one
 * of 131072, one over 500 (32 heads over 8, D = 128) 9.2 and 11.0, where the narrow table saves the merge.
 */
int attn_paged_fwd(const void *q, const long long *strides, void *o, float *lse,
                   const void *k_pages, const void *v_pages, const unsigned char *k_scale, const unsigned char *v_scale,
                   const int *page_table, const int *start, const int *kv_len, int kind,
                   void *workspace, long long workspace_bytes, int max_q,
                   int T, int B, int H_q, int H_kv, int D, int n_pages, int page_size, int table_width,
                   int causal, float scale, void *stream);
int attn_paged_fwd_f16(const void *q, const long long *strides, void *o, float *lse,
                       const void *k_pages, const void *v_pages, const unsigned char *k_scale, const unsigned char *v_scale,
                       const int *page_table, const int *start, const int *kv_len, int kind,
                       void *workspace, long long workspace_bytes, int max_q,
                       int T, int B, int H_q, int H_kv, int D, int n_pages, int page_size, int table_width,
                       int causal, float scale, void *stream);

/* Bytes of workspace attn_paged_fwd (either element type) needs; -1 on invalid arguments. */
long long attn_paged_fwd_workspace_bytes(int T, int B, int H_q, int H_kv, int D);

#ifdef __cplusplus
}
#endif
#endif /* MI355_ATTN_CACHE_H */
