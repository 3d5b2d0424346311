/*
 * attn_evict.h -- C ABI of libmi355attn.so: what attention has looked at in the paged cache of attn_cache.h, which places it
 * keeps, and moving them together, for MI355X (gfx950).
 *
 * A sequence that may keep fewer positions than it has drops the ones that attention looks at least, each key head its own:
 *
 *     attn_cache_weigh    adds the attention weights of new tokens to what every cached position has had
 *     attn_cache_select   finds, for every sequence and key head, the places to keep, as a list of moves: kept places behind the
 *                         new end go into dropped places before it
 *     attn_cache_move     carries moves out; it also moves an accepted path of a tree of drafts (attn_tree.h) together
 *
 * A cached key has its position turned into it, so the order of the places means nothing to attention.  Beside the cache a
 * program keeps, for every sequence of its batch, key head and place,
 *
 *     weights [B][H_kv][table_width * page_size]   fp32, the accumulated weight of what lies there
 *     stamps  [B][H_kv][table_width * page_size]   int32, the number of the token that lies there, 0 for a sequence's first
 *                                                  (optional: without evictions, or with one only, the place says it)
 *
 * with seen [B], int32, the tokens that a sequence has had in all, as kv_len counts what of them is left.  After an eviction
 * all key heads of a sequence have the same number of places, so page_table and kv_len stay as they are in attn_cache.h; pages
 * behind the new length are the caller's again.  Every array is device memory, brought into range by the kernels, so that captured
 * steps can be replayed as lengths change.  Ownership, streams and errors are those of attn_fwd (attn_fwd.h).
 */
#ifndef MI355_ATTN_EVICT_H
#define MI355_ATTN_EVICT_H

#ifdef __cplusplus
extern "C" {
#endif

/*
 * attn_cache_weigh -- enqueue the accumulation of attention weights and return (asynchronous).  For sequence b with n_b > 0 rows
 * t = start[b] + i, key head h with its H_q / H_kv query heads, and every position 0 <= j < kv_len[b]:
 *
 *     w[j]  = sum over rows t that see j and query heads hq of h:  exp(scale * q[t,hq] . k[j,h] - lse[t,hq])
 *     weights_out[b,h,j] = w[j]                                 j >= kv_len[b] - n_b: the rows' own positions begin here
 *                        = decay * weights[b,h,j] + w[j]        otherwise (decay == 0 or weights NULL: w[j], nothing is read)
 *     stamps[b,h,j]      = seen[b] - kv_len[b] + j              j >= kv_len[b] - n_b, if stamps are given
 *
 * Row t sees j <= its own position if causal != 0, otherwise all; a position without a page is seen by none, and a row whose lse is -inf
 * sees nothing.  Sums are fp32, in a fixed order: bitwise reproducible.  Places from kv_len[b] on and sequences
 * without rows are not written.
 *
 *   q, strides, k_pages, k_scale, page_table, start, kv_len, kind, T .. table_width, max_q, causal, scale
 *                 as in attn_paged_fwd (attn_cache.h), whose limits hold
 *   lse           device pointer, fp32, contiguous [T][H_q]: what attention has left for these rows.  The rows of a tree of
 *                 drafts (attn_tree.h) are weighed once their accepted path has moved together: its rows' q and lse, kv_len
 *                 with them; causally each then sees what its mask showed it
 *   weights, weights_out   device pointers, 16-byte aligned, contiguous; the same array, or two that do not overlap
 *                 (ATTN_ERR_SHAPE).  B * H_kv * table_width * page_size at most 2^40
 *   stamps, seen  device pointers, both or neither (ATTN_ERR_NULL); stamps 16-byte aligned
 *   decay         finite and >= 0, else ATTN_ERR_SCALE
 *
 * scale * log2(e) and lse * log2(e) are fp32 numbers, as the scores are: against 64 bits the weights are off by 2.5e-8 to 5.1e-7 of their norm
 * (the formula in fp32 with the exponential of scale * q.k - lse: 2.5e-8 to 4.3e-7).
 *
 * NaN and infinities in a row's q or lse make all weights of its sequence and head unspecified, those in a position's k that position's.
 */
int attn_cache_weigh(const void *q, const long long *strides, const float *lse, const void *k_pages, const unsigned char *k_scale,
                     const int *page_table, const int *start, const int *kv_len, int kind,
                     const float *weights, float *weights_out, int *stamps, const int *seen, float decay, int max_q,
                     int T, int B, int H_q, int H_kv, int D, int n_pages, int page_size, int table_width,
                     int causal, float scale, void *stream);
int attn_cache_weigh_f16(const void *q, const long long *strides, const float *lse, const void *k_pages, const unsigned char *k_scale,
                         const int *page_table, const int *start, const int *kv_len, int kind,
                         const float *weights, float *weights_out, int *stamps, const int *seen, float decay, int max_q,
                         int T, int B, int H_q, int H_kv, int D, int n_pages, int page_size, int table_width,
                         int causal, float scale, void *stream);

/*
 * attn_cache_select -- enqueue the choice of what a cache keeps and return (asynchronous).  For every sequence b and key head h:
 * of the places j < kv_len[b] the keep[b] first ones are kept, in this order: those of a token that always stays (its number is below
 * sinks, or at least seen[b] - recent), then by falling weight; ties go to the lowest place, NaN ranks below everything.
 *
 *     new_len[b]       = min(kv_len[b], max(keep[b], 0))
 *     dst[b,h,0..m-1]  the places below new_len[b] that are dropped, ascending
 *     src[b,h,0..m-1]  the places from new_len[b] on that are kept, ascending (as many)
 *     dst, src[b,h,m..width-1] = -1
 *
 * With attn_cache_move (dst <- src) the kept places are the first new_len[b].  m is at most min(new_len[b], kv_len[b] - new_len[b]): a sequence
 * for which that bound exceeds moves_width drops nothing (new_len[b] = kv_len[b], all of its lists -1).
 *
 *   weights    device pointer, fp32, 16-byte aligned, contiguous [B][H_kv][width]                             (read only)
 *   stamps     device pointer, int32, 16-byte aligned, like weights, or NULL: a place's token is the place     (read only)
 *   seen       device pointer, int32 [B], or NULL: kv_len (both with stamps, else ATTN_ERR_NULL)              (read only)
 *   kv_len, keep   device pointers, int32 [B]; kv_len is taken as if clamped to [0, width]                    (read only)
 *   dst, src   device pointers, int32, contiguous [B][H_kv][moves_width]; every element is written
 *   new_len    device pointer, int32 [B], not the memory of kv_len, keep or seen (ATTN_ERR_SHAPE)
 *   width      a multiple of 16, up to 2^30;  moves_width >= 1;  B, H_kv >= 1, B * H_kv * max(width, moves_width) at most 2^40,
 *              B * H_kv below 2^22
 *   sinks, recent   >= 0
 *   workspace  device pointer, 16-byte aligned, owned by the caller, overwritten; workspace_bytes at least
 *              attn_cache_select_workspace_bytes(B, H_kv, width), else ATTN_ERR_WORKSPACE; NULL where that is 0.  It holds nothing
 *              between calls; calls that overlap in time need one each
 *
 * The host does not see kv_len, so the width says which kernels run: 512 lists of 2176 places, each in a row of 2176 or of 16384, take 12.6
 * or 13.0 us, in a row of 32768 or of 131072 102 or 92.
 */
int attn_cache_select(const float *weights, const int *stamps, const int *seen, const int *kv_len, const int *keep,
                      int *dst, int *src, int *new_len, int sinks, int recent, void *workspace, long long workspace_bytes,
                      int B, int H_kv, int width, int moves_width, void *stream);

/* Bytes of workspace attn_cache_select needs; -1 on invalid arguments.  0 for a width of up to 16384 places.  Beyond, 24580 bytes for every part
 * of a list and 16 for the list, which has ceil(width / part) + 2 of them: parts of 16384 places up to 2^20, and of as many times that beyond
 * as leave no more than 66.  98 KB a list of 16400 places, 246 KB of 131072, 1.6 MB at most. */
long long attn_cache_select_workspace_bytes(int B, int H_kv, int width);

/*
 * attn_cache_move -- enqueue moves of cached positions and return (asynchronous): for every sequence b, key head h and list element e,
 * what lies at place src[b,h,e] of the sequence (key, value, their scales, and weight and stamp if given) goes to place dst[b,h,e].
 * The source keeps what it has.
 *
 *   k_pages .. k_scale, v_scale, page_table, kind, H_kv .. table_width   the cache, as in attn_cache.h; 16-bit elements are
 *                    copied as they are, whatever their type
 *   dst, src         device pointers, int32, contiguous [B][list_heads][moves_width]; list_heads is H_kv, or 1: one list for all heads
 *   weights, stamps  device pointers, contiguous [B][H_kv][table_width * page_size], 4-byte aligned, or NULL (each)
 *
 * An element with a place outside [0, table_width * page_size), or one without a page, moves nothing.  No place may be twice in a list's
 * dst.  In lists of up to 128 elements (moves_width) a place may be both source and destination: all sources of a
 * list are read before anything is written.  In longer ones no place may be both, which attn_cache_select's lists keep to.  Pages that
 * sequences share may not be written by one of them while another one reads them.  A call of 2^32 threads or more is refused
 * (ATTN_ERR_SHAPE).
 *
 * An accepted path m_0 < m_1 < ... of the n_b drafted tokens of a sequence: dst = kv_len - n_b + 0, 1, ..., src = kv_len - n_b + m_0,
 * m_1, ... with list_heads 1; the new kv_len is kv_len - n_b + the path's length.  Its places overlap, so a call takes at most 128
 * tokens of it (moves_width): a longer path in one call leaves it to the order of the workgroups what is read.  Calls of up to 128
 * elements each, in ascending order on one stream, move a path of any length: m_i >= i, so none writes what a later one reads.
 */
int attn_cache_move(void *k_pages, void *v_pages, unsigned char *k_scale, unsigned char *v_scale, const int *page_table,
                    const int *dst, const int *src, int kind, float *weights, int *stamps,
                    int list_heads, int moves_width, int B, int H_kv, int D, int n_pages, int page_size, int table_width,
                    void *stream);

#ifdef __cplusplus
}
#endif
#endif /* MI355_ATTN_EVICT_H */
