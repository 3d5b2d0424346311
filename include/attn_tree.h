/*
 * attn_tree.h -- C ABI of libmi355attn.so: attention of a tree of drafted tokens over the paged cache of attn_cache.h, for
 * MI355X (gfx950).
 */
#ifndef MI355_ATTN_TREE_H
#define MI355_ATTN_TREE_H

#ifdef __cplusplus
extern "C" {
#endif

/*
 * attn_paged_tree -- enqueue the attention of drafted tokens over the cache and return (asynchronous): attn_paged_fwd
 * (attn_cache.h) with a mask among a sequence's new tokens.  Row t = start[b] + i, at position kv_len[b] - n_b + i, sees
 *
 *     J = { j : 0 <= j < kv_len[b] - n_b, j has a page }                             all that lay there before
 *       + { kv_len[b] - n_b + m : 0 <= m < n_b, bit m of the row is set, a position >= 0 that has a page }
 *
 *   mask        device pointer, 8-byte aligned, contiguous [T][mask_words] words of 64 bits: bit m % 64 of word m / 64 of row t
 *               says that row t sees row start[b] + m of its own sequence                               (read only)
 *   mask_words  1 .. 1024; new tokens behind the mask's last bit are seen by none
 *
 * A token of a tree of drafts sees its ancestors and itself, but any set will do: a row's own bit is not taken for granted, and
 * bits from n_b on are ignored.  A lower triangle gives attn_paged_fwd's causal mask.  The drafted tokens' keys and values have
 * to be in the cache, in the order of the rows (attn_cache_write); attn_cache_move (attn_evict.h) moves an accepted path together.
 *
 * The mask is device memory like start and kv_len: its values may change between the replays of a captured graph.
 *
 * workspace_bytes at least attn_paged_tree_workspace_bytes(T, B, H_q, H_kv, D), else ATTN_ERR_WORKSPACE; calls that follow each other may
 * share one, also with attn_paged_fwd (the larger of the two sizes).
 *
 * All other arguments, results, limits, ownership and errors are those of attn_paged_fwd; ATTN_ERR_NULL, ATTN_ERR_SHAPE and ATTN_ERR_ALIGN stand
 * for the mask's arguments too.  Every row reads every key that its sequence has, so no row is cheaper for what its mask hides.  P enters the
 * second product in 16 bits as there: against 64 bits o is off by 0.0018 to 0.0023 of its norm (bf16; 0.00025 to 0.00029 fp16), of which
 * rounding o alone makes 0.0017 (0.00021).
 *
 * The host chooses the kernels by sizes alone, K and V as many as the table can hold: one tree of 15 at 1000 (32 heads over 8, D = 128) takes
 * some 12 us with a table of 1000 positions and 18 with one of 16384 or more, 16 trees of up to 77 at up to 2100 (8 over 2, D = 256, fp16) 30.8
 * and 32.7.
 */
int attn_paged_tree(const void *q, const long long *strides, void *o, float *lse,
                    const void *k_pages, const void *v_pages, const unsigned char *k_scale, const unsigned char *v_scale,
                    const int *page_table, const int *start, const int *kv_len, int kind,
                    const unsigned long long *mask, int mask_words, void *workspace, long long workspace_bytes, int max_q,
                    int T, int B, int H_q, int H_kv, int D, int n_pages, int page_size, int table_width,
                    float scale, void *stream);
int attn_paged_tree_f16(const void *q, const long long *strides, void *o, float *lse,
                        const void *k_pages, const void *v_pages, const unsigned char *k_scale, const unsigned char *v_scale,
                        const int *page_table, const int *start, const int *kv_len, int kind,
                        const unsigned long long *mask, int mask_words, void *workspace, long long workspace_bytes, int max_q,
                        int T, int B, int H_q, int H_kv, int D, int n_pages, int page_size, int table_width,
                        float scale, void *stream);

/* Bytes of workspace attn_paged_tree (either element type) needs; -1 on invalid arguments.  By rows (T * H_q / H_kv) at D = 128: 9 MB up to 16
 * of them, 72 up to 128, 144 beyond, and 16 bytes for every token. */
long long attn_paged_tree_workspace_bytes(int T, int B, int H_q, int H_kv, int D);

#ifdef __cplusplus
}
#endif
#endif /* MI355_ATTN_TREE_H */
