// attn_tree.hip -- entry points of the attention of a tree of drafted tokens over the paged cache (include/attn_tree.h).
//
// The kernels are those of the attention over the paged cache with TREE set: a row sees every key in front of its sequence's new
// tokens, and of those what its mask says.  Only the steps that hold new tokens look at the mask.
//
// 32 sequences of up to 8191 positions and trees of up to 24 drafts, 32 heads over 8, D = 128: 458 MB of K and V in 104 us, 95 of them the
// kernel's (4.8 TB/s).  4 of 32768 in e4m3, 64 drafts, 64 heads over 8: 275 GFLOP in 304 to 313 us.  One tree of 15 at 1000: 11.3 us.
#include "attn_paged_launch.h"
#include "attn_tree.h"

extern "C" long long attn_paged_tree_workspace_bytes(int T, int B, int H_q, int H_kv, int D)
{
    if (T < 1 || B < 1 || H_q < 1 || H_kv < 1 || H_q % H_kv || (D != 64 && D != 128 && D != 256) ||
        (long long)T * H_q > 0x3fffffffLL || B > attn::kMostSequences)
        return -1;
    return attn::tree_workspace_of(T, B, H_q / H_kv, D).bytes;
}

#define ATTN_TREE_ENTRY(name, E)                                                                                                \
    extern "C" int name(const void *q, const long long *strides, void *o, float *lse, const void *k_pages, const void *v_pages, \
                        const unsigned char *k_scale, const unsigned char *v_scale, const int *page_table, const int *start,    \
                        const int *kv_len, int kind, const unsigned long long *mask, int mask_words, void *workspace,           \
                        long long workspace_bytes, int max_q, int T, int B, int H_q, int H_kv, int D, int n_pages,              \
                        int page_size, int table_width, float scale, void *stream)                                              \
    {                                                                                                                           \
        return attn::paged_call<E, true>(q, strides, o, lse, k_pages, v_pages, k_scale, v_scale, page_table, start, kv_len,     \
                                         kind, workspace, workspace_bytes, max_q, T, B, H_q, H_kv, D, n_pages, page_size,       \
                                         table_width, 0, mask, mask_words, scale, stream);                                      \
    }

ATTN_TREE_ENTRY(attn_paged_tree, attn::PagedBF16)
ATTN_TREE_ENTRY(attn_paged_tree_f16, attn::PagedF16)
