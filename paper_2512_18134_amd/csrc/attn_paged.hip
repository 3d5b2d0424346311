// attn_paged.hip -- entry points of the attention over the paged cache (include/attn_cache.h).
#include "attn_paged_launch.h"

extern "C" long long attn_paged_fwd_workspace_bytes(int T, int B, int H_q, int H_kv, int D)
{
    if (T < 1 || B < 1 || H_q < 1 || H_kv < 1 || H_q % H_kv || (D != 64 && D != 128 && D != 256) ||
        (long long)T * H_q > 0x3fffffffLL || B > attn::kMostSequences)
        return -1;
    return attn::workspace_of(T, B, H_q / H_kv, D).bytes;
}

extern "C" int attn_paged_fwd(const void *q, const long long *strides, void *o, float *lse, const void *k_pages,
                              const void *v_pages, const unsigned char *k_scale, const unsigned char *v_scale,
                              const int *page_table, const int *start, const int *kv_len, int kind, void *workspace,
                              long long workspace_bytes, int max_q, int T, int B, int H_q, int H_kv, int D, int n_pages,
                              int page_size, int table_width, int causal, float scale, void *stream)
{
    return attn::paged_call<attn::PagedBF16, false>(q, strides, o, lse, k_pages, v_pages, k_scale, v_scale, page_table, start, kv_len, kind,
                                      workspace, workspace_bytes, max_q, T, B, H_q, H_kv, D, n_pages, page_size, table_width,
                                      causal, nullptr, 0, scale, stream);
}

extern "C" int attn_paged_fwd_f16(const void *q, const long long *strides, void *o, float *lse, const void *k_pages,
                                  const void *v_pages, const unsigned char *k_scale, const unsigned char *v_scale,
                                  const int *page_table, const int *start, const int *kv_len, int kind, void *workspace,
                                  long long workspace_bytes, int max_q, int T, int B, int H_q, int H_kv, int D, int n_pages,
                                  int page_size, int table_width, int causal, float scale, void *stream)
{
    return attn::paged_call<attn::PagedF16, false>(q, strides, o, lse, k_pages, v_pages, k_scale, v_scale, page_table, start, kv_len, kind,
                                     workspace, workspace_bytes, max_q, T, B, H_q, H_kv, D, n_pages, page_size, table_width,
                                     causal, nullptr, 0, scale, stream);
}
