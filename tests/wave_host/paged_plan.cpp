// attn_paged_plan.h on the host: what the workgroups of a launch make of a batch's lengths.
#include "attn_paged_plan.h"

namespace {
attn::PagedParams p;
attn::Unit unit;
bool found;
int wg, bm, row, answer, position;

template <int BM>
void plan(int)
{
    attn::Unit u = {};
    attn::PlanSeq seq;
    const attn::Plan cut = attn::plan_call<BM>(p, seq);
    const bool f = attn::find_unit<BM>(p, cut, seq, wg, u);
    unit = u, found = f;
}

template <int BM>
void cut(int)
{
    attn::leave_cut<BM>(p, attn::WaveScope{p.c.B == 1});
}

template <int BM>
void note(int)
{
    attn::leave_note<BM, 64>(p, unit);
}
}  // namespace

extern "C" int plan_batch(const int *table, const int *start, const int *kv_len, int T, int B, int H_kv, int n_pages,
                          int page_log2, int width, int G, int BM, int rows_above, int rows_upto, int target, int min_range,
                          int n_slots, int causal, int rounds, int n_wg, int *units, int4 *notes, int2 *table_of_units)
{
    p = {};
    p.c.page_table = table, p.c.start = start, p.c.kv_len = kv_len;
    p.c.T = T, p.c.B = B, p.c.H_kv = H_kv, p.c.n_pages = n_pages, p.c.page_log2 = page_log2, p.c.table_width = width;
    p.G = G, p.H_q = G * H_kv;
    p.rows_above = rows_above, p.rows_upto = rows_upto, p.target = target, p.min_range = min_range, p.slots = n_slots, p.causal = causal;
    p.rounds = rounds, p.overhead = 2, p.merging = 1, p.most_units = n_wg, p.halve = causal;
    p.merge = notes;
    int log_g = 0;
    while ((1LL << log_g) < G)
        ++log_g;
    p.g_mul = G == 1 ? 0 : (uint32_t)(((1ULL << (31 + log_g)) + G - 1) / G);
    p.g_shift = G == 1 ? 0 : log_g - 1;
    if (table_of_units) {
        p.cut = table_of_units;
        if (!wave_host::run(BM == 16 ? cut<16> : BM == 32 ? cut<32> : BM == 64 ? cut<64> : BM == 128 ? cut<128> : cut<256>))
            return -1;
    }
    int n = 0;
    for (wg = 0; wg < n_wg; ++wg) {
        if (!wave_host::run(BM == 16 ? plan<16> : BM == 32 ? plan<32> : BM == 64 ? plan<64> : BM == 128 ? plan<128> : plan<256>))
            return -1;
        if (!found)
            continue;
        const attn::Unit &u = unit;
        const int out[14] = {u.b, u.h, u.tile, u.range, u.n_ranges, u.n_tiles, u.row0, u.n_rows, u.n, u.kv, u.key0, u.key1,
                             u.slot0, u.slot};
        memcpy(units + 14 * n++, out, sizeof out);
        if (!wave_host::run(BM == 16 ? note<16> : BM == 32 ? note<32> : BM == 64 ? note<64> : BM == 128 ? note<128> : note<256>))
            return -1;
    }
    return n;
}

// sequence of row t (-1: none), and the page of a position of sequence `row` (page_of)
extern "C" int sequence_of(const int *start, int T, int B, int t)
{
    p = {};
    p.c.start = start, p.c.T = T, p.c.B = B;
    row = t;
    if (!wave_host::run([](int) { answer = p.c.sequence_of(row); }))
        return -2;
    return answer;
}

extern "C" int page_of(const int *table, const int *kv_len, int b, int n_pages, int page_log2, int width, int pos, int *length)
{
    p = {};
    p.c.page_table = table, p.c.kv_len = kv_len, p.c.n_pages = n_pages, p.c.page_log2 = page_log2, p.c.table_width = width;
    *length = p.c.length_of(b);
    return pos < *length && pos >= 0 ? p.c.page_of(b, pos) : -2;
}

extern "C" void layer_place(int w, int H, int n, int *h, int *tile) { attn::place_in_layer(w, H, n, *h, *tile); }

// row / G and a / b as the kernels take them
extern "C" int row_over(int row, int G)
{
    int log_g = 0;
    while ((1LL << log_g) < G)
        ++log_g;
    p.G = G;
    p.g_mul = G == 1 ? 0 : (uint32_t)(((1ULL << (31 + log_g)) + G - 1) / G);
    p.g_shift = G == 1 ? 0 : log_g - 1;
    return p.token_of(row);
}
extern "C" int over(int a, int b) { return attn::quotient(a, b); }
