#!/usr/bin/env python3
"""Emit the hand-scheduled main loop of the attention over a paged cache (attn_paged_asm.h).

The schedule is that of gen_attn_loop.py: P(j-1) V(j-1) and K(j+1) Q^T on the matrix pipe, the softmax of S(j) beside
them, direct loads of K(j+4) and V(j+2) into rings of four stages, one barrier per tile.  What differs is where a tile
lies and which of its keys exist:

  * A wave brings eight rows of every tile.  They lie in one page (pages hold a multiple of 16 positions), so that one
    scalar address serves the wave's loads of a tensor.  It comes from registers that hold, one tile per lane, the
    addresses of the wave's rows of 64 tiles (windows of K and of V, low and high words): two v_readlane per tensor in
    place of the pointer's addition.  Tile t sits in lane t % 64; every 56 iterations an out-of-line section reads the
    page numbers of the 64 tiles from the current one on and fills the windows anew.
  * A page number outside the pool gives the address of eight rows of zeros.  If the walk has any (the
    kernel looks beforehand), every tile takes the mask pre-pass, which then reads the page numbers of the tile's
    16-key parts and masks those without a page.
  * Rows behind the sequence's last position repeat it, found in the eight rows that hold it.
  * A walk may start anywhere in the keys, so a row may see none of its first tiles: the references start at the lowest
    finite number (LOW in gen_attn_loop.py).

usage: gen_attn_paged_loop.py <config> <out.inc> [bf16|f16]
"""
import os
import re
import sys

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import gen_attn_loop  # noqa: E402

CONFIGS = {name: {k: v for k, v in dict(gen_attn_loop.CONFIGS[of], LOW=True).items() if k != "AT"}
           for name, of in (("paged_d64", "d64"), ("paged_d128", "d128a"), ("paged_d256", "d256a"))}

WINDOW = 64      # tiles of a window, one per lane
REFRESH = 56     # iterations between two fillings: iteration j asks for tile j + 5 at most


class PagedGen(gen_attn_loop.Gen):
    configs = CONFIGS
    # (register, name in the kernel) of the scalar operands besides those of the dense loop; pairs are 64-bit
    scalars = [(66, 2, "page_tab"), (68, 2, "zero_rows"), (70, 1, "pos_base"), (71, 1, "end8"), (72, 1, "page_log2"),
               (73, 1, "page_mask"), (74, 1, "page_bytes"), (75, 1, "n_pages"), (76, 1, "missing"), (77, 1, "kv_last"),
               (78, 1, "key0")]

    def __init__(self, name, dtype="bf16"):
        gen_attn_loop.Gen.__init__(self, name, dtype)
        assert self.s_nw < 66 and self.TB // (self.NW * self.ROWB) == 8, "a wave brings eight rows of a tile"
        self.s_tab, self.s_zero, self.s_posbase, self.s_end8, self.s_plog2, self.s_pmask, self.s_pbytes, self.s_npages, \
            self.s_missing, self.s_kvlast, self.s_key0 = (r for r, _, _ in self.scalars)
        self.s_refresh, self.s_spec0, self.s_x = 79, 80, 81
        self.log_bn = {32: 5, 64: 6}[self.BN]
        self.log_row = {128: 7, 256: 8, 512: 9}[self.ROWB]

    def take_temporaries(self, take):
        gen_attn_loop.Gen.take_temporaries(self, take)
        self.WIN = take(4, operand=True)      # K low, K high, V low, V high
        self.RT = take(4)

    # ------------------------------------------------------------ where a tile lies
    def pointer_ops(self, which, ahead):
        """The scalar pointer at this wave's rows of tile j + ahead."""
        ptr, win = (self.s_kptr, self.WIN) if which == "k" else (self.s_vptr, self.WIN + 2)
        return ["s_add_i32 s%d, s%d, %d" % (self.s_t2, self.s_j, ahead),
                "s_and_b32 s%d, s%d, %d" % (self.s_t2, self.s_t2, WINDOW - 1),
                "v_readlane_b32 s%d, v%d, s%d" % (ptr, win, self.s_t2),
                "v_readlane_b32 s%d, v%d, s%d" % (ptr + 1, win + 1, self.s_t2)]

    def bump_ops(self):
        return self.pointer_ops("k", 5) + self.pointer_ops("v", 3) + ["s_add_i32 s%d, s%d, 1" % (self.s_j, self.s_j)]

    def start_pointers(self):
        for ins in self.pointer_ops("k", 4) + self.pointer_ops("v", 2):
            self.e(ins)
        # (a scalar that the vector unit wrote needs five wait states before a load uses it; the loop's are an iteration old)
        self.e("s_nop 4")
        self.e("s_mov_b32 s%d, s%d" % (self.s_spec0, self.s_special))
        self.e("s_mov_b32 s%d, %d" % (self.s_refresh, REFRESH))
        self.e("s_min_i32 s%d, s%d, s%d" % (self.s_special, self.s_special, self.s_refresh))

    def dma_slow(self, which, stage, ahead):
        """Tile j + ahead with rows behind the last position: the pointer is at the eight rows that hold it."""
        tab = self.s_lk if which == "k" else self.s_lv
        self.clamped_loads(which, ahead, lambda i: ("s_add_u32 m0, s%d, %d" % (tab + stage, 1024 * i)) if i
                           else "s_mov_b32 m0, s%d" % (tab + stage))

    def clamped_loads(self, which, ahead, m0):
        ptr = self.s_kptr if which == "k" else self.s_vptr
        t2 = self.s_t2
        # last row that exists of the eight
        self.e("s_add_i32 s%d, s%d, %d" % (t2, self.s_j, ahead))
        self.e("s_lshl_b32 s%d, s%d, %d" % (t2, t2, self.log_bn))
        self.e("s_add_i32 s%d, s%d, s%d" % (t2, t2, self.s_posbase))
        self.e("s_min_i32 s%d, s%d, s%d" % (t2, t2, self.s_end8))
        self.e("s_sub_i32 s%d, s%d, s%d" % (t2, self.s_kvlast, t2))
        self.e("s_min_i32 s%d, s%d, 7" % (t2, t2))
        for i in range(self.NLD):
            t = self.DT + (0 if which == "k" else self.NLD) + i
            self.e("v_min_i32 v%d, s%d, v%d" % (t, t2, self.DROW + i))
            self.e("v_lshlrev_b32 v%d, %d, v%d" % (t, self.log_row, t))
            self.e(m0(i))
            self.e("v_add_u32 v%d, v%d, v%d" % (t, t, self.DCH + i))
            self.e("s_nop 0")
            self.e("global_load_lds_dwordx4 v%d, %s" % (t, self.sr(ptr, 2)))

    def standby_loads(self):
        self.special_entry("SB")
        tb = {8192: 13, 16384: 14}[self.TB]
        for which, ahead in (("k", 4), ("v", 2)):
            lds = self.s_ldsk if which == "k" else self.s_ldsv
            for ins in self.pointer_ops(which, ahead):
                self.e(ins)
            self.e("s_add_i32 s%d, s%d, %d" % (self.s_t3, self.s_j, ahead))
            self.e("s_and_b32 s%d, s%d, 3" % (self.s_t3, self.s_t3 if which == "v" else self.s_j))
            self.e("s_lshl_b32 s%d, s%d, %d" % (self.s_t3, self.s_t3, tb))
            self.e("s_add_u32 s%d, s%d, s%d" % (self.s_t3, self.s_t3, lds))
            self.clamped_loads(which, ahead, lambda i: ("s_add_u32 m0, s%d, %d" % (self.s_t3, 1024 * i)) if i
                               else "s_mov_b32 m0, s%d" % self.s_t3)

    def special_entry(self, tag):
        """Every REFRESH iterations: the windows hold the tiles from the current one on."""
        e, r, L = self.e, self.RT, self.lab
        e("s_cmp_lt_i32 s%d, s%d" % (self.s_j, self.s_refresh))
        e("s_cbranch_scc1 %s" % L("FRESH%s_" % tag))
        e("v_mbcnt_lo_u32_b32 v%d, -1, 0" % r)
        e("v_mbcnt_hi_u32_b32 v%d, -1, v%d" % (r, r))
        e("v_subrev_u32 v%d, s%d, v%d" % (r, self.s_j, r))           # lane - j
        e("v_and_b32 v%d, %d, v%d" % (r, WINDOW - 1, r))
        e("v_add_u32 v%d, s%d, v%d" % (r, self.s_j, r))              # the tile from j on that this lane holds
        e("v_lshlrev_b32 v%d, %d, v%d" % (r, self.log_bn, r))
        e("v_add_u32 v%d, s%d, v%d" % (r, self.s_posbase, r))
        e("v_min_i32 v%d, s%d, v%d" % (r, self.s_end8, r))           # first position of the eight rows
        e("v_lshrrev_b32 v%d, s%d, v%d" % (r + 1, self.s_plog2, r))
        e("v_lshlrev_b32 v%d, 2, v%d" % (r + 1, r + 1))
        e("global_load_dword v%d, v%d, %s" % (r + 1, r + 1, self.sr(self.s_tab, 2)))
        e("v_and_b32 v%d, s%d, v%d" % (r, self.s_pmask, r))
        e("v_lshlrev_b32 v%d, %d, v%d" % (r, self.log_row, r))       # place in the page, bytes
        e("s_waitcnt vmcnt(0)")
        e("v_mul_lo_u32 v%d, v%d, s%d" % (r + 2, r + 1, self.s_pbytes))
        e("v_mul_hi_u32 v%d, v%d, s%d" % (r + 3, r + 1, self.s_pbytes))
        e("v_add_co_u32 v%d, vcc, v%d, v%d" % (r + 2, r + 2, r))
        e("v_addc_co_u32 v%d, vcc, 0, v%d, vcc" % (r + 3, r + 3))
        for base, lo in ((self.s_kbase, self.WIN), (self.s_vbase, self.WIN + 2)):
            e("v_mov_b32 v%d, s%d" % (r, base + 1))
            e("v_add_co_u32 v%d, vcc, s%d, v%d" % (lo, base, r + 2))
            e("v_addc_co_u32 v%d, vcc, v%d, v%d, vcc" % (lo + 1, r, r + 3))
        e("v_cmp_gt_u32 vcc, s%d, v%d" % (self.s_npages, r + 1))
        for word in (0, 1):
            e("v_mov_b32 v%d, s%d" % (r, self.s_zero + word))
            for lo in (self.WIN, self.WIN + 2):
                e("v_cndmask_b32 v%d, v%d, v%d, vcc" % (lo + word, r, lo + word))
        e("s_add_i32 s%d, s%d, %d" % (self.s_refresh, self.s_refresh, REFRESH))
        e("s_min_i32 s%d, s%d, s%d" % (self.s_special, self.s_spec0, self.s_refresh))
        e("s_nop 1")
        e("%s:" % L("FRESH%s_" % tag))

    def mask_more(self, tag, S_cur):
        """Keys without a page, 16 at a time (only a walk that has some comes here with s_missing set)."""
        e, L = self.e, self.lab
        e("s_cmp_eq_u32 s%d, 0" % self.s_missing)
        e("s_cbranch_scc1 %s" % L("WHOLE%s_" % tag))
        for h in range(self.BN // 16):
            e("s_lshl_b32 s%d, s%d, %d" % (self.s_t2, self.s_j, self.log_bn))
            e("s_add_i32 s%d, s%d, s%d" % (self.s_t2, self.s_t2, self.s_key0))
            if h:
                e("s_add_i32 s%d, s%d, %d" % (self.s_t2, self.s_t2, 16 * h))
            e("s_min_i32 s%d, s%d, s%d" % (self.s_t2, self.s_t2, self.s_kvlast))
            e("s_lshr_b32 s%d, s%d, s%d" % (self.s_t2, self.s_t2, self.s_plog2))
            e("s_lshl_b32 s%d, s%d, 2" % (self.s_t2, self.s_t2))
            e("s_load_dword s%d, %s, s%d" % (self.s_x, self.sr(self.s_tab, 2), self.s_t2))
            e("s_waitcnt lgkmcnt(0)")
            e("s_cmp_lt_u32 s%d, s%d" % (self.s_x, self.s_npages))
            e("s_cbranch_scc1 %s" % L("PAGE%s_%d_" % (tag, h)))
            for qb in range(self.QB):
                for r in range(8):
                    e("v_mov_b32 v%d, v%d" % (self.s_reg(S_cur, qb, h // 2, 0, 8 * (h % 2) + r), self.NEGINF))
            e("%s:" % L("PAGE%s_%d_" % (tag, h)))
        e("%s:" % L("WHOLE%s_" % tag))

    # ----------------------------------------------------------- C++ wrapper
    def emit_inc(self):
        text = gen_attn_loop.Gen.emit_inc(self)
        text = text.replace("gen_attn_loop.py", "gen_attn_paged_loop.py").replace("attn_fwd_asm_kernel", "attn_paged_asm_kernel")
        window = '"+{%s}"(page_win)' % self.vr(self.WIN, 4)
        inputs = ", ".join('"{%s}"(%s)' % (self.sr(r, n) if n > 1 else "s%d" % r, name) for r, n, name in self.scalars)
        for old, new in (("(l_run_v)", "(l_run_v), " + window), ("(lds_v_wave)", "(lds_v_wave), " + inputs)):
            assert text.count(old) == 1
            text = text.replace(old, new)
        for i in range(4):
            text, n = re.subn(r'"v%d"(, )?' % (self.WIN + i), "", text)
            assert n == 1
        assert text.endswith('"s%d");\n' % self.s_last)
        return text[:-3] + ", " + ", ".join('"s%d"' % r for r in (self.s_refresh, self.s_spec0, self.s_x)) + ");\n"


def main(argv):
    text = PagedGen(argv[0], argv[2] if len(argv) > 2 else "bf16").emit_inc()
    with open(argv[1], "w") as f:
        f.write(text)


if __name__ == "__main__":
    main(sys.argv[1:])
