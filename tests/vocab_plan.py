"""The launches of a vocabulary loss, as vocab_plan() of the built library chooses them (on the host, no GPU)."""
import ctypes as C

from paper_1804_10574_amd.ddg import DDG_BF16, DDG_F32, load_library

LARGE, MEDIUM, SHORT, SMALL, HALF, FEW, DEEP = range(7)
ROWS = (256, 128, 128, 64, 128, 128, 32)      # of a tile along the vocabulary or the width

# tokens, width, entries: fp32 products in planes over a vocabulary that one tile holds
ONE_TILE = [(40000, 1024, 256), (65536, 768, 193), (65536, 512, 200)]


class Plan(C.Structure):       # VocabPlan
    _fields_ = ([(n, C.c_int) for n in ("tokens", "dim", "vocab", "dtype")] + [(n, C.c_bool) for n in ("grads", "dw_f32", "pack_h", "pack_w", "planes")]
                + [(n, C.c_int) for n in ("dim_p", "panel", "panels")] + [("ld_p", C.c_long)]
                + [(n, C.c_int) for n in ("cfg_z", "cfg_dh", "cfg_dw", "stat_cols", "stats", "splits", "splits_dw")]
                + [(n, C.c_bool) for n in ("whole", "pair", "acc")]
                + [(n, C.c_size_t) for n in ("o_scalar", "o_row", "o_zt", "o_stat", "o_p", "o_planes", "o_part", "o_part_dw", "o_acc", "o_h", "o_w", "bytes")])


def vocab_plan(dtype, tokens, dim, vocab, grads=True, dw_f32=False, pack_h=False, pack_w=False):
    p = Plan(tokens=tokens, dim=dim, vocab=vocab, dtype=DDG_BF16 if dtype == "bf16" else DDG_F32, grads=grads, dw_f32=dw_f32, pack_h=pack_h, pack_w=pack_w)
    load_library()._ZN3ddg10vocab_planEPNS_9VocabPlanE(C.byref(p))
    return p
