"""The launches of a vocabulary loss, as vocab_plan() of the built library chooses them (on the host, no GPU)."""
import ctypes as C

from paper_1804_10574_amd.ddg import DDG_BF16, DDG_F32, load_library

LARGE, MEDIUM, SHORT, SMALL, HALF, FEW, DEEP = range(7)
ROWS = (256, 128, 128, 64, 128, 128, 32)      # of a tile along the vocabulary or the width

# tokens, width, entries: fp32 products in planes over a vocabulary that one tile holds
ONE_TILE = [(40000, 1024, 256), (65536, 768, 193), (65536, 512, 200)]

# every kind of launch with gradients: the logits' tile and whether it holds the vocabulary ("z"), a gradient of its own launch or both in one, the tile and whether its sums
# have parts; a size whose rows are whole 16-byte pieces and one whose are not, as small as the estimate gives the kind
KINDS = [
    ("f32", ("dh", FEW, False), (132, 6457, 270), (158, 6200, 268)),
    ("f32", ("dh", FEW, True), (20, 855, 9238), (21, 472, 15766)),
    ("f32", ("dh", HALF, False), (25627, 68, 21), (24924, 72, 21)),
    ("f32", ("dh", HALF, True), (65, 7523, 1647), (35, 1144, 18064)),
    ("f32", ("dh", LARGE, False), (20632, 463, 503), (25701, 456, 458)),
    ("f32", ("dw", LARGE, True), (20632, 463, 503), (25701, 456, 458)),
    ("f32", ("dh", LARGE, True), (466, 422, 25023), (469, 408, 25189)),
    ("f32", ("dw", LARGE, False), (466, 422, 25023), (469, 408, 25189)),
    ("f32", ("dh", MEDIUM, False), (26573, 196, 21), (25459, 224, 20)),
    ("f32", ("dh", MEDIUM, True), (20055, 65, 1601), (21319, 72, 1329)),
    ("f32", ("dh", SMALL, False), (30655, 17, 21), (34653, 16, 21)),
    ("f32", ("dw", SMALL, True), (30655, 17, 21), (34653, 16, 21)),
    ("f32", ("dh", SMALL, True), (22, 17, 29640), (21, 16, 30069)),
    ("f32", ("dw", SMALL, False), (22, 17, 29640), (21, 16, 30069)),
    ("f32", ("dw", MEDIUM, False), (21, 66, 24579), (20, 72, 25933)),
    ("f32", ("dw", MEDIUM, True), (784, 2442, 476), (1042, 1880, 534)),
    ("f32", ("dw", SHORT, False), (21, 65, 66489), (23, 72, 69310)),
    ("f32", ("dw", SHORT, True), (30290, 71, 1414), (1886, 72, 26648)),
    ("f32", ("pair", LARGE, False, False), (2222, 2834, 2179), (2263, 2696, 2382)),
    ("f32", ("pair", LARGE, False, True), (26199, 211, 386), (28145, 208, 399)),
    ("f32", ("pair", LARGE, True, False), (420, 193, 28827), (387, 200, 28938)),
    ("f32", ("pair", LARGE, True, True), (8801, 193, 1224), (6023, 200, 1668)),
    ("f32", ("z", LARGE, False), (8801, 193, 1224), (6023, 200, 1668)),
    ("f32", ("pair", MEDIUM, False, False), (204, 7239, 129), (131, 7312, 205)),
    ("f32", ("pair", MEDIUM, False, True), (6243, 212, 65), (6452, 200, 70)),
    ("f32", ("pair", MEDIUM, True, False), (65, 212, 6377), (66, 208, 6567)),
    ("f32", ("pair", MEDIUM, True, True), (4292, 66, 465), (467, 72, 4474)),
    ("f32", ("pair", SMALL, False, False), (23, 17, 20), (22, 16, 22)),
    ("f32", ("z", SMALL, True), (23, 17, 20), (22, 16, 22)),
    ("f32", ("pair", SMALL, False, True), (304, 17, 21), (302, 16, 21)),
    ("f32", ("pair", SMALL, True, False), (23, 17, 298), (21, 16, 345)),
    ("f32", ("pair", SMALL, True, True), (99, 17, 296), (320, 16, 105)),
    ("f32", ("z", DEEP, False), (21, 65, 139), (21, 72, 131)),
    ("f32", ("z", DEEP, True), (20, 65, 22), (21, 72, 20)),
    ("f32", ("z", FEW, False), (21, 17, 52613), (24, 16, 53005)),
    ("f32", ("z", FEW, True), (20, 17, 69), (22, 16, 94)),
    ("f32", ("z", HALF, False), (34, 17, 49415), (73, 16, 24792)),
    ("f32", ("z", HALF, True), (8541, 17, 72), (8619, 16, 72)),
    ("f32", ("z", MEDIUM, False), (72, 17, 53647), (76, 16, 49613)),
    ("f32", ("z", MEDIUM, True), (34439, 17, 65), (34663, 16, 65)),
    ("f32", ("z", SMALL, False), (21, 18, 129), (20, 16, 129)),
    ("bf16", ("dh", FEW, False), (129, 6307, 1541), (138, 6272, 1592)),
    ("bf16", ("dh", FEW, True), (25, 2052, 5693), (20, 4144, 2861)),
    ("bf16", ("dh", HALF, False), (265, 6284, 2468), (381, 4624, 2371)),
    ("bf16", ("dh", HALF, True), (178, 65, 152644), (166, 72, 158255)),
    ("bf16", ("dh", LARGE, False), (2966, 5359, 134), (3213, 4784, 147)),
    ("bf16", ("dh", LARGE, True), (139, 1149, 42144), (132, 776, 63720)),
    ("bf16", ("dh", MEDIUM, False), (1945, 2756, 257), (1935, 2824, 257)),
    ("bf16", ("dh", MEDIUM, True), (67, 1993, 18136), (66, 840, 40811)),
    ("bf16", ("dh", SMALL, False), (22, 8081, 1456), (21, 7984, 1449)),
    ("bf16", ("dh", SMALL, True), (21, 17, 90689), (22, 16, 95099)),
    ("bf16", ("dw", SHORT, False), (21, 17, 90689), (22, 16, 95099)),
    ("bf16", ("dw", LARGE, False), (140, 5147, 3000), (135, 4968, 2991)),
    ("bf16", ("dw", LARGE, True), (38283, 161, 2245), (38233, 136, 2312)),
    ("bf16", ("dw", MEDIUM, False), (69, 65, 127020), (67, 72, 123039)),
    ("bf16", ("dw", MEDIUM, True), (30623, 387, 545), (30528, 392, 537)),
    ("bf16", ("dw", SHORT, True), (30689, 18, 11454), (12822, 544, 1059)),
    ("bf16", ("dw", SMALL, False), (21, 17, 114227), (22, 16, 127411)),
    ("bf16", ("dw", SMALL, True), (32173, 21, 1423), (32146, 24, 1418)),
    ("bf16", ("pair", LARGE, False, False), (385, 7725, 537), (400, 7456, 519)),
    ("bf16", ("pair", LARGE, False, True), (21539, 133, 451), (19540, 136, 526)),
    ("bf16", ("pair", LARGE, True, False), (459, 129, 20683), (464, 136, 21672)),
    ("bf16", ("pair", LARGE, True, True), (9833, 132, 1639), (10406, 136, 1224)),
    ("bf16", ("pair", MEDIUM, False, False), (204, 7239, 129), (131, 7312, 205)),
    ("bf16", ("pair", MEDIUM, False, True), (1105, 4097, 20), (3955, 1120, 21)),
    ("bf16", ("pair", MEDIUM, True, False), (20, 4346, 1050), (20, 1656, 2781)),
    ("bf16", ("pair", MEDIUM, True, True), (1325, 66, 4697), (5178, 72, 1193)),
    ("bf16", ("pair", SMALL, False, False), (23, 17, 20), (22, 16, 22)),
    ("bf16", ("z", SMALL, True), (23, 17, 20), (22, 16, 22)),
    ("bf16", ("pair", SMALL, False, True), (1122, 17, 20), (1143, 16, 24)),
    ("bf16", ("pair", SMALL, True, False), (21, 18, 1104), (23, 16, 1117)),
    ("bf16", ("pair", SMALL, True, True), (211, 17, 1089), (1140, 16, 223)),
    ("bf16", ("z", DEEP, False), (20, 825, 136), (20, 800, 139)),
    ("bf16", ("z", DEEP, True), (21, 801, 20), (20, 888, 21)),
    ("bf16", ("z", FEW, False), (21, 17, 52613), (24, 16, 53005)),
    ("bf16", ("z", FEW, True), (20, 17, 69), (22, 16, 94)),
    ("bf16", ("z", HALF, False), (34, 17, 49415), (73, 16, 24792)),
    ("bf16", ("z", HALF, True), (8541, 17, 72), (8619, 16, 72)),
    ("bf16", ("z", LARGE, False), (135, 65, 55722), (129, 72, 51200)),
    ("bf16", ("z", LARGE, True), (32818, 17, 131), (33772, 16, 140)),
    ("bf16", ("z", MEDIUM, False), (65, 17, 36634), (72, 16, 33635)),
    ("bf16", ("z", MEDIUM, True), (34439, 17, 65), (34663, 16, 65)),
    ("bf16", ("z", SMALL, False), (21, 18, 129), (20, 16, 129)),
]
# fp32 products in planes: both gradients in one launch, in launches of their own, in several panels, the tokens in parts; and a neighbour that takes none
PLANES = [((1021, 777, 10007), dict(pair=True, panels=1)), ((1200, 520, 9500), dict(pair=True, panels=1)), ((469, 408, 25189), dict(pair=False, panels=1)),
          ((900, 512, 160000), dict(pair=False, panels=2)), ((40000, 1024, 256), dict(pair=True, splits_dw=48, stats=2)), ((700, 1028, 9000), dict(planes=False))]

# the loss without gradients of many tokens
LOSS_ALONE = [("f32", (40000, 1024, 256), dict(planes=False, whole=False)), ("f32", (1500, 700, 15000), dict(planes=True, panels=1)),
              ("f32", (5000, 24, 1200001), dict(planes=False, panels=2)), ("f32", (8000, 264, 600001), dict(planes=True, panels=2)),
              ("bf16", (40000, 1024, 256), dict(whole=True)), ("bf16", (65536, 768, 193), dict(whole=True)), ("bf16", (5000, 24, 1200001), dict(panels=2)),
              ("bf16", (9000, 264, 200003), dict(cfg_z=LARGE, panels=1))]


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


def kinds(p):
    """The entries of KINDS that a plan is one of."""
    z = ("z", p.cfg_z, p.whole)
    return [z, ("pair", p.cfg_dh, p.splits > 1, p.splits_dw > 1)] if p.pair else [z, ("dh", p.cfg_dh, p.splits > 1), ("dw", p.cfg_dw, p.splits_dw > 1)]
