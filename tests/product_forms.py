"""Sizes at which the layer operators' products run in each of their forms, and
the rules of the library that choose them (no GPU needed)."""
import ctypes

import paper_2609_14706_amd as ff

# tokens, n, m by type: every tile, alone and with k split, with ragged ends of all three
LINEAR = {
    "bf16": [(75, 1545, 64), (131, 300, 257), (1632, 138, 3682), (8342, 6447, 139), (1630, 1202, 1184), (4385, 5603, 130),
             (1615, 134, 2541), (131, 1667, 25018), (2567, 68, 3164), (4436, 66, 2775)],
    "int8": [(70, 3318, 64), (131, 300, 257), (3344, 259, 1783), (71, 12110, 16475), (1167, 2342, 1674), (2729, 15147, 135),
             (3601, 263, 1077), (129, 3161, 25689), (4109, 142, 1977), (2766, 139, 4551)],
}
# tokens, m at which lengths of k from one 128-byte piece to nine run in the larger tiles
LENGTHS = [(11021, 387), (10944, 264), (10883, 653), (11153, 1027)]
# few tokens: every number of token and output tiles and of waves
FEW = {
    "bf16": [(9, 640, 300), (9, 2100, 301), (13, 4100, 299), (24, 100, 310), (27, 1990, 77), (32, 4100, 50), (30, 72, 8200),
             (21, 2002, 8420), (55, 64, 33), (39, 2001, 70), (38, 4111, 90), (64, 136, 8198)],
    "int8": [(9, 640, 300), (9, 4200, 301), (13, 8200, 299), (24, 100, 310), (23, 4001, 77), (28, 8100, 50), (30, 72, 8200),
             (32, 3974, 8325), (55, 64, 33), (55, 4001, 70), (35, 8111, 90), (64, 136, 8198)],
}
# batch, m, n by type: updates of one workgroup, every form of the three products of a
# step, A = X X^T also with k split
ORTHO = {
    "f32": [(2, 90, 61), (8, 198, 6351), (8, 129, 5573), (8, 1174, 519), (8, 65, 4190), (8, 65, 6151), (8, 385, 519), (1, 17, 515),
            (8, 1421, 1427), (3, 1605, 5330), (8, 1284, 1288), (3, 1092, 4306), (8, 969, 971), (8, 652, 642), (8, 4579, 193),
            (1, 16, 833)],
    "bf16": [(2, 90, 61), (3, 17, 515), (8, 198, 6351), (8, 129, 5573), (2, 1730, 1540), (8, 2727, 129), (8, 194, 3105), (1, 1221, 1537),
             (1, 1027, 17), (8, 1421, 1427), (1, 2822, 5961), (8, 1284, 1288), (8, 969, 971), (8, 652, 642), (1, 16, 2625)],
}


class _Linear(ctypes.Structure):
    _fields_ = [("skinny", ctypes.c_bool)] + [(k, ctypes.c_int) for k in ("ti", "tj", "slots", "splits")]


class _Few(ctypes.Structure):
    _fields_ = [(k, ctypes.c_int) for k in ("nt", "rw", "waves")]


class _Ortho(ctypes.Structure):
    _fields_ = [(k, ctypes.c_int) for k in ("small", "gram", "gram_splits", "square", "apply")]


def _rule(name, result, *args):
    fn = ff.load_library()[name]
    fn.argtypes, fn.restype = args, result
    return fn


def linear_form(tokens, n, m, elem_bytes):
    """(ti, tj, slots, splits), or ("few", tiles of tokens, of outputs, waves)."""
    sizes = (tokens, n, m, elem_bytes)
    p = _rule("_ZN2ff11linear_planEllli", _Linear, *[ctypes.c_int64] * 3, ctypes.c_int)(*sizes)
    if not p.skinny:
        return p.ti, p.tj, p.slots, p.splits
    k = _rule("_ZN2ff11skinny_planEllli", _Few, *[ctypes.c_int64] * 3, ctypes.c_int)(*sizes)
    return "few", k.nt, k.rw, k.waves


def ortho_form(batch, m, n, bf16):
    """(parts in one workgroup or 0, forms of A with its splits, of A A, of the product with X)."""
    p = _rule("_ZN2ff10ortho_planElllb", _Ortho, *[ctypes.c_int64] * 3, ctypes.c_bool)(batch, m, n, bf16)
    return p.small, p.gram, p.gram_splits, p.square, p.apply
