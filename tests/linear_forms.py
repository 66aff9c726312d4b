"""The forms of the experts' products (rows of a tile, contractions shared by groups of waves or not) and, for each of them, a
product that takes it: widths that are no whole tiles and no whole k-tiles, several tiles, experts of unlike size."""
import ctypes

from operator_refs import DT
from paper_2406_00023_amd import binding as B

ACT = {"none": B.ACT_NONE, "silu": B.ACT_SILU, "gelu": B.ACT_GELU, "swiglu": B.ACT_SWIGLU}
FORWARD, INPUT, WEIGHT, JOINT = range(4)
TILES = ("16", "32", "64", "128", "256")

# {(product, type, activation): {form: (rows, experts, K, N)}}; "+": shared contractions.  With SwiGLU dx has a contraction in two halves
CASES = {
    (FORWARD, "bf16", "none"): {"16+": (5, 2, 904, 136), "32": (33, 3, 520, 264), "32+": (11, 2, 728, 136), "64": (608, 2, 208, 136),
                                "64+": (552, 2, 464, 136), "128": (10969, 4, 200, 144), "256": (952, 7, 200, 5080)},
    (FORWARD, "bf16", "swiglu"): {"16+": (5, 2, 792, 136), "32": (33, 3, 520, 264), "32+": (1675, 7, 1248, 296), "64": (551, 2, 224, 136),
                                  "64+": (4, 2, 648, 136), "128": (6408, 8, 200, 136), "256": (1694, 12, 200, 1488)},
    (FORWARD, "f32", "none"): {"16+": (3, 2, 200, 136), "32": (492, 2, 208, 136), "32+": (471, 2, 336, 152), "64": (741, 2, 208, 136),
                               "64+": (650, 2, 376, 208)},
    (FORWARD, "f32", "swiglu"): {"16+": (5, 2, 200, 136), "32": (7, 4, 200, 2712), "32+": (33, 12, 360, 720), "64": (483, 2, 208, 144),
                                 "64+": (937, 4, 360, 136)},
    (INPUT, "bf16", "none"): {"16+": (267, 2, 216, 792), "32": (262, 2, 200, 544), "32+": (406, 2, 2528, 1256), "64": (519, 2, 272, 544),
                              "64+": (293, 2, 200, 712), "128": (6491, 2, 264, 544), "256": (806, 6, 5728, 504)},
    (INPUT, "bf16", "swiglu"): {"16+": (270, 2, 216, 544), "32": (1187, 6, 744, 504), "32+": (531, 4, 1744, 624), "64": (4254, 6, 200, 552),
                                "64+": (1097, 5, 216, 504), "128": (783, 6, 2200, 504), "256": (790, 6, 5728, 504)},
    (INPUT, "f32", "none"): {"16+": (309, 2, 200, 536), "32": (543, 4, 1960, 504), "32+": (970, 5, 784, 552), "64": (1084, 6, 208, 528),
                             "64+": (1110, 4, 200, 504)},
    (INPUT, "f32", "swiglu"): {"16+": (295, 2, 208, 528), "32": (398, 3, 2648, 528), "32+": (796, 6, 936, 560), "64": (1333, 5, 736, 520),
                               "64+": (2276, 6, 200, 520)},
    (WEIGHT, "bf16", "none"): {"64": (294, 2, 200, 136), "64+": (909, 2, 200, 136), "128": (799, 6, 1872, 144), "256": (821, 6, 5856, 136)},
    (WEIGHT, "bf16", "swiglu"): {"64": (268, 2, 208, 144), "64+": (998, 2, 208, 144), "128": (790, 6, 928, 144), "256": (529, 4, 4120, 136)},
    (WEIGHT, "f32", "none"): {"64": (265, 2, 216, 144), "64+": (743, 2, 200, 160)},
    (WEIGHT, "f32", "swiglu"): {"64": (264, 2, 224, 136), "64+": (757, 2, 216, 136)},
    # dx and dw in one launch
    (JOINT, "bf16", "none"): {"apart": (295, 2, 200, 2032), "64": (294, 2, 200, 136), "64+": (285, 2, 200, 488)},
    (JOINT, "bf16", "swiglu"): {"apart": (282, 2, 208, 944), "64": (268, 2, 208, 144), "64+": (262, 2, 232, 200)},
    (JOINT, "f32", "none"): {"apart": (263, 2, 208, 656), "64": (265, 2, 216, 144), "64+": (304, 2, 200, 240)},
    (JOINT, "f32", "swiglu"): {"apart": (268, 2, 232, 344), "64": (577, 4, 392, 136), "64+": (264, 2, 224, 136)},
}

# more tiles of 256 rows than a chip of 256 CUs has places: workgroups go from tile to tile, and a last round goes whole, in halves or in quarters
WALKS = [(FORWARD, "bf16", "none", "256", 3303, 3, 200, 6152), (FORWARD, "bf16", "swiglu", "256", 3303, 3, 200, 2568),
         (INPUT, "bf16", "none", "256", 2603, 3, 5896, 200), (INPUT, "bf16", "swiglu", "256", 2603, 3, 6664, 136),
         (WEIGHT, "bf16", "none", "256", 700, 4, 2056, 2056), (WEIGHT, "bf16", "swiglu", "256", 700, 4, 2056, 2056)]


def listed(*products):
    cases = [(p, dtype, act, form, *shape) for (p, dtype, act), forms in CASES.items() for form, shape in forms.items()]
    return [c for c in cases + WALKS if c[0] in products]


def plan(product, dtype, act, rows, E, K, N):
    """The form that the library takes.  Host only, launches nothing."""
    fn = B.load_library().etr_linear_plan
    fn.restype, fn.argtypes = ctypes.c_int, [ctypes.POINTER(B.EtrLinearConfig), ctypes.c_int]
    n = fn(ctypes.byref(B.make_linear_config(rows, K, N, E, DT[dtype], act=ACT[act])), product)
    return ("apart", "64", "64+")[n] if product == JOINT else TILES[n & 7] + "+" * (n >> 3)


def counts(rows, E):
    """Rows of each expert, more for the later ones, none for the second of three or more; and rows that belong to nobody."""
    spare = 3 if rows > 40 else 1 if rows > 4 else 0
    used = rows - spare
    ends = [used * (e + 1) ** 2 // E ** 2 for e in range(E)]
    n = [b - a for a, b in zip([0] + ends, ends)]
    if E > 2:
        n[-1], n[1] = n[-1] + n[1], 0
    return tuple(n), spare
