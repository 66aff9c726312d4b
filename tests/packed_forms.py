"""The forms of the products of packed operands and, for each of them, a product that takes it: widths that are no whole blocks, several tiles, experts of
unlike size.  Both types of results take the same forms."""
import ctypes

from linear_forms import ACT, counts                           # noqa: F401
from operator_refs import DT
from paper_2406_00023_amd import binding as B

FORWARD, PACKING, WEIGHT = range(3)
FORMS = ("rows16", "rows32", "rows128", "32", "64", "128", "256")

# {(product, activation): {form: (rows, experts, K, N)}}
CASES = {
    (FORWARD, "none"): {"rows16": (3, 2, 184, 152), "rows32": (12, 8, 688, 4488), "32": (40, 2, 136, 928), "64": (7, 8, 152, 4960), "128": (1173, 3, 152, 5184),
                        "256": (6259, 8, 168, 1504)},
    (FORWARD, "swiglu"): {"rows16": (3, 2, 152, 152), "rows32": (26, 12, 200, 5272), "32": (324, 3, 144, 1016), "64": (20, 6, 296, 4896), "256": (1515, 8, 152, 1160)},
    (PACKING, "none"): {"rows128": (10, 6, 800, 5200), "32": (20, 2, 144, 136), "64": (7, 8, 136, 5208), "128": (1045, 12, 152, 4424), "256": (2079, 2, 136, 4568)},
    (PACKING, "swiglu"): {"rows128": (17, 12, 440, 2664), "32": (2, 2, 168, 144), "64": (7, 8, 328, 4312), "256": (5445, 12, 144, 280)},
    (WEIGHT, "none"): {"32": (8, 2, 152, 136), "64": (3, 6, 144, 2128), "128": (1, 12, 136, 2360), "256": (4, 8, 160, 4784)},
    (WEIGHT, "swiglu"): {"32": (10, 2, 168, 136), "64": (6, 8, 144, 776), "128": (2, 6, 136, 2200), "256": (3, 8, 136, 2520)},
}

# more tiles of 256 rows than a chip of 256 CUs has places: workgroups go from tile to tile, and a last round goes whole, in halves or in quarters
WALKS = [(FORWARD, "none", "256", 3303, 3, 392, 6152), (FORWARD, "swiglu", "256", 3303, 3, 200, 3336), (PACKING, "swiglu", "256", 3303, 3, 392, 3336),
         (WEIGHT, "none", "256", 900, 4, 2056, 2056), (WEIGHT, "swiglu", "256", 900, 4, 2056, 2056)]


def listed(*products):
    cases = [(p, act, form, *shape) for (p, act), forms in CASES.items() for form, shape in forms.items()]
    return [c for c in cases + WALKS if c[0] in products]


def plan(product, act, rows, E, K, N, dtype="bf16"):
    """The form that the library takes.  Host only, launches nothing."""
    fn = B.load_library().etr_packed_plan
    fn.restype, fn.argtypes = ctypes.c_int, [ctypes.POINTER(B.EtrLinearConfig), ctypes.c_int]
    return FORMS[fn(ctypes.byref(B.make_linear_config(rows, K, N, E, DT[dtype], act=ACT[act])), product)]
