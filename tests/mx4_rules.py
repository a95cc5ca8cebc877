"""The rules of csrc/mx4_rules.h once more, for GPU tests that have to know which kernel a product takes
(test_mx4_rules.py holds the two together)."""
import math

FEW, T32, T64_FOUR, T64_TWO, T128, T256 = range(-1, 5)
# tile, groups, launch, start, slab, round, whole
FORMS = [(32, 4, 3.2, 0.4, 0.31, 1.5, False), (64, 4, 3.6, 1.2, 0.54, 2.4, True), (64, 2, 2.8, 1.9, 0.61, 0.8, False), (128, 1, 1.1, 4.5, 0.85, 0.6, False),
         (256, 1, 4.0, 8.9, 1.53, 1.27, True)]


def estimate(form, m, n, slabs):
    tile, groups, launch, start, slab, each, whole = form
    r = -(-m // tile) * -(-n // tile) / 256
    further = 0 if r <= 1 else 0.5 * (math.ceil(r) + r) - 1 if whole else r - 1
    return launch + (start + slab * -(-slabs // groups)) * (1 + each * further)


def form(m, n, k):
    slabs = -(-k // 256)
    if m <= 16 and (m <= 4 or n < 4000 or slabs < 10):
        return FEW
    return min(range(5), key=lambda i: estimate(FORMS[i], m, n, slabs))
