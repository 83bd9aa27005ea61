"""Row operators through the LDS-poisoning debug build, against their float64
forms (run by tests/test_gpu_rows_poison.py in a child process).

argv[1] is a directory holding a copy of the package whose library is the poison
build; it goes first on sys.path. Every layout runs once: one, two, four and
sixteen waves a row, cut rows, lists of few and many places, tokens listed
twice, rows of few different values."""

import os
import sys

sys.path.insert(0, sys.argv[1])
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(1, ROOT)

from paper_2608_21343_amd import capi  # noqa: E402
from tests import test_gpu_rows as T  # noqa: E402

assert os.path.dirname(str(capi.LIB_PATH)).startswith(sys.argv[1]), capi.LIB_PATH

for dtype, widths in ((T.F32, (2, 300, 1025, 2051, 4100, 8196, 20000, 65539, 70001)),
                      (T.BF16, (9, 300, 1025, 8193, 16000, 20000, 70001, 131073, 140001))):
    for C in widths:
        T.test_scores_at_every_width(dtype, C)
        T.test_gradients_at_every_width(dtype, C)
        for tail in (False, True):
            T.test_distill_at_every_width(dtype, C, tail)
        print(f"{T.ids(dtype)} {C}: ok", flush=True)
for dtype, C in ((T.F32, 1025), (T.BF16, 1025), (T.BF16, 9000), (T.F32, 70000)):
    T.test_ties_go_to_the_lowest_token(dtype, C)
    T.test_gradients_of_lists(dtype, C, 33)
    T.test_special_rows(dtype, C, 40)
    for tail in (False, True):
        T.test_distill_lists(dtype, C, 64, tail)
    print(f"lists {T.ids(dtype)} {C}: ok", flush=True)
print("poison rows: ok", flush=True)
