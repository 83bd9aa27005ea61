"""Every layout of the row operators through the LDS-poisoning debug build (run by
tests/test_gpu_rows_poison_layouts.py in a child process; argv[1] is a directory
holding a copy of the package whose library is that build)."""

import os
import sys

sys.path.insert(0, sys.argv[1])
sys.path.insert(1, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2608_21343_amd import capi  # noqa: E402
from tests import rows_layouts as L  # noqa: E402

assert os.path.dirname(str(capi.LIB_PATH)).startswith(sys.argv[1]), capi.LIB_PATH

for dtype, layout, C, n in L.cases(L.READ):
    print("read", L.name(dtype), L.name(layout), C, n, flush=True)
    L.check_scores(dtype, C, n)
    L.check_distill(dtype, C, n, True, grad=False)
for dtype, layout, C, n in L.cases(L.GRAD):
    print("gradient", L.name(dtype), L.name(layout), C, n, flush=True)
    L.check_grad(dtype, C, n)
    for tail in (False, True):
        L.check_distill(dtype, C, n, tail)
print("poison row layouts: ok", flush=True)
