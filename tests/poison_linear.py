"""The output layer's cross entropy through the LDS-poisoning debug build, against its
float64 form (run by tests/test_gpu_linear_poison.py in a child process).

argv[1] is a directory holding a copy of the package whose library is the poison
build; it goes first on sys.path."""

import os
import sys

sys.path.insert(0, sys.argv[1])
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(1, ROOT)

from paper_2608_21343_amd import capi  # noqa: E402
from tests import test_gpu_adamw as A  # noqa: E402
from tests import test_gpu_linear as T  # noqa: E402
from tests import test_gpu_linear_tiles as G  # noqa: E402

assert os.path.dirname(str(capi.LIB_PATH)).startswith(sys.argv[1]), capi.LIB_PATH

for dtype in (T.F32, T.BF16):
    for sizes in T.SIZES:
        T.test_sizes(*sizes, dtype)
    print(f"{dtype} sizes: ok", flush=True)
    for sizes in G.TILES + G.FEW:
        G.test_in_one_call_and_in_two(*sizes, dtype)
    print(f"{dtype} tiles: ok", flush=True)
    T.test_masked_tokens(dtype)
    T.test_rows_left_out_hold_anything(dtype)
for kind in A.KINDS:
    A.test_every_bit(*kind, 1)
A.test_moments(3)
print("poison linear: ok", flush=True)
