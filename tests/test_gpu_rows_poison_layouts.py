"""No layout of the row operators reads an LDS word that it has not written: the
checks of tests/rows_layouts.py through the LDS-poisoning debug build, in a
child process (tests/poison_row_layouts.py) that imports the package from a
temporary copy with that library."""

import os
import shutil
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PKG = os.path.join(ROOT, "paper_2608_21343_amd")


def test_lds_poison_build_in_every_layout(tmp_path):
    lib = os.path.join(PKG, "libtbias_poison.so")
    if not os.path.exists(lib):
        pytest.skip("libtbias_poison.so is not built (python -m paper_2608_21343_amd.build --poison)")
    dst = tmp_path / "paper_2608_21343_amd"
    dst.mkdir()
    for f in os.listdir(PKG):
        if f.endswith(".py"):
            shutil.copy(os.path.join(PKG, f), dst / f)
    shutil.copy(lib, dst / "libtbias.so")
    r = subprocess.run([sys.executable, "-u", os.path.join(ROOT, "tests", "poison_row_layouts.py"),
                        str(tmp_path)], capture_output=True, text=True, timeout=600)
    print(r.stdout[-3000:])
    assert r.returncode == 0, (r.stdout[-4000:], r.stderr[-4000:])
    assert "poison row layouts: ok" in r.stdout
