"""What the package needs to be imported: numpy and libpahq.so for the counts, ids and sizes; torch at the first use of what takes
tensors."""
import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
NAMES = ("Mx4", "mx4_quantize", "mx4_dequantize", "mx4_gemm", "rotary_table", "rotary")


def run(code):
    got = subprocess.run([sys.executable, "-c", code], cwd=ROOT, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    assert got.returncode == 0, got.stdout


def test_the_package_without_torch():
    run("import sys; sys.modules['torch'] = None\n"
        "import paper_2510_23264_amd as P\n"
        "assert P.lib() and len(P.rotary_entries(64)) == 32\n"
        "assert len(P.tau_grid()) == 21\n"
        "try: P.mx4_gemm\n"
        "except ImportError: pass\n"
        "else: raise AssertionError('torch came from somewhere')\n"
        "from paper_2510_23264_amd import *\n"
        "assert n_senders and Model\n")


def test_importing_it_does_not_import_torch():
    run("import sys, paper_2510_23264_amd as P\n"
        "assert 'torch' not in sys.modules\n"
        "assert set(%r) <= set(dir(P))\n"
        "assert P.lib() and 'torch' not in sys.modules\n"
        "assert P.rotary is P.tensors.rotary and P.Mx4 is P.tensors.Mx4 and 'torch' in sys.modules\n"
        "try: P.no_such_name\n"
        "except AttributeError: pass\n"
        "else: raise AssertionError\n" % (NAMES,))


def test_all_its_names():
    run("from paper_2510_23264_amd import *\n"
        "import paper_2510_23264_amd.tensors as t\n"
        "assert all(globals()[n] is getattr(t, n) for n in %r) and Model and lib\n"
        "from paper_2510_23264_amd import rotary, Mx4\n" % (NAMES,))


def test_the_build_check_loads_the_extension():
    run("import __graft_entry__ as g\n"
        "from paper_2510_23264_amd import build\n"
        "build.build = lambda **how: None\n"
        "g.build()\n")


@pytest.mark.parametrize("first", ["P.lib()", "import torch", "P.n_senders", "P.mx4_gemm"])
def test_one_hip_runtime_whatever_is_loaded_first(first):
    run("import re, paper_2510_23264_amd as P\n"
        "%s\n"
        "P.lib()\n"
        "import torch\n"
        "from paper_2510_23264_amd import _tensors\n"
        "maps = open('/proc/self/maps').read()\n"
        "assert 'libpahq.so' in maps and '_tensors.so' in maps\n"
        "for name in ('libamdhip64', 'libhsa-runtime64'):\n"
        "    found = set(re.findall(r'/\\S*/' + name + r'\\S*', maps))\n"
        "    assert len(found) == 1, found\n" % first)
