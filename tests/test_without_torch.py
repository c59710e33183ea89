"""The simulator without torch: it imports, loads and is built; only the
operators on torch tensors need torch."""
from __future__ import annotations

import os
import subprocess
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
BLOCK = "import sys; sys.modules['torch'] = None\n"  # import torch raises ImportError


def python(code):
    r = subprocess.run([sys.executable, "-c", code], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr
    return r.stdout.strip()


def test_simulator_imports_and_loads_without_torch():
    from paper_2606_10440_amd import sim
    if not os.path.exists(sim.LIB_PATH):
        from paper_2606_10440_amd import build
        build.build()
    assert python(BLOCK + "import paper_2606_10440_amd as p\np.sim.lib(); p.Simulator; p.SimError\nprint('ok')") == "ok"


def test_simulator_import_leaves_torch_alone():
    assert python("import sys, paper_2606_10440_amd\nprint('torch' in sys.modules)") == "False"


def test_operators_are_there_when_asked_for():
    assert python("import paper_2606_10440_amd as p\nprint(p.ops.Mx4.__name__)") == "Mx4"
    assert python("from paper_2606_10440_amd import ops\nprint(ops.Mx4.__name__)") == "Mx4"
    assert python("import paper_2606_10440_amd as p\nprint(hasattr(p, 'opss'))") == "False"
    assert python(BLOCK + "import paper_2606_10440_amd as p\ntry:\n    p.ops\nexcept ImportError:\n    print('no torch')") == "no torch"


def test_build_without_torch_takes_the_library_alone():
    # the commands and the files that it would move, in place of a compilation
    assert python(BLOCK + """
import os
from paper_2606_10440_amd import build as b
cmds, moved = [], []
b._run = lambda cmd, verbose: cmds.append(cmd)
b.os.replace = lambda a, c: moved.append(c)
assert b.build() == b.LIB
assert moved == [b.LIB] and len(cmds) == len(b.SOURCES) + 1
assert not any('ops_torch.cpp' in w for c in cmds for w in c)
print('ok')""") == "ok"
