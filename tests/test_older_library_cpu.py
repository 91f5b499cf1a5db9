"""binding.py beside a libcottn.so that was built before the calls with a decay and the tree calls: it imports, the calls that
the library has are made, and one that it lacks raises where it is made and names the function."""
import os
import re
import shutil
import subprocess
import sys

import paper_2409_18747_amd.binding as binding

HERE = os.path.dirname(binding.library_path)
LATER = ["cottn_fwd_causal_decay", "cottn_bwd_causal_decay", "cottn_step_decay", "cottn_tree", "cottn_tree_accept"]

PROGRAM = """
import warnings
warnings.simplefilter("ignore")   # (that _marshal.so is not there)
import torch
import paper_2409_18747_amd.binding as b
assert b.cottn_workspace_bytes(b.OP_FWD_CAUSAL, 1, 2, 4096, 64) == 77
for name in {later!r}:
    try:
        getattr(b.lib, name)
    except AttributeError as e:
        assert name in str(e), e
    else:
        raise AssertionError("found")
x = torch.zeros(1, 2, 64)
try:
    b.cottn_step_decay(x, x, x, torch.ones(2), None, torch.zeros(1, 2, 64, 64))
except ValueError as e:
    assert "must live on the GPU" in str(e), e
else:
    raise AssertionError("accepted")
"""


def test_it_imports_and_makes_the_calls_that_are_there(tmp_path):
    with open(os.path.join(HERE, "..", "include", "cottn.h")) as f:
        names = sorted(set(re.findall(r"\b(cottn_[a-z0-9_]+)\(", re.sub(r"/\*.*?\*/", "", f.read(), flags=re.S))))
    assert set(LATER) < set(names)
    package = tmp_path / "paper_2409_18747_amd"
    package.mkdir()
    for name in ("__init__.py", "binding.py", "build.py"):
        shutil.copy(os.path.join(HERE, name), package / name)
    src = tmp_path / "older.cpp"
    src.write_text('extern "C" {\n' + "".join("unsigned long %s() { return 77; }\n" % n for n in names if n not in LATER) + "}\n")
    subprocess.run(["g++", "-shared", "-fPIC", str(src), "-o", str(package / "libcottn.so")], check=True)
    done = subprocess.run([sys.executable, "-c", PROGRAM.format(later=LATER)], cwd=tmp_path, capture_output=True, text=True)
    assert done.returncode == 0, done.stderr
