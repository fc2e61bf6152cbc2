"""What an import of the package says where a native module is not built (no GPU)."""
import os
import shutil
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
NAME = "paper_2608_11742_amd"
BUILT = ("libdllm_rps.so", "_marshal.so")


@pytest.mark.parametrize("missing", [BUILT, BUILT[:1], BUILT[1:]], ids="+".join)
def test_import_of_an_unbuilt_tree_says_how_to_build(tmp_path, missing):
    source, there = os.path.join(ROOT, NAME), tmp_path / NAME
    if not all(os.path.exists(os.path.join(source, f)) for f in BUILT if f not in missing):
        pytest.skip("not built")
    there.mkdir()
    for f in os.listdir(source):
        if f.endswith(".py") or (f in BUILT and f not in missing):
            shutil.copy(os.path.join(source, f), there)
    r = subprocess.run([sys.executable, "-c", f"import {NAME}"], cwd=tmp_path, capture_output=True, text=True, timeout=300)
    assert r.returncode != 0
    last = r.stderr.strip().splitlines()[-1]
    assert last.startswith("ImportError: ") and missing[0] in last and "is missing" in last and "__graft_entry__" in last, last
