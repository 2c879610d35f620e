"""The compiled argument checks belong to one torch and one Python: build() makes them anew for another, and the package refuses
a file that was built for another."""
import os
import shutil
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def entry():
    import __graft_entry__ as g
    g.build()
    return g


def test_built_for_this_torch(entry):
    import torch
    from paper_2508_15706_b200 import inner
    assert inner._checks.built_for == entry.checks_built_for() and torch.__version__ in entry.checks_built_for()
    assert not entry.checks_stale(entry.CHECKS, entry.checks_built_for())


def test_another_torch_makes_it_stale(entry, tmp_path):
    copy = str(tmp_path / "_checks.so")
    assert entry.checks_stale(copy, entry.checks_built_for())  # missing
    shutil.copy(entry.CHECKS, copy)
    assert not entry.checks_stale(copy, entry.checks_built_for())
    assert entry.checks_stale(copy, entry.checks_built_for().replace("torch ", "torch 9."))
    assert entry.checks_stale(copy, entry.checks_built_for()[:-1])  # (a name that begins like this one)


def test_import_refuses_a_file_for_another_torch(entry):
    code = "import torch; torch.__version__ = '9.9.9'; import paper_2508_15706_b200.inner"
    r = subprocess.run([sys.executable, "-c", code], cwd=ROOT, capture_output=True, text=True)
    assert r.returncode != 0 and "built for another torch" in r.stderr and "ImportError" in r.stderr
