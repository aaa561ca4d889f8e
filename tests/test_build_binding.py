"""The extension module of the binding: the library and what is called through ctypes do
without it."""
import os
import shutil
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PKG = "paper_2608_08684_gb300"


@pytest.fixture
def tree(lib, tmp_path):
    """A copy of the package with its built library, without the extension module."""
    skip = shutil.ignore_patterns("_build*", "libripple_checked.so", "_binding*.so", "__pycache__")
    shutil.copytree(os.path.join(ROOT, PKG), tmp_path / PKG, ignore=skip)
    shutil.copytree(os.path.join(ROOT, "include"), tmp_path / "include")
    return tmp_path


def _run(tree, code, **env):
    r = subprocess.run([sys.executable, "-c", code], cwd=tree, env=dict(os.environ, **env),
                       capture_output=True, text=True, timeout=600)
    assert r.returncode == 0, r.stdout + r.stderr
    return r.stdout.split()


def test_library_works_where_the_extension_module_cannot_be_built(tree):
    code = f"""
import warnings
from {PKG} import build
with warnings.catch_warnings(record=True) as w:
    warnings.simplefilter("always")
    build.build_library()
assert [x.category for x in w] == [RuntimeWarning] and "could not be built" in str(w[0].message)
from {PKG} import ripple as R
import torch
print(R.ripple_keep_count(10 ** 6, 100, 16))  # all rows
try:
    R.ripple_token_logprobs(torch.zeros(1, 3), entropy_out=torch.zeros(1))
except ImportError as e:
    print("unavailable" if "not built" in str(e) else e)
"""
    assert _run(tree, code, CXX="false") == ["100", "unavailable"]
