"""The extension module of the binding: the library and what is called through ctypes do
without it, and one that was built for another Python or PyTorch is neither loaded nor taken
for the present one."""
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
    return _copy(tmp_path, "_binding*.so")


@pytest.fixture
def built(lib, tmp_path):
    """The same with the extension module."""
    return _copy(tmp_path)


def _copy(to, *without):
    skip = shutil.ignore_patterns("_build*", "libripple_checked.so", "__pycache__", *without)
    shutil.copytree(os.path.join(ROOT, PKG), to / PKG, ignore=skip)
    shutil.copytree(os.path.join(ROOT, "include"), to / "include")
    return to


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


CALL = f"""
from {PKG} import ripple as R
try:
    R.ripple_token_logprobs(torch.zeros(1, 3), entropy_out=torch.zeros(1))
except ImportError as e:
    print("unavailable" if "not built" in str(e) else e)
except ValueError:
    print("loaded")  # and refuses host tensors
"""


def test_present_versions_load(built):
    assert _run(built, "import torch" + CALL) == ["loaded"]


@pytest.mark.parametrize("other", [
    "torch.__version__ = torch.version.__version__ = '0.1.2+other'",
    "torch.version.git_version = '0123456789abcdef'",
    "import sysconfig; sysconfig.get_config_vars()['SOABI'] = 'cpython-0-other'",
])
def test_a_module_for_other_versions_is_not_taken(built, other):
    code = f"import torch\n{other}\n"
    assert _run(built, code + CALL) == ["unavailable"]
    # and the build makes one for the present ones instead of keeping it (here: tries to)
    build = f"""
from {PKG} import build
try:
    print(build.build_binding())
except RuntimeError as e:
    print("built anew" if "compile failed" in str(e) else e)
"""
    assert _run(built, code + build, CXX="false") == ["built", "anew"]


def test_builds_at_the_same_time_do_not_share_a_file(built):
    # every compiler call writes a file of its own and leaves nothing behind when it fails
    code = f"""
import subprocess
from {PKG} import build
seen = []
def run(cmd, **kw):
    seen.append(cmd[cmd.index("-o") + 1])
    open(seen[-1], "w").close()
    return subprocess.CompletedProcess(cmd, 1, "", "")
build.subprocess.run = run
try:
    build.build_binding(force=True)
except RuntimeError:
    print(seen[0])
"""
    first, second = (_run(built, code)[0] for _ in range(2))
    assert first != second and not os.path.exists(first) and not os.path.exists(second)
