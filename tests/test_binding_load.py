"""The library is usable without the compiled calls (csrc/torch_calls.cpp), which only shorten some of them."""
import os
import subprocess
import sys
import types

import pytest

import paper_2506_05632_b200 as gls

PKG = "paper_2506_05632_b200"
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _run(code, cwd, **env):
    """(exit code, output) of a Python program in a tree of its own."""
    e = dict(os.environ, PYTHONPATH=str(cwd), PYTHONDONTWRITEBYTECODE="1", **env)
    p = subprocess.run([sys.executable, "-c", code], cwd=cwd, env=e, capture_output=True, text=True, timeout=300)
    return p.returncode, p.stdout + p.stderr


@pytest.fixture
def tree(tmp_path):
    """A tree of links to this one's package and header, with libgls.so and without the compiled calls."""
    gls.load()
    (tmp_path / PKG).mkdir()
    (tmp_path / "include").symlink_to(os.path.join(ROOT, "include"))
    for f in os.listdir(os.path.join(ROOT, PKG)):
        if f != "__pycache__" and not f.startswith("gls_torch_calls"):
            (tmp_path / PKG / f).symlink_to(os.path.join(ROOT, PKG, f))
    return tmp_path


USE = """
import warnings
import paper_2506_05632_b200 as gls, torch
with warnings.catch_warnings(record=True) as said:
    warnings.simplefilter("always")
    assert gls.version() >= 210
    assert [w.category for w in said if "ctypes" in str(w.message)] == [RuntimeWarning], said
try:  # the general way takes the call, and refuses this one
    gls.embed_tokens(torch.zeros(3, 2), torch.zeros(1, dtype=torch.int32))
except gls.GlsError as e:
    assert "device" in str(e)
    print("usable")
"""


def test_a_spoilt_module(tree):
    rc, out = _run("from paper_2506_05632_b200 import binding as b; open(b._CALLS_LIB, 'wb').write(b'not a library')", tree)
    assert rc == 0, out
    rc, out = _run(USE, tree)
    assert rc == 0 and "usable" in out, out


def test_no_host_compiler(tree):
    rc, out = _run(USE, tree, CXX=str(tree / "no-such-compiler"))
    assert rc == 0 and "usable" in out, out


def test_a_module_of_another_torch_is_not_taken(tree):
    name = "import torch%s; from paper_2506_05632_b200 import binding as b; print(b._CALLS_LIB)"
    names = {_run(name % v, tree)[1] for v in ("", "; torch.__version__ = '1.0'", "; torch.version.cuda = '1.0'")}
    assert len(names) == 3, names


def test_this_tree_has_the_module():
    gls.load()
    assert isinstance(gls.binding._calls, types.ModuleType)
