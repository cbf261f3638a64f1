"""The compiled marshalling of the cache's calls: who needs it, and when it is built again."""
import os
import shutil
import subprocess
import sys

import pytest

from conftest import ROOT


@pytest.fixture(scope="module")
def build():
    from paper_2407_11062_b200 import build
    build.build_library()
    return build


def run(tmp_path, code, module=None):
    """A process whose copy of the package has the library, and these bytes for the module."""
    package = tmp_path / "paper_2407_11062_b200"
    package.mkdir()
    for name in ("__init__.py", "binding.py", "build.py", "libeqat_b200.so"):
        shutil.copy(os.path.join(ROOT, "paper_2407_11062_b200", name), package)
    if module is not None:
        (package / "_marshal.so").write_bytes(module)
    return subprocess.run([sys.executable, "-c", code], cwd=tmp_path, capture_output=True, text=True)


def test_only_the_caches_calls_need_it(build, tmp_path):
    done = run(tmp_path, (
        "from paper_2407_11062_b200 import binding as e\n"
        "assert e.LIB_PATH.startswith(%r)\n"
        "print(e.lib.eqat_version() > 0)\n"
        "d = e.make_cache_desc(64, 64, 1, 16, 1, 1, 1, 1)\n"
        "print(e.cache_workspace_bytes(d, e.make_attention_desc(1, 1, 0.1)) >= 0)\n"
        "for call in (lambda: e.eqat_cache_append(d, *[None] * 6), lambda: e.eqat_cache_read(d, *[None] * 6),\n"
        "             lambda: e.eqat_cache_attention(d, None, *[None] * 6)):\n"
        "    try:\n"
        "        call()\n"
        "    except ImportError as x:\n"
        "        print('_marshal.so is missing' in str(x))\n") % str(tmp_path))
    assert done.returncode == 0 and done.stdout.split() == ["True"] * 5, (done.stdout, done.stderr[-600:])


def test_another_torch_or_python_builds_it_again_and_the_library_not(build, tmp_path, monkeypatch):
    assert build.marshal_fits() and not build._marshal_stale() and not build._stale()
    for tag in ("built for cpython-312, torch 1.0.", "built for cpython-399, torch 2.11.0."):
        monkeypatch.setattr(build, "marshal_tag", lambda: tag)
        assert not build.marshal_fits() and build._marshal_stale() and not build._stale()
    made = []
    monkeypatch.setattr(build, "_build_marshal", lambda: made.append(1))
    assert build.build_library() == build.LIB and made == [1]


def test_a_module_for_another_torch_is_refused(build, tmp_path):
    """Before it is loaded: its symbols may be missing or mean something else."""
    done = run(tmp_path, (
        "from paper_2407_11062_b200 import binding as e\n"
        "try:\n"
        "    e.eqat_cache_read(None, *[None] * 6)\n"
        "except ImportError as x:\n"
        "    print('another Python or torch' in str(x))\n"), b"built for cpython-312, torch 1.0.")
    assert done.returncode == 0 and done.stdout.split() == ["True"], (done.stdout, done.stderr[-600:])
