"""The CPython entry to the microscaled calls and the way through ctypes where it is not built (no GPU needed)."""
import os
import subprocess
import sys
import warnings

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture
def build(monkeypatch, tmp_path):
    """The build script with the module's path in a folder of its own, which holds one built from older sources."""
    from paper_2512_14090_b200 import build
    build.build()
    path = tmp_path / "_mxcall.so"
    path.write_bytes(b"built long ago")
    os.utime(path, (1, 1))
    monkeypatch.setattr(build, "CALL_PATH", str(path))
    return build


def test_a_module_of_the_present_sources_stays(build):
    os.utime(build.CALL_PATH)
    assert build.build_call() == build.CALL_PATH
    assert open(build.CALL_PATH, "rb").read() == b"built long ago"


def test_without_a_compiler_an_older_module_goes(build, monkeypatch):
    monkeypatch.setattr(build.shutil, "which", lambda name: None)
    assert build.build_call() is None
    assert not os.path.exists(build.CALL_PATH)


def test_a_compiler_that_fails_is_reported_and_an_older_module_goes(build, monkeypatch):
    monkeypatch.setattr(build.shutil, "which", lambda name: "/bin/false")
    with warnings.catch_warnings(record=True) as seen:
        warnings.simplefilter("always")
        assert build.build_call() is None
    assert any("ctypes" in str(w.message) for w in seen)
    assert not os.path.exists(build.CALL_PATH)


def test_the_module_is_built(build):
    import shutil
    if not (shutil.which("gcc") or shutil.which("cc")):
        pytest.skip("no C compiler")
    assert build.build_call() == build.CALL_PATH
    assert os.path.getsize(build.CALL_PATH) > 1000


def test_the_binding_without_the_module():
    code = ("import sys; sys.modules['paper_2512_14090_b200._mxcall'] = None\n"
            "from paper_2512_14090_b200 import binding as b\n"
            "assert b._mxcall is b.lib\n"
            "assert b.aiq_mx_row_bytes(129) == 128\n"
            "assert b._mxcall.aiq_mx_quantize(None, 0, 1, 32, 32, 4096, 4096, None) == b.ERR_INVALID_ARG\n")
    r = subprocess.run([sys.executable, "-c", code], cwd=ROOT, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
