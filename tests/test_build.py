"""What the build leaves behind where a compiler is missing or fails: the library needs hipcc
alone, the tensor-table module is GradClip's, and neither failure leaves a process or a stale file.
The compilers are stand-ins that write their output files; nothing is compiled."""
import os
import stat

import pytest

from paper_2602_04940_amd import build


def _script(path, body):
    path.write_text("#!/bin/sh\n" + body)
    path.chmod(path.stat().st_mode | stat.S_IXUSR)
    return str(path)


# Writes "new" to the file after -o.
WRITE = 'while [ $# -gt 0 ]; do [ "$1" = -o ] && echo new > "$2"; shift; done\n'


@pytest.fixture
def tree(tmp_path, monkeypatch):
    lib, tensors = tmp_path / "lib.so", tmp_path / "tensors.so"
    for f in (lib, tensors):
        f.write_text("old\n")
    monkeypatch.setattr(build, "LIB", str(lib))
    monkeypatch.setattr(build, "TENSORS", str(tensors))
    bin_dir = tmp_path / "bin"
    bin_dir.mkdir()
    monkeypatch.setenv("PATH", f"{bin_dir}:/usr/bin:/bin")

    def tools(hipcc, gxx):
        _script(bin_dir / "hipcc", hipcc)
        if gxx is None:
            which = build.shutil.which
            monkeypatch.setattr(build.shutil, "which", lambda n: None if n == "g++" else which(n))
        else:
            _script(bin_dir / "g++", gxx)
    return lib, tensors, tools


def test_both_are_replaced(tree):
    lib, tensors, tools = tree
    tools(WRITE, WRITE)
    assert build.build_library() == str(lib)
    assert lib.read_text() == tensors.read_text() == "new\n"


@pytest.mark.parametrize("gxx", [None, "echo no headers; exit 1\n"])
def test_the_library_needs_no_host_compiler(tree, gxx):
    """hipcc ends after the other compiler has failed."""
    lib, tensors, tools = tree
    tools("sleep 0.5\n" + WRITE, gxx)
    with pytest.warns(UserWarning, match="GradClip"):
        assert build.build_library() == str(lib)
    assert lib.read_text() == "new\n" and not tensors.exists()


def test_a_failed_library_is_an_error_and_keeps_the_old_one(tree):
    lib, _, tools = tree
    tools("echo broken; exit 3\n", WRITE)
    with pytest.raises(RuntimeError, match="failed \\(3\\)(.|\n)*broken"):
        build.build_library()
    assert lib.read_text() == "old\n"


def test_no_compiler_outlives_the_build(tree, tmp_path):
    _, _, tools = tree
    tools(f"sleep 0.5\necho done > {tmp_path}/ended\nexit 1\n", None)
    with pytest.warns(UserWarning), pytest.raises(RuntimeError):
        build.build_library()
    assert os.path.exists(tmp_path / "ended")
