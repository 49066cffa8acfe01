"""What the build does where only hipcc is at hand."""

import os
import stat

import pytest

from paper_2411_12692_amd import build


@pytest.fixture
def small(tmp_path, monkeypatch):
    """The build in a folder of its own, of no source, with a stand-in for hipcc."""
    hipcc = tmp_path / "hipcc"
    hipcc.write_text('#!/bin/sh\nwhile [ $# -gt 0 ]; do [ "$1" = -o ] && echo built > "$2"; shift; done\n')
    hipcc.chmod(hipcc.stat().st_mode | stat.S_IXUSR)
    for name, value in (("HIPCC", str(hipcc)), ("SOURCES", ["api.hip"]), ("BUILD", str(tmp_path / "_build")),
                        ("LIB", str(tmp_path / "lib.so")), ("AUTOGRAD_LIB", str(tmp_path / "_autograd.so"))):
        monkeypatch.setattr(build, name, value)
    return tmp_path


def test_nothing_is_missing_here():
    assert build.autograd_lacks() == ""


@pytest.mark.parametrize("what", ["compiler", "Python's headers", "PyTorch's headers"])
def test_the_library_is_built_without_what_the_nodes_need(small, monkeypatch, capfd, what):
    """The library is made, nodes of an older build are not left beside it, and it is said."""
    if what == "compiler":
        monkeypatch.setattr(build, "CXX", str(small / "none"))
    elif what == "Python's headers":
        monkeypatch.setattr(build.sysconfig, "get_paths", lambda: {"include": str(small)})
    else:
        from torch.utils import cpp_extension
        monkeypatch.setattr(cpp_extension, "include_paths", lambda: [str(small)])
    (small / "_autograd.so").write_text("old")
    path = build.build()
    assert path == str(small / "lib.so") and os.path.exists(path)
    assert not os.path.exists(build.AUTOGRAD_LIB)
    err = capfd.readouterr().err
    assert what in err and "gradients are not available" in err


def test_a_failing_build_of_the_nodes_is_an_error(small, monkeypatch):
    """Where all is at hand a failure is no reason to go without."""
    wrong = small / "cxx"
    wrong.write_text("#!/bin/sh\nexit 1\n")
    wrong.chmod(0o755)
    monkeypatch.setattr(build, "CXX", str(wrong))
    with pytest.raises(RuntimeError, match="command failed"):
        build.build()
