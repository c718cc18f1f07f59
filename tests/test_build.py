"""What is built where not everything can be (stand-ins for the compilers; no GPU, no nvcc needed)."""
import os
import stat
import sys

import pytest

from paper_2603_09215_b200 import build

MAKES = '#!/bin/sh\nwhile [ "$1" != -o ]; do shift; done\n: > "$2"\n'
FAILS = "#!/bin/sh\nexit 3\n"


@pytest.fixture
def tools(tmp_path, monkeypatch):
    def put(**scripts):
        for name, text in scripts.items():
            p = tmp_path / name.replace("gxx", "g++")
            p.write_text(text)
            p.chmod(p.stat().st_mode | stat.S_IEXEC)
    monkeypatch.setenv("PATH", f"{tmp_path}{os.pathsep}/usr/bin{os.pathsep}/bin")
    monkeypatch.setattr(build, "LIB", str(tmp_path / "libsparsk.so"))
    monkeypatch.setattr(build, "PAGED", str(tmp_path / "_paged.so"))
    return put


def test_both_are_built(tools):
    tools(nvcc=MAKES, gxx=MAKES)
    assert build._stale() and build.build() == build.LIB
    assert os.path.exists(build.LIB) and os.path.exists(build.PAGED) and not build._stale()


def test_the_library_is_built_where_the_marshalling_is_not(tools):
    tools(nvcc=MAKES, gxx=FAILS)
    with pytest.raises(RuntimeError, match="is built, but"):
        build.build()
    assert os.path.exists(build.LIB) and not os.path.exists(build.PAGED) and build._stale()


def test_the_library_is_built_without_torch(tools, monkeypatch):
    tools(nvcc=MAKES, gxx=FAILS)
    monkeypatch.setitem(sys.modules, "torch", None)
    assert build._stale() and build.build() == build.LIB and os.path.exists(build.LIB) and not build._stale()


def test_a_library_that_does_not_build_is_an_error(tools):
    tools(nvcc=FAILS, gxx=MAKES)
    with pytest.raises(Exception):
        build.build()
    assert not os.path.exists(build.LIB)
