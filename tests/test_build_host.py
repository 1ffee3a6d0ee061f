"""The binding's host code is optional: the kernel library is built without it, and
one that exists but does not load is not passed over in silence."""
import subprocess
import sys
import warnings

import pytest

import paper_2607_01831_amd as package
from paper_2607_01831_amd import build, lynx


@pytest.mark.parametrize("error", [subprocess.CalledProcessError(1, "g++"), FileNotFoundError("g++")])
def test_the_library_is_built_where_the_host_code_is_not(monkeypatch, tmp_path, error):
    made = []

    def compiled(cmd, target, verbose):
        if target == build.ARGS:
            raise error
        made.append(target)
        return target

    monkeypatch.setattr(build, "ARGS", tmp_path / "_args.so")
    build.ARGS.write_bytes(b"of other sources")
    monkeypatch.setattr(build, "_compile", compiled)
    with pytest.warns(UserWarning, match="_args.so was not built"):
        assert build.build() == build.LIBRARY
    assert made == [build.LIBRARY] and not build.ARGS.exists()


def test_both_are_built(monkeypatch):
    made = []
    monkeypatch.setattr(build, "_compile", lambda cmd, target, verbose: made.append(target) or target)
    with warnings.catch_warnings():
        warnings.simplefilter("error")
        assert build.build() == build.LIBRARY
    assert made == [build.LIBRARY, build.ARGS]


def test_host_code_that_does_not_load_is_named(monkeypatch, tmp_path):
    monkeypatch.setattr(lynx, "ARGS", tmp_path / "_args.so")
    monkeypatch.setattr(lynx, "_args", None, raising=False)
    with warnings.catch_warnings():
        warnings.simplefilter("error")
        assert lynx._fastest_typed() is lynx._typed_form  # absent: nothing to say
    lynx.ARGS.write_bytes(b"")
    monkeypatch.delattr(package, "_args", raising=False)
    monkeypatch.setitem(sys.modules, package.__name__ + "._args", None)  # an import that fails
    with pytest.warns(RuntimeWarning, match="does not load"):
        assert lynx._fastest_typed() is lynx._typed_form
