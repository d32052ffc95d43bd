"""What the build does with and without torch; the compiler is not run."""
import sys

from paper_2505_06641_amd import build


def commands(monkeypatch):
    seen = []
    monkeypatch.setattr(build.subprocess, "run", lambda cmd, check: seen.append(cmd))
    assert build.build_library(verbose=False) == build.LIB
    return seen


def test_the_library_is_built_first_and_the_extension_behind_it(monkeypatch):
    library, extension = commands(monkeypatch)
    assert library[-1] == build.LIB and build.NATIVE in extension


def test_the_library_is_built_without_torch(monkeypatch):
    monkeypatch.setitem(sys.modules, "torch", None)            # as if it were not installed
    monkeypatch.setitem(sys.modules, "torch.utils", None)
    library, = commands(monkeypatch)
    assert library[-1] == build.LIB
