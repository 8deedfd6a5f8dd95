"""The build of the library and of the module over it (no compiler runs here)."""
import pytest

from paper_2411_01238_amd import build


def test_the_library_is_linked_where_the_module_does_not_compile(monkeypatch):
    links = []

    def no_torch_headers():
        raise RuntimeError("no headers")

    monkeypatch.setattr(build, "_compile", lambda unit: unit[1])
    monkeypatch.setattr(build, "_compile_native", no_torch_headers)
    monkeypatch.setattr(build.subprocess, "check_call", links.append)
    with pytest.raises(RuntimeError, match="no headers"):
        build.build(verbose=False)
    assert len(links) == 1 and build.LIB in links[0] and all(u[1] in links[0] for u in build.UNITS)
