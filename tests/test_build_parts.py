"""The library is built where only hipcc is there; the compiled marshalling needs more, and says what it misses."""
import pytest

from paper_2506_22771_amd import binding, build


@pytest.mark.parametrize("missing", ["g++", "Python's headers", "torch's headers"])
def test_a_build_without_what_the_marshalling_needs(tmp_path, monkeypatch, capsys, missing):
    stale = tmp_path / "_bind.so"
    stale.write_bytes(b"of an older library")
    monkeypatch.setattr(build, "BIND", str(stale))
    if missing == "g++":
        monkeypatch.setattr(build.shutil, "which", lambda name: None)
    elif missing == "Python's headers":
        monkeypatch.setattr(build.sysconfig, "get_paths", lambda: {"include": str(tmp_path)})
    else:
        monkeypatch.setattr(build.importlib.util, "find_spec", lambda name: None)
    monkeypatch.setattr(build.subprocess, "run", lambda *a, **k: pytest.fail("nothing is to be run"))
    build._build_bind(force=True)
    assert missing in capsys.readouterr().err and not stale.exists()


def test_nothing_is_missing_here_that_is_there():
    assert set(build._bind_needs()) == {"g++", "Python's headers", "torch's headers"}


def test_calls_without_the_marshalling_name_it(monkeypatch):
    import sys
    monkeypatch.setattr(binding, "_bind", None)
    monkeypatch.setattr(binding, "lib", lambda: None)
    monkeypatch.setitem(sys.modules, "paper_2506_22771_amd._bind", None)    # (an import of it fails)
    monkeypatch.delattr(sys.modules["paper_2506_22771_amd"], "_bind", raising=False)
    with pytest.raises(FileNotFoundError, match="_bind.so"):
        binding._native()
