"""The binding's helper is something that a machine without torch's headers, or without a C++ compiler, does without."""
import os
import sys

import pytest

import __graft_entry__ as entry


@pytest.mark.parametrize("compiler", ["false", os.path.join(os.sep, "nowhere", "g++")])
def test_build_goes_on_without_the_helper(monkeypatch, tmp_path, capfd, compiler):
    monkeypatch.setenv("CXX", compiler)
    tmp, out = str(tmp_path / "helper.tmp"), str(tmp_path / "helper.so")
    with open(out, "w") as f:
        f.write("one of an older source")
    assert not entry.finish_tables(entry.start_tables(tmp), tmp, out)
    assert "not built" in capfd.readouterr().err
    assert not os.path.exists(out) and not os.path.exists(tmp)


def test_build_goes_on_without_the_headers(monkeypatch, tmp_path, capfd):
    def missing(out):
        raise ImportError("no torch.utils.cpp_extension")
    monkeypatch.setattr(entry, "tables_command", missing)
    assert not entry.finish_tables(entry.start_tables(str(tmp_path / "t")), str(tmp_path / "t"), str(tmp_path / "o"))
    assert "cpp_extension" in capfd.readouterr().err


def test_helper_that_is_built_takes_its_place(monkeypatch, tmp_path):
    tmp, out = str(tmp_path / "t"), str(tmp_path / "o")
    monkeypatch.setattr(entry, "tables_command", lambda o: [sys.executable, "-c", "open(%r, 'w').write('built')" % o])
    assert entry.finish_tables(entry.start_tables(tmp), tmp, out)
    with open(out) as f:
        assert f.read() == "built"
    assert not os.path.exists(tmp)
