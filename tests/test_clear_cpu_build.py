"""The binding's reader of tensor lists is built for the torch that is loaded, and the C library without it."""
import pytest

torch = pytest.importorskip("torch")

from paper_2504_17785_amd import build, clear  # noqa: E402


def test_a_reader_built_for_another_torch_is_not_loaded(monkeypatch):
    asked = []

    def stub():
        asked.append(torch.__version__)
        raise RuntimeError("no compiler")

    monkeypatch.setattr(build, "_build_tensors", stub)
    monkeypatch.setattr(torch, "__version__", "0.0.1+other")
    clear._tensors.cache_clear()
    try:
        with pytest.raises(RuntimeError, match="no compiler"):
            clear._tensors()
        assert asked == ["0.0.1+other"]
    finally:
        clear._tensors.cache_clear()


def test_the_c_library_is_built_where_the_reader_cannot_be(monkeypatch, tmp_path):
    def no_headers():
        raise RuntimeError("no headers")

    linked = []
    monkeypatch.setattr(build, "_build_tensors", no_headers)
    monkeypatch.setattr(build, "_compile", lambda src: src)
    monkeypatch.setattr(build, "LIB", str(tmp_path / "lib.so"))

    def link(cmd):
        linked.append(cmd)
        with open(cmd[cmd.index("-o") + 1], "w") as f:
            f.write("library")

    monkeypatch.setattr(build.subprocess, "check_call", link)
    # it says so, and leaves the library behind
    with pytest.raises(RuntimeError, match="no headers"):
        build.build()
    assert len(linked) == 1 and (tmp_path / "lib.so").read_text() == "library"
