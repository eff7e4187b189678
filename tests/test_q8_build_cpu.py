"""The extension module of the 8-bit wrappers is no condition of the library, and belongs to the torch it was built for."""
import os
import types

import pytest


def test_the_library_is_linked_without_the_extension_module(tmp_path, monkeypatch, capsys):
    from paper_2503_17707_amd import build as b

    lib, args = str(tmp_path / "lib.so"), str(tmp_path / "args.so")
    open(args, "w").close()  # of an earlier build: must not stay beside a newer library

    def run(cmd, **kw):
        assert cmd[0] != "g++"
        open(cmd[cmd.index("-o") + 1], "w").close()
        return types.SimpleNamespace(returncode=0, stdout="", stderr="")

    def no_headers():
        raise ImportError("no torch here")

    monkeypatch.setattr(b, "ROOT", str(tmp_path))
    monkeypatch.setattr(b, "LIB", lib)
    monkeypatch.setattr(b, "ARGS", args)
    monkeypatch.setattr(b.subprocess, "run", run)
    monkeypatch.setattr(b, "build_args", no_headers)
    assert b.build(out=lib) == lib
    assert os.path.exists(lib) and not os.path.exists(args)
    said = capsys.readouterr().err
    assert "args.so" in said and "no torch here" in said


def test_the_extension_module_is_for_one_torch(monkeypatch):
    import torch

    from paper_2503_17707_amd import binding as pb

    assert pb._q8_ready().TORCH == str(torch.__version__)
    monkeypatch.setattr(pb, "_q8", None)
    monkeypatch.setattr(torch, "__version__", "1.0.0")
    with pytest.raises(RuntimeError, match="torch"):
        pb._q8_ready()
    assert pb._q8 is None
