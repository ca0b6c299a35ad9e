"""The marshalling extension of the calls around the paged cache is loaded by those calls alone."""
import pytest
import torch

from paper_2510_25739_b200 import binding, build


def test_the_library_loads_without_the_extension(monkeypatch, tmp_path):
    build.build()
    monkeypatch.setattr(binding, "_lib", None)
    monkeypatch.setattr(binding, "_marshal", None)
    monkeypatch.setattr(binding, "_MARSHAL_PATH", tmp_path / "_hawk_marshal.so")
    lib = binding.load_library()
    assert lib.hawk_version() and binding.spec_cache_slots(4, 3) > 0
    with binding.alternate_library(build.LIB):
        assert binding.spec_cache_slots(4, 3) > 0
    for call in (lambda: binding.qk_norm_rope(None, None, None, None), lambda: binding.paged_attn(*[None] * 9),
                 lambda: binding.rope_append(*[None] * 10)):
        with pytest.raises(RuntimeError, match="_hawk_marshal.* is missing"):
            call()


def test_the_first_call_loads_it(monkeypatch):
    build.build()
    monkeypatch.setattr(binding, "_marshal", None)
    with pytest.raises(ValueError, match="one of them"):
        binding.qk_norm_rope(None, None, None, None)
    assert binding._marshal is not None


def test_the_extension_is_rebuilt_for_another_torch(monkeypatch, tmp_path):
    build.build()
    made = []

    def compiler(cmd, **_):
        made.append(cmd)
        open(cmd[cmd.index("-o") + 1], "w").close()
        return type("Done", (), {"returncode": 0})()

    monkeypatch.setattr(build, "MARSHAL_LIB", tmp_path / "_hawk_marshal.so")
    monkeypatch.setattr(build, "MARSHAL_TAG", tmp_path / "b" / "marshal.txt")
    monkeypatch.setattr(build.subprocess, "run", compiler)
    build.build_marshal()
    build.build_marshal()
    assert len(made) == 1
    monkeypatch.setattr(torch, "__version__", "9.0.1+cu999")
    build.build_marshal()
    build.build_marshal()
    assert len(made) == 2


def test_an_extension_of_another_torch_is_not_called(monkeypatch):
    build.build()
    monkeypatch.setattr(binding, "_marshal", None)
    monkeypatch.setattr(binding.torch, "__version__", "9.0.1+cu999")
    with pytest.raises(RuntimeError, match="was built for torch .* this is 9.0.1"):
        binding.qk_norm_rope(None, None, None, None)
    assert binding._marshal is None
