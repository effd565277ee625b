"""The binding's module of the interpreter: compiled anew for another torch, named for its interpreter, missed with a word."""
import os
import sysconfig

import pytest
import torch


@pytest.fixture
def built(monkeypatch, tmp_path):
    """build.py on files of its own; the module's builds, counted."""
    from paper_2609_33390_gb300 import build
    count = []

    def fake(src):
        count.append(src)
        with open(build.MARSHAL, "w"):
            pass

    for name in ("MARSHAL", "MARSHAL_OF"):
        if hasattr(build, name):
            monkeypatch.setattr(build, name, str(tmp_path / os.path.basename(getattr(build, name))))
    monkeypatch.setattr(build, "build_marshal", fake)
    monkeypatch.setattr(build, "build_library", lambda *a: "library")
    return build, count


def test_another_torch_is_compiled_for_anew(built, monkeypatch):
    build, count = built
    assert build.build() == "library" and len(count) == 1
    build.build()
    assert len(count) == 1
    for version in ("9.8.7", "9.8.8"):
        monkeypatch.setattr(torch, "__version__", version)
        before = len(count)
        build.build()
        build.build()
        assert len(count) == before + 1, version


def test_a_build_that_fails_is_tried_again(built, monkeypatch):
    build, count = built
    build.build()
    monkeypatch.setattr(torch, "__version__", "9.8.7")

    def fails(src):
        raise RuntimeError("no compiler")

    with monkeypatch.context() as m:
        m.setattr(build, "build_marshal", fails)
        for _ in range(2):
            with pytest.raises(RuntimeError, match="no compiler"):
                build.build()
    build.build()
    assert len(count) == 2


def test_its_name_tells_the_interpreter(monkeypatch):
    from paper_2609_33390_gb300 import build
    build.build()
    assert os.path.basename(build.MARSHAL) == "_marshal" + sysconfig.get_config_var("EXT_SUFFIX")
    from paper_2609_33390_gb300 import _marshal
    assert os.path.samefile(_marshal.__file__, build.MARSHAL)


def test_a_missing_module_is_named(monkeypatch):
    import sys
    import paper_2609_33390_gb300 as package
    from paper_2609_33390_gb300 import brisk, build
    build.build()
    monkeypatch.delattr(package, "_marshal", raising=False)
    monkeypatch.setitem(sys.modules, package.__name__ + "._marshal", None)
    with pytest.raises(RuntimeError, match="_marshal is missing.*g.build()"):
        brisk.PackedAttention(1, 1, 1, 1, 16, 0, 4, torch.bfloat16, device="cpu")
    brisk.PrefixAttention(1, 1, 1, 1, 16, 0, 4, torch.bfloat16, device="cpu")
