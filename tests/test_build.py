"""What build() makes where torch, or what it takes to build against it, is not there."""
import os

import pytest

from paper_2606_03770_gb300 import build as B


@pytest.fixture
def elsewhere(tmp_path, monkeypatch):
    """An empty place to build in, and a library of one short file."""
    for name in ("LIB", "BINDING", "BUILT_FOR"):
        monkeypatch.setattr(B, name, str(tmp_path / os.path.basename(getattr(B, name))))
    monkeypatch.setattr(B, "OUT_DIR", str(tmp_path))
    monkeypatch.setattr(B, "sources", lambda: [os.path.join(B.CSRC, "ops_common.cu")])
    return tmp_path


def test_without_torch(elsewhere, monkeypatch):
    monkeypatch.setattr(B.importlib.util, "find_spec", lambda name: None)
    B.build()
    B.build()
    assert sorted(p.name for p in elsewhere.iterdir()) == ["libe2ga.so", "ops_common.o"]


def test_with_a_torch_that_the_module_does_not_build_against(elsewhere, monkeypatch):
    (elsewhere / "torch").mkdir()
    (elsewhere / "torch" / "version.py").write_text("__version__ = '0.1'\n")
    monkeypatch.setattr(B, "_torch", lambda: str(elsewhere / "torch"))
    with pytest.warns(UserWarning, match="e2binding.so was not built"):
        B.build()
    assert os.path.exists(B.LIB) and not os.path.exists(B.BINDING) and B.binding_built_for() is None
    assert B.binding_for().endswith("torch 0.1")


def test_another_torch_takes_another_module(elsewhere, monkeypatch):
    monkeypatch.setattr(B, "_build_library", lambda *a: open(B.LIB, "w").close())
    monkeypatch.setattr(B, "_compile_binding", lambda: built.append(B.binding_for()) or ["-shared", "-x", "c", os.devnull])
    built = []
    for version in ("a", "a", "b"):
        monkeypatch.setattr(B, "binding_for", lambda: version)
        B.build()
        assert B.binding_built_for() == version
    assert built == ["a", "b"]
    # (one that fails does not leave the older one to be loaded)
    monkeypatch.setattr(B, "binding_for", lambda: "c")
    monkeypatch.setattr(B, "_compile_binding", lambda: ["-shared", "no such file"])
    with pytest.warns(UserWarning, match="not built"):
        B.build()
    assert B.binding_built_for() is None


def test_calls_without_the_module(monkeypatch):
    torch = pytest.importorskip("torch")
    from paper_2606_03770_gb300 import ops
    if not os.path.exists(B.LIB):
        pytest.skip("the library is not built")
    monkeypatch.setattr(ops, "_binding", None)
    for built_for in (None, "another"):
        monkeypatch.setattr(B, "binding_built_for", lambda: built_for)
        with pytest.warns(UserWarning, match="e2binding.so"):
            b = ops.binding()
        assert b.verify() is b.attend_tree(1, 2) is b.keep() is None
        assert ops.binding() is b                             # (said once)
        with pytest.raises(ValueError, match="on the GPU"):
            ops.verify_drafts(torch.zeros(2, 8), *[torch.zeros(2, dtype=torch.int32)] * 3, torch.zeros(2))
        monkeypatch.setattr(ops, "_binding", None)
