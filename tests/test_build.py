"""The build's own decisions, with the compilers replaced by fakes (no GPU, nothing is compiled)."""
import os

import pytest

from paper_2605_25655_b200 import _build


@pytest.fixture
def fakes(monkeypatch, tmp_path):
    """Targets in a scratch folder and a Popen that writes its target, or fails for the names in `broken`."""
    for name in ("LIB", "LIB_BF16", "OPS"):
        monkeypatch.setattr(_build, name, str(tmp_path / os.path.basename(getattr(_build, name))))
    monkeypatch.setattr(_build, "OPS_TORCH", str(tmp_path / "version"), raising=False)
    monkeypatch.setattr(_build, "VARIANTS", ((_build.LIB, []), (_build.LIB_BF16, ["-DTHINFER_BF16"])))
    monkeypatch.setattr(_build, "_nvcc", lambda: "nvcc")
    state = {"broken": set(), "missing": set(), "run": []}

    class Popen:
        def __init__(self, cmd, **_):
            self.target = cmd[cmd.index("-o") + 1]
            self.name = os.path.basename(self.target)
            if self.name in state["missing"]:
                raise FileNotFoundError(cmd[0])
            state["run"].append(self.name)
            self.returncode = None

        def communicate(self):
            self.returncode = int(self.name in state["broken"])
            if not self.returncode:
                with open(self.target, "w"):
                    pass
            return "text of the compiler", None

    monkeypatch.setattr(_build.subprocess, "Popen", Popen)
    monkeypatch.setattr(_build, "_ops_command", lambda: ["g++", "-o", _build.OPS])
    return state


BOTH = ["libthinfer.so", "libthinfer_bf16.so"]


def test_without_torch_the_libraries_alone_are_built(fakes, monkeypatch):
    monkeypatch.setattr(_build, "_torch_version", lambda: None)
    assert _build.is_stale()
    assert _build.build() == _build.LIB and fakes["run"] == BOTH and not _build.is_stale()
    assert _build.build() == _build.LIB and fakes["run"] == BOTH


@pytest.mark.parametrize("how", ["broken", "missing"])
def test_a_module_that_cannot_be_compiled_leaves_the_libraries(fakes, how):
    fakes[how].add("_ops.so")
    with pytest.raises(RuntimeError) as e:
        _build.build()
    assert "_ops.so" in str(e.value) and os.path.exists(_build.LIB) and os.path.exists(_build.LIB_BF16)
    assert not _build.is_stale(_build.LIB) and _build.is_stale()


def test_every_failure_is_told(fakes):
    fakes["broken"].update(["libthinfer.so", "_ops.so"])
    with pytest.raises(RuntimeError) as e:
        _build.build()
    assert "libthinfer.so" in str(e.value) and "_ops.so" in str(e.value) and os.path.exists(_build.LIB_BF16)


def test_another_torch_makes_the_module_stale(fakes, monkeypatch):
    monkeypatch.setattr(_build, "_torch_version", lambda: "1.2.3")
    _build.build()
    assert not _build.is_stale() and fakes["run"] == BOTH + ["_ops.so"]
    monkeypatch.setattr(_build, "_torch_version", lambda: "1.2.4")
    assert _build.is_stale()
    _build.build()
    assert fakes["run"] == BOTH + ["_ops.so"] * 2 and not _build.is_stale()


def test_a_module_for_another_torch_is_not_loaded(monkeypatch, tmp_path):
    from paper_2605_25655_b200 import thinfer
    _build.build()
    note = tmp_path / "version"
    note.write_text("0.0.1\n")
    monkeypatch.setattr(_build, "OPS_TORCH", str(note), raising=False)
    monkeypatch.setattr(thinfer, "_fast", None)
    with pytest.raises(thinfer.ThinferError) as e:
        thinfer._load_fast()
    assert "0.0.1" in str(e.value)
